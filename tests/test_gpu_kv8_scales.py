"""The attention over the 8-bit cache where value scales lie far apart.

Bar.  Everything is taken over the keys that the row sees, and no others: S = max scale ks sum_d |q_d k_d|, A = sum p_j |v_j| / sum p_j, W the weight that the
kernel's roundings are relative to.  Scores in FP32 are off by at most 2^-23 (D + 4) S + 2^-21, the exponential included (derived in test_gpu_kv8.py), and by what a
query loses: 2^-22 of its row's largest magnitude in each number (24-bit fixed point; f16 loses less), so
   E = 2^-23 (D + 4) S + 2^-21 + 2^-22 max |q_d| max scale ks sum_d |k_d|
Weights p_j vs_j:
   up to 32 rows a sequence and key-value head: 24 bits of the largest among 128 tokens, off by 2^-25 W with W = max p_j vs_j;
   more: f16, off by 2^-11 of each, or by half of f16's smallest step, 2^-25, where 2^5 or more stands for max p times max vs: 2^-25 W with W = 2^-5 max p max vs.
n keys move the numerator by at most n 2^-25 W 127.  The sum of the exponentials is relative to a number that is at most 2^60 away from the largest, which FP32
bears.  So, with the result's own rounding to bf16:
   |out - o| <= 2^-8 |o| + (2^-11 + 2 E + 2^-20) A + n 2^-25 127 W / sum p_j
   |lse - exact| <= E + 2^-22 |exact| + 2^-21
"""
import pytest
import torch

from test_gpu_kv8 import Batch, b, queries, visible64  # noqa: F401

pytestmark = pytest.mark.gpu


def check_rows(b, s, q, few):  # noqa: F811
    """The call's output and log-sum, and their distance from the definition row by row."""
    G = q.shape[1] // s.H
    s.device(b)
    ws = b.alloc_attn_workspace(s.cache, s.H * G, "cuda")
    got, got_lse = b.razer_attn_kv8(s.cache, q.cuda(), *s.args, workspace=ws)
    b.razer_workspace_status(ws)
    out, lse, x = got.double().cpu(), got_lse.double().cpu(), q.double()
    for i in range(len(s.new)):
        rows, limit = (torch.tensor(t) for t in zip(*s.tokens(i)))
        hidden = torch.arange(s.total[i])[None, :] > limit[:, None]
        pages = s.table[i, :-(-s.total[i] // s.page)].long()
        for h in range(s.H):
            k, v = visible64(s, i, h, s.k, s.ks), visible64(s, i, h, s.v, s.vs)
            sv = s.vs[pages, h].double().repeat_interleave(s.page)[:s.total[i]].expand(len(rows), -1).masked_fill(hidden, 0.0)
            for g in range(G):
                xq = x[rows, h * G + g]
                a = (s.D ** -0.5 * (xq @ k.t())).masked_fill(hidden, -float("inf"))
                room = (s.D ** -0.5 * (xq.abs() @ k.abs().t())).masked_fill(hidden, 0.0).max(dim=1).values
                want_lse = torch.logsumexp(a, dim=1)
                p = torch.exp(a - want_lse[:, None])
                want, size = p @ v, p @ v.abs()
                lost = (s.D ** -0.5 * k.abs().sum(1)).expand(len(rows), -1).masked_fill(hidden, 0.0).max(dim=1).values * xq.abs().max(dim=1).values
                e = (2.0 ** -23 * (s.D + 4) * room + 2.0 ** -21 + 2.0 ** -22 * lost)[:, None]
                most = (p * sv).max(dim=1).values if few else 2.0 ** -5 * p.max(dim=1).values * sv.max(dim=1).values
                bar = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2 * e + 2.0 ** -20) * size + (limit + 1)[:, None] * 2.0 ** -25 * 127 * most[:, None]
                off = (out[rows, h * G + g] - want).abs()
                assert (off <= bar).all(), (i, h, g, int((off > bar).any(1).nonzero()[0]), float((off / bar.clamp(min=1e-300)).max()))
                assert ((lse[rows, h * G + g] - want_lse).abs() <= e[:, 0] + 2.0 ** -22 * want_lse.abs() + 2.0 ** -21).all()
    return got, got_lse


# new tokens, query heads a group, dimensions: 4, 8, 16, 32 rows; 60, 300 rows; 1024 rows and more (pairs of CTAs)
SHAPES = [(4, 1, 64), (8, 1, 128), (4, 4, 128), (32, 1, 64), (16, 2, 128), (60, 1, 64), (75, 4, 128), (260, 4, 128)]


@pytest.mark.parametrize("power", [20, 40, 75])
@pytest.mark.parametrize("n,G,D", SHAPES)
def test_value_scales_of_hidden_pages(b, n, G, D, power):  # noqa: F811
    """The last page's value scale is a power of two larger: rows that do not see it come out as well as without it, those that do like any other."""
    s = Batch([n], [n + 30], 2, D, 16, seed=n + power)
    s.vs[int(s.table[0, s.width - 1])] *= 2.0 ** power
    check_rows(b, s, queries(s, G), few=n * G <= 32)


@pytest.mark.parametrize("n,G,D", SHAPES)
def test_values_behind_the_mask_change_nothing(b, n, G, D):  # noqa: F811
    """Large, small, zero: rows that do not see the page are the same number for number in the kernel for many rows (in that for few the sum of the exponentials is
    relative to what the page's tile has, a rounding's difference)."""
    want = None
    for power in (0, 1, 12, 30, -40):
        s = Batch([n], [n + 30], 2, D, 16, seed=n)
        last = s.width - 1
        s.vs[int(s.table[0, last])] *= 2.0 ** power
        got, lse = check_rows(b, s, queries(s, G), few=n * G <= 32)
        before = last * 16 - 30                                # rows of positions in front of the last page
        if want is None:
            want = got[:before], lse[:before]
        assert before > 0
        if n * G > 32:
            assert torch.equal(got[:before], want[0]) and torch.equal(lse[:before], want[1]), power


@pytest.mark.parametrize("rows", [1, 4, 8, 16, 32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("low", [0.0, 2.0 ** -90, 2.0 ** -61, 2.0 ** -59])
def test_pages_that_matter_without_the_largest_scores(b, rows, D, low):  # noqa: F811
    """A page with far larger scores and hardly any values: what comes out is the other pages', to 24 bits of the largest weight among 128 tokens."""
    s = Batch([1], [300], 1, D, 16, seed=rows)
    q = torch.full((1, rows, D), 1.0).bfloat16()
    q += (torch.randint(-4, 5, q.shape, generator=s.g) / 128).bfloat16()
    for block in (2, 9, 17):                                   # of two tiles of 128 tokens and of the last, which has no full one
        at = int(s.table[0, block])
        s.k[at] = 127
        s.ks[at] = 70.0 / (127 * D ** 0.5)                     # scores of about 70, the others within some units of 0
        s.vs[at] *= low
    s.ks[s.table[0, [0, 1]].long()] *= 0.1
    check_rows(b, s, q, few=True)


def test_a_tile_of_values_that_are_all_zero(b):  # noqa: F811
    """No value scale in 128 tokens, and one in the next; broken ones beside zeros show."""
    for rows in (1, 8, 32, 40):
        s = Batch([1], [300], 1, 64, 16, seed=rows)
        s.vs[s.table[0, :8].long()] = 0.0
        q = queries(s, rows)
        check_rows(b, s, q, few=rows <= 32)
        s.vs[int(s.table[0, 3])] = float("nan")
        s.device(b)
        assert torch.isnan(b.razer_attn_kv8(s.cache, q.cuda(), *s.args)[0]).all()


@pytest.mark.parametrize("rows", [1, 8, 32])
def test_queries_in_24_bit_fixed_point(b, rows):  # noqa: F811
    """Up to 32 rows: each number of a query is held to 2^-22 of the row's largest (half a step of 2^(e - 21), the largest in [2^e, 2^(e + 1))).  The largest meets no key here,
    so that a small one is all that the score, which is the log-sum of one key, has."""
    unit = 64 ** -0.5 * 2.0 ** 13 * 127
    for first in range(1, 200, rows):
        s = Batch([1], [1], 1, 64, 16, seed=first)
        at = int(s.table[0, 0])
        s.k[at], s.ks[at] = 127, 2.0 ** 13
        s.k[at, 0, :, 0] = 0
        q = torch.zeros((1, rows, 64), dtype=torch.float64)
        q[..., 0] = 1.0
        for r in range(rows):
            q[0, r, 1 + r % 63] = (first + r) * 2.0 ** -23 * (-1) ** r
        s.device(b)
        _, lse = b.razer_attn_kv8(s.cache, q.bfloat16().cuda(), *s.args)
        want = unit * q[0, :, 1:].sum(1)
        off = (lse[0].double().cpu() - want).abs()
        assert (off <= unit * 2.0 ** -22 + (2.0 ** -23 * 68 + 2.0 ** -22) * want.abs() + 2.0 ** -21).all(), (first, float(off.max() / unit))
