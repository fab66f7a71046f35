"""The paged 8-bit cache on the GPU: its writer bit for bit, and the attention over it against the definition in 64 bits.

Bar of the attention.  Exact result o = sum p_j v_j / sum p_j.  What is rounded: the query row to f16 or 24 bits with a scale of its own (exact
for bf16 but for values below 2^-14 of the row's largest, which are off by at most 2^-23 of it), scores and their exponents in FP32 (a score of
magnitude S is off by at most (D + 4) 2^-24 S_abs with S_abs = scale * ks * sum_d |q_d k_d|; the tensor core's truncated additions are counted as
2^-23 each, and the exponential as 2^-21), weights p_j vs_j to 24 bits of the largest among 128 tokens (off by 2^-25 of that), or to f16 (off by
2^-11 of each, or, where f16 has no more bits, by half its smallest step 2^-24; 2^6 stands for the row's largest p times twice the largest vs or more,
so that this is at most 2^-30 max p max vs), sums in FP32, the result to bf16 (2^-8).
A weight that is off by 2^-25 W, W = max(max_j p_j vs_j, 2^-5 max p max vs), moves the numerator by at most 2^-25 W |code| <= 2^-25 W 127, and n keys
by n times that.  So with A = sum p_j |v_j| / sum p_j and E = 2^-23 (D + 4) max S_abs + 2^-21:
   |out - o| <= 2^-8 |o| + (2^-11 + 2 E + 2^-20) A + 2^-38 max |v| + 2^-25 127 n W / sum p_j
   |lse - exact| <= E + 2^-22 |exact| + 2^-21
"""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_2501_04052_b200 import binding
    return binding


class Batch:
    """Sequences with random pages; `new`, `total`: new tokens and tokens in all of each."""

    def __init__(self, new, total, H, D, page, seed=0, spare=2, extra_width=0, pad_rows=0):
        g = torch.Generator().manual_seed(seed)
        self.new, self.total, self.H, self.D, self.page = new, total, H, D, page
        held = [-(-t // page) for t in total]
        self.pages, self.width = sum(held) + spare, max(max(held), 1) + extra_width
        order = torch.randperm(self.pages, generator=g).tolist()
        self.table = torch.full((len(new), self.width), -7, dtype=torch.int32)     # entries behind the last page name none
        at = 0
        for i, n in enumerate(held):
            self.table[i, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            at += n
        self.free = order[at:]
        self.starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.T = int(self.starts[-1]) + pad_rows
        shape = (self.pages, H, page, D)
        self.k, self.v = (torch.randint(-127, 128, shape, generator=g, dtype=torch.int8) for _ in range(2))
        self.ks, self.vs = (0.005 + 0.02 * torch.rand((self.pages, H), generator=g) for _ in range(2))
        self.g = g

    def device(self, b):
        self.dev = [t.cuda() for t in (self.k, self.v, self.ks, self.vs)]
        self.cache = b.make_kv8(*self.dev)
        self.args = (self.table.cuda(), torch.from_numpy(self.starts).cuda(), torch.tensor(self.total, dtype=torch.int32).cuda())
        return self

    def tokens(self, i):
        """[(row, position)] of sequence i's new tokens."""
        return [(int(self.starts[i]) + j, self.total[i] - self.new[i] + j) for j in range(self.new[i])]


def append64(s, x, codes, scales):
    """The writer's definition on numpy copies: codes int8, scales float32."""
    codes, scales = codes.numpy().copy(), scales.numpy().copy()
    x = x.double().numpy()
    for i in range(len(s.new)):
        by_block = {}
        for row, pos in s.tokens(i):
            if pos >= 0:
                by_block.setdefault(pos // s.page, []).append((row, pos % s.page))
        for block, rows in by_block.items():
            at = int(s.table[i, block]) if block < s.width else -1
            if not 0 <= at < s.pages:
                continue
            for h in range(s.H):
                with np.errstate(all="ignore"):
                    new = np.stack([x[r, h] for r, _ in rows])
                    s0 = scales[at, h] if rows[0][1] > 0 else np.float32(0)
                    top = np.abs(new).max() if np.isfinite(new).all() else np.nan
                    fresh = np.float32(top / 127.0)
                    if fresh == 0 and top > 0:
                        fresh = np.float32(2.0 ** -149)
                    if not (np.isfinite(fresh) and np.isfinite(s0)):
                        scales[at, h] = np.nan
                        for _, p in rows:
                            codes[at, h, p] = 0
                        continue
                    step = max(s0, fresh)
                    if step > s0 > 0:                        # the page's other codes keep their values
                        codes[at, h] = np.rint(codes[at, h].astype(np.float64) * float(s0) / float(step)).astype(np.int8)
                    scales[at, h] = step
                    for (r, p), v in zip(rows, new):
                        codes[at, h, p] = np.clip(np.rint(v / float(step)), -127, 127).astype(np.int8) if step > 0 else 0
    return codes, scales


def check_append(b, s, k_new, v_new, times=1):
    s.device(b)
    for _ in range(times):
        b.razer_kv8_append(s.cache, k_new.cuda() if not k_new.is_cuda else k_new, v_new.cuda() if not v_new.is_cuda else v_new, *s.args)
    for x, codes, scales, got_c, got_s in ((k_new, s.k, s.ks, s.dev[0], s.dev[2]), (v_new, s.v, s.vs, s.dev[1], s.dev[3])):
        want_c, want_s = append64(s, x.cpu(), codes, scales)
        got_s = got_s.cpu().numpy()
        assert np.array_equal(np.isnan(got_s), np.isnan(want_s)) and np.array_equal(np.nan_to_num(got_s), np.nan_to_num(want_s))
        assert np.array_equal(got_c.cpu().numpy(), want_c)


def fresh(s, scale=1.0):
    return tuple((torch.randn((s.T, s.H, s.D), generator=s.g) * scale).bfloat16() for _ in range(2))


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("D,H", [(64, 1), (128, 3)])
def test_append_lengths(b, page, D, H):
    """One token at each place of a page, prompts from nothing, and everything between; small and large values, so that some scales grow."""
    new = [1, 1, 1, 1, 5, page, page + 1, 3 * page, 2, 0, 17, 1]
    total = [1, page, page + 1, 2 * page - 1, 5, page, page + 1, 3 * page + 7, page + 1, 40, page + 16, 700]
    for scale in (0.3, 1.5, 40.0):
        s = Batch(new, total, H, D, page, seed=page + D)
        check_append(b, s, *fresh(s, scale))


def test_append_twice_is_once(b):
    s = Batch([3, 1, 30], [20, 33, 30], 2, 64, 16, seed=5)
    check_append(b, s, *fresh(s, 2.0), times=3)


def test_append_columns_of_a_projection(b):
    s = Batch([2, 9, 1], [5, 40, 64], 2, 64, 32, seed=6)
    wide = torch.randn((s.T, 3 * 2 * 64 + 8), generator=s.g).bfloat16().cuda()
    check_append(b, s, wide[:, 128:256].unflatten(1, (2, 64)), wide[:, 256:384].unflatten(1, (2, 64)))


def test_append_token_by_token_and_many_sequences(b):
    """300 sequences, more than a CTA has threads; then 40 tokens one after another, the cache kept between."""
    s = Batch([1 + i % 3 for i in range(300)], [1 + (7 * i) % 90 + i % 3 for i in range(300)], 1, 64, 16, seed=7)
    check_append(b, s, *fresh(s))
    s = Batch([1, 1], [1, 1], 2, 64, 16, seed=8, spare=8)
    s.table = torch.tensor([[0, 1, 2], [3, 4, 5]], dtype=torch.int32)
    s.width = 3
    for t in range(1, 41):
        s.total = [t, t + 5]
        k, v = fresh(s, 1.0 + t / 4 * (t % 5 == 0))
        check_append(b, s, k, v)
        s.k, s.v, s.ks, s.vs = (x.cpu() for x in s.dev)


def test_append_zeros_and_broken_values(b):
    s = Batch([4, 1, 1, 20, 1], [4, 10, 10, 20, 18], 2, 64, 16, seed=9)
    k, v = fresh(s)
    k[0:4] = 0                                               # a page of zeros
    k[4, 0, 3], k[5, 1, 63], v[6, 0, 0] = float("nan"), float("inf"), float("-inf")
    v[4] = 0                                                 # zeros behind older values
    s.ks[int(s.table[4, 1]), 0] = float("nan")               # a scale that is broken already stays so
    s.vs[int(s.table[4, 1]), 1] = 0.0
    check_append(b, s, k, v)


def test_append_skips_what_has_no_place(b):
    """Pages that the table does not name, tokens before the sequence's beginning, rows beyond the last sequence, a sequence longer than the table."""
    s = Batch([3, 40, 5, 2], [10, 64, 3, 20], 2, 64, 16, seed=10, pad_rows=3)
    s.table[0, 0] = s.pages
    s.table[1, 2] = -1
    s.width, s.table = 4, s.table[:, :4].contiguous()
    s.total[3] = 66                                          # tokens 64 and 65: behind the table's four pages
    check_append(b, s, *fresh(s))


def visible64(s, i, h, codes, scales):
    """[total, D] values of sequence i, head h in 64 bits."""
    at = s.table[i, :-(-s.total[i] // s.page)].long()
    x = codes[at, h].double() * scales[at, h].double()[:, None, None]
    return x.reshape(-1, s.D)[:s.total[i]]


def check_attn(b, s, q, scale=None, workspace=None):
    G = q.shape[1] // s.H
    scale = s.D ** -0.5 if scale is None else scale
    s.device(b)
    ws = b.alloc_attn_workspace(s.cache, s.H * G, "cuda") if workspace is None else workspace
    qd = q if q.is_cuda else q.cuda()
    out = torch.full((s.T, s.H * G, s.D), 5.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((s.T, s.H * G), 5.0, device="cuda")
    b.razer_attn_kv8(s.cache, qd, *s.args, scale=scale, out=out, lse=lse, workspace=ws)
    b.razer_workspace_status(ws)
    second = b.razer_attn_kv8(s.cache, qd, *s.args, scale=scale, workspace=ws)
    b.razer_workspace_status(ws)
    used = int(s.starts[-1])
    assert torch.equal(torch.nan_to_num(out[:used], 9.0), torch.nan_to_num(second[0][:used], 9.0)), "the same call twice"
    assert torch.equal(torch.nan_to_num(lse[:used], 9.0), torch.nan_to_num(second[1][:used], 9.0))
    assert (out[used:] == 5).all() and (lse[used:] == 5).all()
    out, lse, q = out.double().cpu(), lse.double().cpu(), q.double().cpu()
    worst = 0.0
    for i in range(len(s.new)):
        toks = s.tokens(i)
        if not toks:
            continue
        rows = torch.tensor([r for r, _ in toks])
        limit = torch.tensor([p for _, p in toks])
        hidden = torch.arange(max(s.total[i], 0))[None, :] > limit[:, None]
        for h in range(s.H):
            k, v = visible64(s, i, h, s.k, s.ks), visible64(s, i, h, s.v, s.vs)
            for gq in range(G):
                x = q[rows, h * G + gq]
                a = scale * (x @ k.t())
                room = (abs(scale) * (x.abs() @ k.abs().t())).masked_fill(hidden, 0.0)
                room = room.max(dim=1).values if room.shape[1] else torch.zeros(len(toks), dtype=torch.float64)
                a = a.masked_fill(hidden, -math.inf)
                want_lse = torch.logsumexp(a, dim=1) if a.shape[1] else torch.full((len(toks),), -math.inf, dtype=torch.float64)
                p = torch.exp(a - want_lse[:, None].clamp(min=-1e300)).masked_fill(hidden, 0.0)
                want = p @ v
                size = p @ v.abs()
                top = v.abs().max() if v.numel() else 0.0
                e = 2.0 ** -23 * (s.D + 4) * room + 2.0 ** -21
                sv = s.vs[s.table[i, :-(-s.total[i] // s.page)].long(), h].double().repeat_interleave(s.page)[:max(s.total[i], 0)]
                most = 0.0
                if p.shape[1]:
                    most = torch.maximum((p * sv).max(dim=1, keepdim=True).values, 2.0 ** -5 * p.max(dim=1, keepdim=True).values * sv.max())
                    most = most * 127 * (limit[:, None] + 1).clamp(min=0)
                bar = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2 * e[:, None] + 2.0 ** -20) * size + 2.0 ** -38 * top + 2.0 ** -25 * most
                off = (out[rows, h * G + gq] - want).abs()
                assert (off <= bar).all(), (i, h, gq, float((off / bar.clamp(min=1e-300)).max()))
                worst = max(worst, float((off / bar.clamp(min=1e-300)).max()))
                got = lse[rows, h * G + gq]
                empty = torch.isinf(want_lse)
                assert torch.equal(got[empty], want_lse[empty])
                assert ((got - want_lse)[~empty].abs() <= (e + 2.0 ** -22 * want_lse.abs() + 2.0 ** -21)[~empty]).all()
    print(f"[attn] {len(s.new)} sequences, worst {worst:.2f} of the bar")


def queries(s, G, scale=1.0):
    return (torch.randn((s.T, s.H * G, s.D), generator=s.g) * scale).bfloat16()


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 3, 8])
def test_attn_decode_lengths(b, page, D, G):
    total = [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 300, 1000, page, page + 1, 0]
    s = Batch([1] * len(total), total, 2, D, page, seed=page + D + G)
    check_attn(b, s, queries(s, G))


@pytest.mark.parametrize("H,G,D,total", [(1, 1, 128, 5000), (8, 4, 64, 4096), (1, 8, 128, 20000), (2, 16, 128, 3001), (3, 5, 64, 2999), (1, 40, 128, 1500), (1, 71, 64, 777)])
def test_attn_one_long_sequence(b, H, G, D, total):
    """A single row of queries over all SMs: units cut among many CTAs."""
    s = Batch([1], [total], H, D, 16, seed=total)
    check_attn(b, s, queries(s, G))


@pytest.mark.parametrize("G,H", [(1, 2), (2, 2), (4, 1), (5, 1), (16, 1), (33, 1)])
@pytest.mark.parametrize("D", [64, 128])
def test_attn_several_new_tokens(b, G, H, D):
    """Causal rows: from a few tokens (speculative decoding) to chunks of prompts, mixed with decoding sequences and with sequences that have no row."""
    new = [1, 4, 0, 9, 1, 64, 70, 2]
    total = [50, 4, 33, 100, 1, 64, 200, 129]
    s = Batch(new, total, H, D, 32, seed=G + D, pad_rows=5)
    check_attn(b, s, queries(s, G))


@pytest.mark.parametrize("G", [1, 4])
def test_attn_prompt_chunk(b, G):
    s = Batch([300, 7, 129], [1500, 900, 129], 2, 128, 64, seed=G)
    check_attn(b, s, queries(s, G))


def test_attn_ragged_batch(b):
    """Lengths from 1 to 9000 in one batch, more sequences than a CTA has threads."""
    g = np.random.default_rng(1)
    total = [int(x) for x in np.exp(g.uniform(0, math.log(300), 290))] + [9000, 1, 4097]
    s = Batch([1] * len(total), total, 1, 64, 16, seed=11)
    check_attn(b, s, queries(s, 4))


@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
def test_attn_scales(b, scale):
    """No weighting, weighting turned round, and scores far apart (one key has nearly all)."""
    s = Batch([2, 3], [100, 257], 2, 64, 32, seed=12)
    check_attn(b, s, queries(s, 4), scale=scale)


def test_attn_magnitudes(b):
    """Rows of queries of very different sizes, key and value scales over many binades, pages of zeros."""
    s = Batch([3, 2], [500, 70], 2, 128, 16, seed=13)
    q = queries(s, 4)
    q *= torch.logspace(-30, 0, q.shape[0] * q.shape[1], base=2).view(q.shape[0], q.shape[1], 1)
    q[0, 0] = 0
    s.ks *= torch.logspace(-20, 0, s.pages, base=2)[:, None]
    s.vs *= torch.logspace(-12, 12, s.pages, base=2)[:, None]
    s.vs[int(s.table[0, 3])], s.ks[int(s.table[0, 4])], s.vs[int(s.table[1, 0])] = 0.0, 0.0, 0.0
    check_attn(b, s, q.bfloat16())
    s.vs *= 0
    check_attn(b, s, q.bfloat16())
    tiny = Batch([1], [40], 1, 64, 16, seed=14)
    tiny.ks, tiny.vs = tiny.ks * 2.0 ** 100, tiny.vs * 2.0 ** -110
    check_attn(b, tiny, (queries(tiny, 2).double() * 2.0 ** -125).bfloat16())


def test_attn_columns_of_a_projection_and_rows_left_alone(b):
    s = Batch([2, 9, 1], [5, 40, 64], 2, 64, 32, seed=15, pad_rows=4)
    wide = torch.randn((s.T, 8 * 64 + 16), generator=s.g).bfloat16().cuda()
    check_attn(b, s, wide[:, 16:16 + 4 * 64].unflatten(1, (4, 64)))


def test_attn_more_rows_than_keys(b):
    """More new tokens than the sequence has: the first rows have no position and see nothing."""
    s = Batch([5, 3], [2, 0], 1, 64, 16, seed=16)
    check_attn(b, s, queries(s, 2))


def test_attn_broken_scales_and_pages(b):
    """A NaN scale, and a page that the table does not name, show in the rows that see the page and in no other; neither does what lies behind."""
    for what in ("key", "value", "page", "query", "long"):
        s = Batch([20, 1, 1], [40, 30, 90], 2, 64, 16, seed=17, extra_width=1)
        q = queries(s, 2)
        bad = torch.zeros((s.T, 4), dtype=torch.bool)
        behind = int(s.table[0, 2])                          # positions 32 .. 39 of sequence 0, whose rows are positions 20 .. 39: seen from row 12 on
        if what == "key":
            s.ks[behind, 1] = float("nan")
            bad[12:20, 2:] = True
        elif what == "value":
            s.vs[behind, 0] = float("nan")
            bad[12:20, :2] = True
        elif what == "page":
            s.table[0, 2] = s.pages + 5
            bad[12:20] = True
        elif what == "query":
            q[3, 1, 5], q[21, 0, 0] = float("nan"), float("inf")
            bad[3, 1] = bad[21, 0] = True
        else:
            s.total[2] = s.width * 16 + 1
            bad[21] = True
        # pages that nobody sees
        for p in s.free:
            s.ks[p] = s.vs[p] = float("nan")
        s.device(b)
        out, lse = b.razer_attn_kv8(s.cache, q.cuda(), *s.args)
        assert torch.equal(torch.isnan(out).any(2).cpu(), bad) and torch.equal(torch.isnan(out).all(2).cpu(), bad), what
        if what != "value":
            assert torch.equal(torch.isnan(lse).cpu(), bad), what
        if what in ("key", "value", "page"):                 # the rest is what it would be without
            clean = Batch([20, 1, 1], [40, 30, 90], 2, 64, 16, seed=17, extra_width=1).device(b)
            ref, _ = b.razer_attn_kv8(clean.cache, q.cuda(), *clean.args)
            good = ~bad.cuda()
            assert ((out - ref)[good].abs() <= 2.0 ** -7 * ref[good].abs() + 1e-3).all()


def test_attn_workspace_serves_batches_in_turn_and_graphs(b):
    """One workspace, many batches in a row without waiting; then a captured step replayed as lengths grow."""
    ws = None
    runs = []
    for i, (new, total, G) in enumerate([([1], [3000], 4), ([5, 1], [70, 600], 8), ([1] * 40, [100 + 7 * j for j in range(40)], 1), ([90], [2000], 2)] * 2):
        s = Batch(new, total, 2, 64, 16, seed=20 + i % 4).device(b)
        q = queries(s, G).cuda()
        if ws is None:
            ws = b.alloc_attn_workspace(s.cache, 16, "cuda")
        runs.append((s, q, b.razer_attn_kv8(s.cache, q, *s.args, workspace=ws)))
    b.razer_workspace_status(ws)
    for s, q, (out, lse) in runs:
        alone, alone_lse = b.razer_attn_kv8(s.cache, q, *s.args)
        assert torch.equal(out, alone) and torch.equal(lse, alone_lse)
    s = Batch([1, 1], [60, 300], 2, 64, 16, seed=30).device(b)
    q, k, v = queries(s, 4).cuda(), *(x.cuda() for x in fresh(s))
    out, lse = torch.empty_like(q), torch.empty((s.T, 8), device="cuda")
    b.razer_attn_kv8(s.cache, q, *s.args, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.razer_kv8_append(s.cache, k, v, *s.args)
        b.razer_attn_kv8(s.cache, q, *s.args, out=out, lse=lse, workspace=ws)
    for total in ([50, 290], [51, 291], [64, 304]):
        s.args[2].copy_(torch.tensor(total, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        s.total, (s.k, s.v, s.ks, s.vs) = total, (x.cpu() for x in s.dev)
        got, got_lse = out.clone(), lse.clone()
        want, want_lse = b.razer_attn_kv8(s.cache, q, *s.args)
        assert torch.equal(got, want) and torch.equal(got_lse, want_lse)


def test_a_decode_step_as_it_is_used(b):
    """Quantize, project, write, attend, project: each stage on what the one before has just written, against 64 bits from the same stage's input."""
    hidden, H, G, D, page = 512, 2, 4, 64, 16
    s = Batch([1, 3, 1], [33, 40, 200], H, D, page, seed=40).device(b)
    g = torch.Generator().manual_seed(41)
    width = (H * G + 2 * H) * D
    w_qkv = (0.05 * torch.randn((width, hidden), generator=g)).cuda()
    w_out = (0.05 * torch.randn((hidden, H * G * D), generator=g)).cuda()
    x = torch.randn((s.T, hidden), generator=g).bfloat16().cuda()
    qkv_codes, out_codes = b.razer_quant_i8(w_qkv), b.razer_quant_i8(w_out)
    ws = b.alloc_attn_workspace(s.cache, H * G, "cuda")
    xc, xs = b.razer_quant_i8(x)
    qkv = b.razer_gemm_i8(xc, xs, *qkv_codes)
    q = qkv[:, :H * G * D].unflatten(1, (H * G, D))
    k = qkv[:, H * G * D:(H * G + H) * D].unflatten(1, (H, D))
    v = qkv[:, (H * G + H) * D:].unflatten(1, (H, D))
    b.razer_kv8_append(s.cache, k, v, *s.args)
    out, _ = b.razer_attn_kv8(s.cache, q, *s.args, workspace=ws)
    oc, os_ = b.razer_quant_i8(out.flatten(1))
    y = b.razer_gemm_i8(oc, os_, *out_codes)
    b.razer_workspace_status(ws)
    # every weight and value in 8 bits with its own scale is off by half a step, 1/254 of its row's largest: a percent or two in norm per stage
    exact = x.double() @ w_qkv.double().t()
    assert (qkv.double() - exact).norm() <= 0.03 * exact.norm()
    want = (oc.double() * os_.double()[:, None]) @ (out_codes[0].double() * out_codes[1].double()[:, None]).t()
    assert ((y.double() - want).abs() <= (2.0 ** -8 + 2.0 ** -22) * want.abs()).all()
    s.k, s.v, s.ks, s.vs = (t.cpu() for t in s.dev)
    check_attn(b, s, q)


@pytest.mark.parametrize("kernel", ["few", "many", "pair"])
def test_attn_either_kernel_takes_any_batch(kernel):
    """The attention's tests with all calls on one of its kernels (the choice is read once a process)."""
    here = os.path.abspath(__file__)
    r = subprocess.run([sys.executable, "-m", "pytest", here, "-q", "-x", "-m", "gpu", "-k", "attn and not either_kernel and not beyond_32_bits"],
                       env=dict(os.environ, RAZER_ATTN=kernel), capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-1000:]


@pytest.mark.parametrize("D,page", [(128, 16), (64, 128)])
def test_pools_beyond_32_bits(b, D, page):
    """Pages whose bytes lie past 2^31 and 2^32: written and attended to like any other."""
    H, pages = 8, (1 << 32) // (8 * page * D) + 300
    pools = [torch.zeros((pages, H, page, D), dtype=torch.int8, device="cuda") for _ in range(2)]
    scales = [torch.zeros((pages, H), device="cuda") for _ in range(2)]
    cache = b.make_kv8(*pools, *scales)
    n = 5 * page + 3
    places = torch.tensor([[pages - 1, 7, (1 << 31) // (H * page * D) + 1, pages - 200, 0, pages // 2]], dtype=torch.int32)
    starts, lens = torch.tensor([0, n], dtype=torch.int32).cuda(), torch.tensor([n], dtype=torch.int32).cuda()
    g = torch.Generator().manual_seed(page)
    k, v = (torch.randn((n, H, D), generator=g).bfloat16() for _ in range(2))
    b.razer_kv8_append(cache, k.cuda(), v.cuda(), places.cuda(), starts, lens)
    small = Batch([n], [n], H, D, page, seed=1)
    small.table = torch.arange(6, dtype=torch.int32)[None, :]
    small.pages = 6
    small.k, small.v = (torch.zeros((6, H, page, D), dtype=torch.int8) for _ in range(2))
    small.ks, small.vs = (torch.zeros((6, H)) for _ in range(2))
    want = [append64(small, x, c, s) for x, c, s in ((k, small.k, small.ks), (v, small.v, small.vs))]
    for i in range(2):
        at = places[0].long().cuda()
        assert np.array_equal(pools[i][at].cpu().numpy(), want[i][0]) and np.array_equal(scales[i][at].cpu().numpy(), want[i][1])
        assert int((pools[i] != 0).sum()) == int((torch.from_numpy(want[i][0]) != 0).sum())      # nothing anywhere else
    (small.k, small.ks), (small.v, small.vs) = ((torch.from_numpy(c), torch.from_numpy(s)) for c, s in want)
    for rows in (1, n):                                      # few rows and many
        q = torch.randn((rows, 2 * H, D), generator=g).bfloat16().cuda()
        qs = torch.tensor([0, rows], dtype=torch.int32).cuda()
        small.device(b)
        got = b.razer_attn_kv8(cache, q, places.cuda(), qs, lens)
        ref = b.razer_attn_kv8(small.cache, q, small.args[0], qs, lens)
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


@pytest.mark.parametrize("compiled", [True, False])
def test_both_ways_into_the_library(b, monkeypatch, compiled):
    """Plain calls through the compiled part of the binding and through ctypes, given and allocated outputs, and what each refuses."""
    if compiled and b._call is None:
        pytest.skip(b.call_route())
    if not compiled:
        monkeypatch.setattr(b, "_call", None)
    s = Batch([3, 1], [40, 90], 2, 64, 16, seed=50)
    q = queries(s, 4)
    check_append(b, s, *fresh(s))
    s.k, s.v, s.ks, s.vs = (x.cpu() for x in s.dev)
    check_attn(b, s, q)
    d = q.cuda()
    for bad in (d.float(), d[:, :, ::2], d.transpose(0, 1), q):
        with pytest.raises((AssertionError, RuntimeError)):
            b.razer_attn_kv8(s.cache, bad, *s.args)
    k = fresh(s)[0].cuda()
    for args in ((k, k[:2], *s.args), (k[:, :1], k[:, :1], *s.args), (k, k, s.args[0].long(), *s.args[1:]), (k, k, s.args[0], s.args[1][:2], s.args[2]),
                 (k, k, s.args[0].t(), *s.args[1:])):
        with pytest.raises((AssertionError, RuntimeError)):
            b.razer_kv8_append(s.cache, *args)
    with pytest.raises(b.RazerError):
        b.razer_attn_kv8(s.cache, d, *s.args, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    x = torch.randn((5, 64), generator=s.g).bfloat16().cuda()
    codes, scales = b.razer_quant_i8(x)
    mine = torch.empty_like(codes)
    assert b.razer_quant_i8(x, mine)[0] is not None and torch.equal(mine, codes)
    y = b.razer_gemm_i8(codes, scales, codes, scales)
    out = torch.empty_like(y)
    assert torch.equal(b.razer_gemm_i8(codes, scales, codes, scales, out), y) and torch.equal(out, y)
    for args in ((codes, scales[:4], codes, scales), (codes[:, :48], scales, codes, scales), (codes.t(), scales, codes, scales), (codes, scales.double(), codes, scales)):
        with pytest.raises((AssertionError, RuntimeError)):
            b.razer_gemm_i8(*args)
    with pytest.raises(b.RazerError):
        b.razer_quant_i8(torch.zeros((2, 24), dtype=torch.bfloat16, device="cuda"))


def test_two_streams_with_a_workspace_each(b):
    """Two batches at once on two streams, many times; each as if it were alone."""
    batches = [Batch([1] * 9, [900 + 31 * i for i in range(9)], 2, 64, 16, seed=60).device(b), Batch([70, 2], [1500, 333], 2, 128, 32, seed=61).device(b)]
    qs = [queries(s, 4).cuda() for s in batches]
    alone = [b.razer_attn_kv8(s.cache, q, *s.args) for s, q in zip(batches, qs)]
    spaces = [b.alloc_attn_workspace(s.cache, 8, "cuda") for s in batches]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in batches]
    got = [[], []]
    for _ in range(30):
        for i, (s, q, st) in enumerate(zip(batches, qs, streams)):
            with torch.cuda.stream(st):
                got[i].append(b.razer_attn_kv8(s.cache, q, *s.args, workspace=spaces[i]))
    torch.cuda.synchronize()
    for i in range(2):
        b.razer_workspace_status(spaces[i])
        assert all(torch.equal(o, alone[i][0]) and torch.equal(l, alone[i][1]) for o, l in got[i])


def test_full_pages_may_be_shared(b):
    """Two sequences over the same first pages (a common prompt)."""
    s = Batch([1, 4], [70, 90], 2, 64, 16, seed=62)
    s.table[1, :3] = s.table[0, :3]
    check_attn(b, s, queries(s, 4))


def test_rows_outside_the_buffers_count_as_none(b):
    """q_start that leaves 0 .. T or falls: those sequences have no rows, the others are as ever."""
    s = Batch([2, 3, 2], [20, 30, 40], 1, 64, 16, seed=63).device(b)
    q = queries(s, 2).cuda()
    ref, ref_lse = b.razer_attn_kv8(s.cache, q, *s.args)
    for starts, fine in (([0, 2, 5, 9], [0, 1]), ([-1, 2, 5, 7], [1, 2]), ([0, 2, 1, 1], [0])):
        st = torch.tensor(starts, dtype=torch.int32).cuda()
        out, lse = torch.full_like(ref, 5.0), torch.full_like(ref_lse, 5.0)
        ws = b.alloc_attn_workspace(s.cache, 2, "cuda")
        b.razer_attn_kv8(s.cache, q, s.args[0], st, s.args[2], out=out, lse=lse, workspace=ws)
        b.razer_workspace_status(ws)
        for i in fine:
            lo, hi = starts[i], starts[i + 1]
            assert torch.equal(out[lo:hi], ref[lo:hi]) and torch.equal(lse[lo:hi], ref_lse[lo:hi]), starts
        b.razer_kv8_append(s.cache, q[:, :1].contiguous(), q[:, :1].contiguous(), s.args[0], st, s.args[2])
        torch.cuda.synchronize()
        for t, keep in zip(s.dev, (s.k, s.v, s.ks, s.vs)):
            t.copy_(keep)


def test_a_captured_decode_step_replayed(b):
    """The whole step in one graph, its inputs and lengths changed between replays, against the same calls one by one."""
    hidden, H, G, D, page, steps = 256, 2, 4, 64, 16, 20
    first = [1, 30, 200]
    s = Batch([1] * 3, [t + steps for t in first], H, D, page, seed=50).device(b)
    g = torch.Generator().manual_seed(51)
    weights = b.razer_quant_i8((0.05 * torch.randn(((H * G + 2 * H) * D, hidden), generator=g)).cuda())
    xs = torch.randn((steps, 3, hidden), generator=g).bfloat16().cuda()
    table, starts = s.args[0], s.args[1]
    x, lens = xs[0].clone(), torch.zeros(3, dtype=torch.int32, device="cuda")

    def step(cache, ws):
        qkv = b.razer_gemm_i8(*b.razer_quant_i8(x), *weights)
        q = qkv[:, :H * G * D].unflatten(1, (H * G, D))
        k = qkv[:, H * G * D:(H * G + H) * D].unflatten(1, (H, D))
        v = qkv[:, (H * G + H) * D:].unflatten(1, (H, D))
        b.razer_kv8_append(cache, k, v, table, starts, lens)
        return b.razer_attn_kv8(cache, q, table, starts, lens, workspace=ws)

    pools = [t.clone() for t in s.dev]
    apart = b.make_kv8(*pools)
    ws = [b.alloc_attn_workspace(s.cache, H * G, "cuda") for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(s.cache, ws[0])
    for i in range(steps):
        x.copy_(xs[i])
        lens.copy_(torch.tensor([t + i + 1 for t in first], dtype=torch.int32))
        graph.replay()
        want = step(apart, ws[1])
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), i
    assert all(torch.equal(p, t) for p, t in zip(pools, s.dev))
    for w in ws:
        b.razer_workspace_status(w)
