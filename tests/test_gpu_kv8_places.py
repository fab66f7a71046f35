"""The 8-bit operators in calls of other shapes: long prompts, many sequences, pools at any 16 bytes, captured work that forks and joins, batches of one kernel after another
on one workspace.

The bar is that of test_gpu_kv8_scales.py where values are compared with 64 bits; the rest is equal number for number.
"""
import numpy as np
import pytest
import torch

from test_gpu_kv8 import Batch, append64, b, fresh, queries  # noqa: F401
from test_gpu_kv8_scales import check_rows

pytestmark = pytest.mark.gpu


def test_a_prompt_of_seventy_thousand_tokens(b):  # noqa: F811
    """Written and attended to in one call; some rows against 64 bits."""
    n, page, D = 70001, 64, 64
    pages = -(-n // page)
    g = torch.Generator(device="cuda").manual_seed(1)
    pools = [torch.zeros((pages, 1, page, D), dtype=torch.int8, device="cuda") for _ in range(2)]
    scales = [torch.zeros((pages, 1), device="cuda") for _ in range(2)]
    cache = b.make_kv8(*pools, *scales)
    table = torch.randperm(pages, generator=g, device="cuda").int()[None, :]
    starts, lens = torch.tensor([0, n], dtype=torch.int32, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda")
    q, k, v = (torch.randn((n, 1, D), generator=g, device="cuda").bfloat16() for _ in range(3))
    b.razer_kv8_append(cache, k, v, table, starts, lens)
    ws = b.alloc_attn_workspace(cache, 1, "cuda")
    out, lse = b.razer_attn_kv8(cache, q, table, starts, lens, workspace=ws)
    b.razer_workspace_status(ws)
    keys, values = ((p[table[0].long()].double() * s[table[0].long()].double()[..., None, None]).reshape(-1, D)[:n] for p, s in zip(pools, scales))
    for x, y in ((k, keys), (v, values)):                     # half a step of the page's largest, 4.6 or less here
        assert (x[:, 0].double() - y).abs().max() <= x.abs().max().double() / 254
    rows = torch.tensor([0, 1, 63, 64, 127, 128, 255, 256, 1000, 32767, 32768, 65535, 65536, 69999, 70000], device="cuda")
    a = (q[rows, 0].double() @ keys.t()) * D ** -0.5
    a.masked_fill_(torch.arange(n, device="cuda")[None, :] > rows[:, None], -float("inf"))
    room = ((q[rows, 0].double().abs() @ keys.abs().t()) * D ** -0.5).max(dim=1).values
    want_lse = torch.logsumexp(a, dim=1)
    p = torch.exp(a - want_lse[:, None])
    want, size = p @ values, p @ values.abs()
    e = (2.0 ** -23 * (D + 4) * room + 2.0 ** -21)[:, None]
    most = 2.0 ** -5 * p.max(dim=1, keepdim=True).values * scales[1].max().double()
    bar = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2 * e + 2.0 ** -20) * size + (rows + 1)[:, None] * 2.0 ** -25 * 127 * most
    assert ((out[rows, 0].double() - want).abs() <= bar).all()
    # sums of up to n FP32 terms: pairs of columns by two running sums, off by 2^-24 of themselves for each of the n / 2 additions at most
    assert ((lse[rows, 0].double() - want_lse).abs() <= e[:, 0] + 2.0 ** -22 * want_lse.abs() + 2.0 ** -21 + rows * 2.0 ** -25).all()


def test_five_thousand_sequences(b):  # noqa: F811
    """More sequences than slots a thread looks at once, most of them short, some without rows: written, attended to by the kernel for few rows."""
    rng = np.random.default_rng(2)
    total = [int(x) for x in rng.integers(1, 20, 5000)]
    new = [int(min(t, x)) for t, x in zip(total, rng.integers(0, 3, 5000))]
    s = Batch(new, total, 1, 64, 16, seed=3)
    k, v = fresh(s)
    s.device(b)
    b.razer_kv8_append(s.cache, k.cuda(), v.cuda(), *s.args)
    for x, codes, scales, got_c, got_s in ((k, s.k, s.ks, s.dev[0], s.dev[2]), (v, s.v, s.vs, s.dev[1], s.dev[3])):
        want_c, want_s = append64(s, x, codes, scales)
        assert np.array_equal(got_c.cpu().numpy(), want_c) and np.array_equal(got_s.cpu().numpy(), want_s)
    q = queries(s, 2).cuda()
    ws = b.alloc_attn_workspace(s.cache, 2, "cuda")
    out, lse = b.razer_attn_kv8(s.cache, q, *s.args, workspace=ws)
    b.razer_workspace_status(ws)
    for lo in range(0, 5000, 625):                            # the same sequences a few at a time
        a, z = int(s.starts[lo]), int(s.starts[lo + 625])
        part = b.razer_attn_kv8(s.cache, q[a:z], s.args[0][lo:lo + 625], (s.args[1][lo:lo + 626] - a).contiguous(), s.args[2][lo:lo + 625], workspace=ws)
        # units are cut otherwise, so that sums are put together otherwise: two bf16 roundings, and FP32 of up to 20 terms
        assert ((out[a:z].float() - part[0].float()).abs() <= 2.0 ** -7 * part[0].float().abs() + 2.0 ** -12).all()
        assert ((lse[a:z] - part[1]).abs() <= 2.0 ** -18 * (1 + part[1].abs())).all()


@pytest.mark.parametrize("D,n,G", [(64, 1, 4), (128, 8, 4), (128, 60, 2), (128, 300, 4)])
def test_pools_at_any_sixteen_bytes(b, D, n, G):  # noqa: F811
    """Pools that begin 16 bytes into an allocation: no more is asked of them."""
    s = Batch([n], [n + 200], 2, D, 16, seed=n).device(b)
    q = queries(s, G).cuda()
    k, v = (x.cuda() for x in fresh(s))
    b.razer_kv8_append(s.cache, k, v, *s.args)
    want = b.razer_attn_kv8(s.cache, q, *s.args)
    def moved(t, by):
        buf = torch.zeros(t.numel() + by, dtype=t.dtype, device="cuda")
        return buf[by:].view(t.shape).copy_(t)
    odd = b.make_kv8(moved(s.k.cuda(), 16), moved(s.v.cuda(), 48), moved(s.ks.cuda(), 1), moved(s.vs.cuda(), 3))
    b.razer_kv8_append(odd, moved(k, 8), moved(v, 24), *s.args)
    got = b.razer_attn_kv8(odd, moved(q, 8), *s.args, out=moved(torch.zeros_like(q), 8), lse=moved(torch.zeros((s.T, 2 * G), device="cuda"), 1))
    assert all(torch.equal(x, y) for x, y in zip(odd.tensors, s.dev)) and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_captured_work_that_forks_and_joins(b):  # noqa: F811
    """Two streams of one graph, calls that follow a join of both, a workspace for each branch."""
    s = [Batch([1, 5], [70, 90], 2, 64, 16, seed=70), Batch([80, 1], [300, 90], 2, 128, 32, seed=71)]
    data = []
    for x in s:
        k, v = (t.cuda() for t in fresh(x))
        x.device(b)
        data.append((k, v, queries(x, 4).cuda(), b.alloc_attn_workspace(x.cache, 8, "cuda")))
    w = b.razer_quant_i8(torch.randn((96, 64 * 8), generator=s[0].g).cuda())

    def branch(i):
        k, v, q, ws = data[i]
        b.razer_kv8_append(s[i].cache, k, v, *s[i].args)
        return b.razer_attn_kv8(s[i].cache, q, *s[i].args, workspace=ws)

    def end(x, y):
        a = torch.cat([x[0].flatten(1), y[0].flatten(1)[:, :512]])
        return b.razer_gemm_i8(*b.razer_quant_i8(a), *w)

    want = [branch(0), branch(1)]
    want.append(end(*want))
    for x in s:
        for t, keep in zip(x.dev, (x.k, x.v, x.ks, x.vs)):
            t.copy_(keep)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        with torch.cuda.stream(side):
            second = branch(1)
        first = branch(0)
        main.wait_stream(side)
        # directly behind the join: a call whose operands both branches wrote
        again = b.razer_attn_kv8(s[1].cache, data[1][2], *s[1].args, workspace=data[0][3] if data[0][3].numel() >= data[1][3].numel() else data[1][3])
        last = end(first, second)
    for _ in range(3):
        for t in (*first, *second, *again, last):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for got, exact in ((first, want[0]), (second, want[1]), (again, want[1]), ((last,), (want[2],))):
            assert all(torch.equal(x, y) for x, y in zip(got, exact))
        for _, _, _, ws in data:
            b.razer_workspace_status(ws)


def test_batches_of_both_kernels_on_one_workspace_in_a_graph(b):  # noqa: F811
    """Few rows, many, pairs and few again, one behind the other without waiting, replayed."""
    shapes = [([1] * 9, 4), ([70], 2), ([300, 20], 8), ([2, 1], 4), ([33], 1), ([1], 40)]
    s = [Batch(new, [n + 500 for n in new], 2, 128, 16, seed=80 + i).device(b) for i, (new, _) in enumerate(shapes)]
    q = [queries(x, g).cuda() for x, (_, g) in zip(s, shapes)]
    want = [b.razer_attn_kv8(x.cache, y, *x.args) for x, y in zip(s, q)]
    ws = b.alloc_attn_workspace(s[0].cache, 16, "cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [b.razer_attn_kv8(x.cache, y, *x.args, workspace=ws) for _ in range(3) for x, y in zip(s, q)]
    for _ in range(5):
        graph.replay()
    b.razer_workspace_status(ws)
    for i, (out, lse) in enumerate(got):
        assert torch.equal(out, want[i % 6][0]) and torch.equal(lse, want[i % 6][1])


@pytest.mark.parametrize("G", [300, 520])
def test_more_query_heads_than_a_row_tile(b, G):  # noqa: F811
    s = Batch([3, 1], [200, 70], 1, 128, 32, seed=G)
    check_rows(b, s, queries(s, G), few=False)
