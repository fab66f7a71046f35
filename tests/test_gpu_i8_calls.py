"""The 8-bit operators' calls: what they refuse, what they leave alone, and what they let others do."""
import ctypes

import numpy as np
import pytest
import torch

from test_gpu_kv8 import Batch, append64, b, fresh, queries  # noqa: F401

pytestmark = pytest.mark.gpu


def test_compiled_calls_let_other_threads_run(b):  # noqa: F811
    """The library's function is called without the interpreter's lock, as through ctypes: PyGILState_Check in its place says whether the thread holds it, 0 or 1,
    which the call takes for the library's status."""
    if b._call is None:
        pytest.skip(b.call_route())
    check = ctypes.cast(ctypes.pythonapi.PyGILState_Check, ctypes.c_void_p).value
    s = Batch([1], [40], 2, 64, 16, seed=52).device(b)
    q, (k, v) = queries(s, 4).cuda(), (x.cuda() for x in fresh(s))
    ws = b.alloc_attn_workspace(s.cache, 8, "cuda")
    x = torch.zeros((3, 64), dtype=torch.bfloat16, device="cuda")
    codes, scales = b.razer_quant_i8(x)
    assert type(b._call.quant_i8(check, x, None, None)) is tuple
    assert torch.is_tensor(b._call.gemm_i8(check, codes, scales, codes, scales, None))
    assert b._call.kv8_append(check, b.RazerKv8, s.cache, k, v, *s.args) == 0
    assert type(b._call.attn_kv8(check, b.RazerKv8, s.cache, q, *s.args, None, None, None, ws)) is tuple


def test_workspaces_that_are_no_bytes_side_by_side(b):  # noqa: F811
    """A workspace whose numbers are not bytes side by side is not taken for one.  (All of these have the memory behind them.)"""
    s = Batch([1], [40], 2, 64, 16, seed=51).device(b)
    q = queries(s, 4).cuda()
    ws = b.alloc_attn_workspace(s.cache, 8, "cuda")
    for bad in (ws[:1].expand(ws.numel()), torch.empty(2 * ws.numel(), dtype=torch.uint8, device="cuda")[::2], ws.view(torch.int32)):
        with pytest.raises(AssertionError):
            b.razer_attn_kv8(s.cache, q, *s.args, workspace=bad)


@pytest.mark.parametrize("H,D,page,B,G", [(8, 128, 16, 70, 4), (8, 64, 128, 40, 1), (2, 64, 16, 150, 1), (4, 128, 32, 5, 40)])
def test_scales_that_the_kernel_directly_ahead_has_written(b, H, D, page, B, G):  # noqa: F811
    """The writer raises the scales of pages, several to a cache line and each by a CTA that has read the line before, and the attention behind it is resident by then: as if
    every call had been waited for."""
    steps, width = 25, 3
    g = torch.Generator().manual_seed(B)
    table = torch.randperm(B * width, generator=g).view(B, width).int().cuda()
    starts = torch.arange(B + 1, dtype=torch.int32).cuda()
    lens = torch.randint(page + 1, 2 * page, (B,), generator=g, dtype=torch.int32).cuda()
    news = [[(torch.randn((B, H, D), generator=g) * 1.05 ** i).bfloat16().cuda() for _ in range(2)] for i in range(steps)]
    q = torch.randn((B, H * G, D), generator=g).bfloat16().cuda()
    pool = torch.randint(-127, 128, (B * width, H, page, D), generator=g, dtype=torch.int8).cuda()
    want = None
    for wait in (True, False, False, False):
        cache = b.make_kv8(pool.clone(), pool.clone(), *(torch.full((B * width, H), 1e-3, device="cuda") for _ in range(2)))
        ws = b.alloc_attn_workspace(cache, H * G, "cuda")
        got = []
        for k, v in news:
            b.razer_kv8_append(cache, k, v, table, starts, lens)
            if wait:
                torch.cuda.synchronize()
            got.append(b.razer_attn_kv8(cache, q, table, starts, lens, workspace=ws))
            if wait:
                torch.cuda.synchronize()
        b.razer_workspace_status(ws)
        want = want or got
        assert all(torch.equal(x, y) for a, c in zip(got, want) for x, y in zip(a, c))


def test_append_leaves_what_bad_rows_would_write(b):  # noqa: F811
    """q_start that leaves 0 .. T: those sequences write nothing, the others all of theirs."""
    for starts, bad in (([0, 2, 5, 9], [2]), ([-1, 2, 5, 7], [0]), ([-3, -1, 4, 8], [0, 1, 2])):
        s = Batch([2, 3, 2], [20, 30, 40], 2, 64, 16, seed=63)
        k, v = fresh(s)
        s.starts = np.array(starts, dtype=np.int32)
        s.device(b)
        b.razer_kv8_append(s.cache, k.cuda(), v.cuda(), *s.args)
        s.new = [0 if i in bad else starts[i + 1] - starts[i] for i in range(3)]
        for x, codes, scales, got_c, got_s in ((k, s.k, s.ks, s.dev[0], s.dev[2]), (v, s.v, s.vs, s.dev[1], s.dev[3])):
            want_c, want_s = append64(s, x, codes, scales)
            assert np.array_equal(got_c.cpu().numpy(), want_c) and np.array_equal(got_s.cpu().numpy(), want_s), starts


@pytest.mark.parametrize("compiled", [True, False])
def test_attention_refuses_bad_tensors_beside_a_workspace(b, monkeypatch, compiled):  # noqa: F811
    """A call with a workspace of its own goes through the compiled part first."""
    if compiled and b._call is None:
        pytest.skip(b.call_route())
    if not compiled:
        monkeypatch.setattr(b, "_call", None)
    s = Batch([3, 1], [40, 90], 2, 64, 16, seed=50).device(b)
    q = queries(s, 4).cuda()
    ws = b.alloc_attn_workspace(s.cache, 8, "cuda")
    table, starts, lens = s.args
    out, lse = torch.empty_like(q), torch.empty((s.T, 8), device="cuda")
    for bad in (q.float(), q[:, :, ::2], q.transpose(0, 1), q.cpu(), q[0]):
        with pytest.raises((AssertionError, RuntimeError, IndexError)):
            b.razer_attn_kv8(s.cache, bad, *s.args, workspace=ws)
    for args in ((table.long(), starts, lens), (table.t(), starts, lens), (table[:1], starts, lens), (table, starts[:2], lens), (table, starts, lens[:1]), (table, starts.cpu(), lens)):
        with pytest.raises((AssertionError, RuntimeError)):
            b.razer_attn_kv8(s.cache, q, *args, workspace=ws)
    for other in (dict(out=out.float()), dict(out=out[:2]), dict(out=out.transpose(0, 1)), dict(lse=lse.double()), dict(lse=lse[:, :4]), dict(out=out.cpu())):
        with pytest.raises((AssertionError, RuntimeError)):
            b.razer_attn_kv8(s.cache, q, *s.args, workspace=ws, **other)
    with pytest.raises(b.RazerError):
        b.razer_attn_kv8(s.cache, q, *s.args, workspace=ws, scale=float("nan"))
    want = b.razer_attn_kv8(s.cache, q, *s.args)
    got = b.razer_attn_kv8(s.cache, q, *s.args, workspace=ws, out=out, lse=lse)
    assert got[0].data_ptr() == out.data_ptr() and torch.equal(out, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("new,total,G", [([1, 1], [300, 40], 4), ([1], [3000], 8), ([70], [200], 4), ([300], [900], 4)])
def test_attention_without_a_log_sum(b, new, total, G):  # noqa: F811
    """lse_dev NULL: the same output, by either kernel, from whole units and from joined parts."""
    s = Batch(new, total, 2, 128, 32, seed=53).device(b)
    q = queries(s, G).cuda()
    ws = b.alloc_attn_workspace(s.cache, 2 * G, "cuda")
    want, _ = b.razer_attn_kv8(s.cache, q, *s.args, workspace=ws)
    out = torch.empty_like(q)
    table, starts, lens = s.args
    rc = b.lib().razer_attn_kv8(ctypes.byref(s.cache), q.data_ptr(), q.stride(0), 2 * G, table.data_ptr(), table.shape[1], starts.data_ptr(), lens.data_ptr(), len(new), s.T,
                                128 ** -0.5, out.data_ptr(), None, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    b.razer_workspace_status(ws)
    assert torch.equal(out, want)


def test_attention_with_the_largest_scale(b):  # noqa: F811
    """Scores of 0 under it are 0, by either kernel."""
    for rows in (1, 40):
        s = Batch([1], [200], 1, 64, 16, seed=54)
        s.k[:] = 0
        q = queries(s, rows)
        s.device(b)
        for scale in (2.0 ** 62, -2.0 ** 62):
            out, lse = b.razer_attn_kv8(s.cache, q.cuda(), *s.args, scale=scale)
            plain, plain_lse = b.razer_attn_kv8(s.cache, q.cuda(), *s.args, scale=0.0)
            assert torch.equal(out, plain) and torch.equal(lse, plain_lse)
