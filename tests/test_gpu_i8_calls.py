"""The 8-bit operators' calls: what they refuse, what they leave alone, and what they let others do."""
import ctypes

import pytest
import torch

from test_gpu_kv8 import Batch, b, fresh, queries  # noqa: F401

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
