"""The 8-bit operators refuse bad arguments on the host, before any CUDA work (no GPU needed)."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def b():
    from paper_2501_04052_b200 import build
    build.build()
    from paper_2501_04052_b200 import binding
    return binding


AT = 1 << 20                                                # addresses are looked at for their alignment only


def test_struct_matches_header(b):
    assert ctypes.sizeof(b.RazerKv8) == 48 and b.RazerKv8.k_codes_dev.offset == 16 and b.RazerKv8.v_scales_dev.offset == 40


@pytest.mark.parametrize("args,code", [
    ((AT, 0, 0, 64, 64, AT, AT, None), "INVALID_ARG"),       # no rows
    ((AT, 0, 4, 72, 72, AT, AT, None), "INVALID_ARG"),       # K % 16
    ((AT, 0, 4, 0, 64, AT, AT, None), "INVALID_ARG"),
    ((AT, 0, 4, 64, 48, AT, AT, None), "INVALID_ARG"),       # rows that overlap
    ((AT, 0, 4, 64, 68, AT, AT, None), "INVALID_ARG"),       # rows off their 16 bytes
    ((AT, 1, 4, 64, 66, AT, AT, None), "INVALID_ARG"),
    ((AT + 8, 0, 4, 64, 64, AT, AT, None), "INVALID_ARG"),
    ((None, 0, 4, 64, 64, AT, AT, None), "INVALID_ARG"),
    ((AT, 0, 4, 64, 64, AT + 4, AT, None), "INVALID_ARG"),
    ((AT, 0, 4, 64, 64, AT, AT + 2, None), "INVALID_ARG"),
])
def test_quant_i8_refuses(b, args, code):
    assert b.lib().razer_quant_i8(*args) == getattr(b, "ERR_" + code) and b.last_error()


@pytest.mark.parametrize("args,code", [
    ((AT, AT, AT, AT, 0, 8, 64, AT, None), "INVALID_ARG"),
    ((AT, AT, AT, AT, 8, 0, 64, AT, None), "INVALID_ARG"),
    ((AT, AT, AT, AT, 8, 8, 40, AT, None), "INVALID_ARG"),
    ((AT, AT, AT, AT, 8, 8, 131072, AT, None), "UNSUPPORTED"),     # (-128)^2 * 131072 = 2^31
    ((AT, AT, AT, AT, 0x7FFFFF01, 8, 64, AT, None), "UNSUPPORTED"),
    ((AT, AT, AT, AT, 8, 0x7FFFFFFF, 64, AT, None), "UNSUPPORTED"),
    ((AT + 8, AT, AT, AT, 8, 8, 64, AT, None), "INVALID_ARG"),
    ((AT, AT + 2, AT, AT, 8, 8, 64, AT, None), "INVALID_ARG"),
    ((AT, AT, AT + 8, AT, 8, 8, 64, AT, None), "INVALID_ARG"),
    ((AT, AT, AT, None, 8, 8, 64, AT, None), "INVALID_ARG"),
    ((AT, AT, AT, AT, 8, 8, 64, AT + 1, None), "INVALID_ARG"),
])
def test_gemm_i8_refuses(b, args, code):
    assert b.lib().razer_gemm_i8(*args) == getattr(b, "ERR_" + code) and b.last_error()


def _cache(b, **other):
    c = b.RazerKv8()
    c.pages, c.page, c.heads, c.head_dim = 4, 16, 2, 64
    c.k_codes_dev = c.v_codes_dev = c.k_scales_dev = c.v_scales_dev = AT
    for k, v in other.items():
        setattr(c, k, v)
    return c


def _append(b, cache, k=AT, ks=128, v=AT, vs=128, table=AT, width=4, starts=AT, lens=AT, B=1, T=1):
    return b.lib().razer_kv8_append(ctypes.byref(cache) if cache else None, k, ks, v, vs, table, width, starts, lens, B, T, None)


def _attn(b, cache, q=AT, qs=256, heads=4, table=AT, width=4, starts=AT, lens=AT, B=1, T=1, scale=0.1, out=AT, lse=None, ws=AT, size=1 << 30):
    return b.lib().razer_attn_kv8(ctypes.byref(cache) if cache else None, q, qs, heads, table, width, starts, lens, B, T, scale, out, lse, ws, size, None)


@pytest.mark.parametrize("other,code", [
    (dict(page=8), "UNSUPPORTED"), (dict(page=48), "UNSUPPORTED"), (dict(page=256), "UNSUPPORTED"), (dict(head_dim=96), "UNSUPPORTED"),
    (dict(pages=0), "INVALID_ARG"), (dict(heads=0), "INVALID_ARG"), (dict(heads=40000), "INVALID_ARG"), (dict(pages=1 << 30), "INVALID_ARG"),
    (dict(k_codes_dev=AT + 8), "INVALID_ARG"), (dict(v_codes_dev=None), "INVALID_ARG"), (dict(k_scales_dev=AT + 2), "INVALID_ARG"),
    (dict(v_scales_dev=None), "INVALID_ARG"),
])
def test_caches_that_are_refused(b, other, code):
    c, n = _cache(b, **other), ctypes.c_size_t()
    for rc in (_append(b, c), _attn(b, c), b.lib().razer_attn_kv8_workspace_bytes(ctypes.byref(c), 80000, ctypes.byref(n))):
        assert rc == getattr(b, "ERR_" + code) and b.last_error()


def test_batches_that_are_refused(b):
    c = _cache(b)
    bad = [dict(B=-1), dict(T=-1), dict(width=0), dict(width=(1 << 27)), dict(table=None), dict(table=AT + 2), dict(starts=None), dict(lens=None)]
    for other in bad:
        assert _append(b, c, **other) == b.ERR_INVALID_ARG and _attn(b, c, **other) == b.ERR_INVALID_ARG, other
    assert _append(b, None) == b.ERR_INVALID_ARG and _attn(b, None) == b.ERR_INVALID_ARG
    for other in (dict(k=None), dict(k=AT + 8), dict(ks=120), dict(ks=132), dict(v=AT + 2), dict(vs=64)):
        assert _append(b, c, **other) == b.ERR_INVALID_ARG, other
    for other in (dict(q=None), dict(q=AT + 8), dict(qs=248), dict(qs=260), dict(heads=3), dict(heads=0), dict(out=None), dict(out=AT + 8), dict(lse=AT + 2),
                  dict(scale=float("nan")), dict(scale=float("inf")), dict(ws=AT + 16)):
        assert _attn(b, c, **other) == b.ERR_INVALID_ARG, other
    n = ctypes.c_size_t()
    assert b.lib().razer_attn_kv8_workspace_bytes(ctypes.byref(c), 4, ctypes.byref(n)) == 0 and n.value % 256 == 0
    assert _attn(b, c, ws=None) == b.ERR_WORKSPACE and _attn(b, c, size=n.value - 1) == b.ERR_WORKSPACE
    assert b.lib().razer_attn_kv8_workspace_bytes(ctypes.byref(c), 3, ctypes.byref(n)) == b.ERR_INVALID_ARG
    assert b.lib().razer_attn_kv8_workspace_bytes(ctypes.byref(c), 4, None) == b.ERR_INVALID_ARG


def test_batches_without_work(b):
    c = _cache(b)
    for other in (dict(B=0), dict(T=0), dict(B=0, T=0, table=None, starts=None, lens=None)):
        assert _append(b, c, **other) == 0 and _attn(b, c, **other) == 0


def test_tensors_that_the_binding_refuses(b):
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    for bad in (x, x.float(), x.half(), x.t(), x[0]):          # on the host, other types, columns apart, one axis
        with pytest.raises((AssertionError, RuntimeError)):
            b.razer_quant_i8(bad)
    codes, scales = torch.zeros((4, 64), dtype=torch.int8), torch.zeros(4)
    for args in ((codes, scales, codes, scales), (codes.float(), scales, codes, scales), (codes, scales[:3], codes, scales), (codes, scales, codes[:, :32], scales)):
        with pytest.raises((AssertionError, RuntimeError)):
            b.razer_gemm_i8(*args)
    pool, sc = torch.zeros((4, 2, 16, 64), dtype=torch.int8), torch.zeros((4, 2))
    for args in ((pool, pool, sc, sc), (pool, pool[:2], sc, sc), (pool, pool, sc.half(), sc), (pool, pool, sc[:2], sc[:2]), (pool[0], pool[0], sc, sc)):
        with pytest.raises(AssertionError):
            b.make_kv8(*args)
