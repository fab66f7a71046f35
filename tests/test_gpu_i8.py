"""8-bit integers on the GPU: the row quantizer and the integer product against their definitions in 64 bits.

Bars.  Codes and scales: equal (the quotient's border is decided by the exact quotient; x / s of two 24-bit numbers in 64 bits never
crosses a border that the exact one does not cross).  The product: the integer sum is exact, then one FP32 rounding each of the sum, of the
scales' product and of their product, and one to bf16: |y - exact| <= (2^-8 + 4 * 2^-24) |exact|, a bf16 rounding being off by at most 2^-8 of the value
(half a step of 2^-7).
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BAR = 2.0 ** -8 + 4 * 2.0 ** -24


@pytest.fixture(scope="module")
def b():
    from paper_2501_04052_b200 import binding
    return binding


def quantize64(x):
    """codes int8, scales float32 of rows of a float64 array holding bf16 or FP32 values."""
    with np.errstate(all="ignore"):
        top = np.abs(x).max(axis=1)
        scale = (top / 127.0).astype(np.float32)
        scale = np.where((scale == 0) & (top > 0), np.float32(2.0 ** -149), scale)
        scale = np.where(np.isfinite(x).all(axis=1), scale, np.float32(np.nan)).astype(np.float32)
        step = scale.astype(np.float64)[:, None]
        q = np.where((step > 0) & np.isfinite(step), np.clip(np.rint(x / np.where(step > 0, step, 1.0)), -127, 127), 0.0)
    return np.nan_to_num(q).astype(np.int8), scale


def same_quantized(b, x, **kw):
    codes, scales = b.razer_quant_i8(x, **kw)
    want_codes, want_scales = quantize64(x.double().cpu().numpy())
    assert np.array_equal(scales.cpu().numpy().view(np.uint32) & 0x7FFFFFFF, want_scales.view(np.uint32) & 0x7FFFFFFF)
    assert np.array_equal(codes.cpu().numpy(), want_codes)
    return codes, scales


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,K", [(1, 16), (3, 32), (5, 128), (7, 272), (130, 512), (2, 1040), (9, 4096), (33, 4112), (4, 8192), (3, 8208), (2, 16400), (2, 32768),
                                 (2, 33024), (1, 70000)])
def test_quant_i8_rows(b, M, K, dtype):
    g = torch.Generator().manual_seed(M * 100003 + K)
    x = torch.randn((M, K), generator=g) * torch.exp(4 * torch.randn((M, 1), generator=g))
    same_quantized(b, x.to(dtype).cuda())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quant_i8_values_on_borders(b, dtype):
    """Halves of the scale, where the scale is a power of two and the quotients are ties exactly, and where its rounding puts them to one side."""
    K = 1024
    n = torch.arange(K, dtype=torch.float32)
    rows = [(n % 255 - 127) / 2, (n % 255 - 127) * 0.5 * 1.25, n % 254 - 127, (n % 253 - 126) / 2 + 0.25]
    for top in (127.0, 254.0, 1.0, 3.0, 4.0, 1.9921875, 100.0, 2.0 ** -60, 3.0 * 2.0 ** 90):
        for r in rows:
            x = (r / 127 * top).clone()
            x[5] = top
            same_quantized(b, x.clamp(-top, top).to(dtype).cuda()[None, :])
    # halves of an exact step: x = (n + 1/2) s with s = fl32(top / 127) a power of two
    x = (n % 127).clone() + 0.5
    x[0] = 127.0
    same_quantized(b, x.clamp(-127, 127).to(dtype).cuda()[None, :])


@pytest.mark.parametrize("dtype,log2s", [(torch.bfloat16, (-133, -126, -100, 0, 100, 126)), (torch.float32, (-149, -147, -140, -126, -118, -93, -92, 0, 100, 126))])
def test_quant_i8_magnitudes(b, dtype, log2s):
    g = torch.Generator().manual_seed(3)
    for e in log2s:
        x = (torch.rand((4, 96), generator=g, dtype=torch.float64) * 2 - 1) * 2.0 ** e * 1.9
        x[1] = x[1].abs().clamp(max=2.0 ** e)
        same_quantized(b, x.to(dtype).cuda())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quant_i8_rows_without_a_scale(b, dtype):
    """Zeros, NaN, infinities: their own rows only."""
    x = torch.randn((7, 4112), generator=torch.Generator().manual_seed(4))
    x[1] = 0
    x[2, 4111] = float("nan")
    x[3, 0] = float("inf")
    x[4, 77] = float("-inf")
    x[5] = -0.0
    codes, scales = same_quantized(b, x.to(dtype).cuda())
    assert torch.isnan(scales[2:5]).all() and (codes[1:6] == 0).all() and (scales[[1, 5]] == 0).all()


def test_quant_i8_strided_rows_and_given_outputs(b):
    wide = torch.randn((37, 3 * 400), generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    codes = torch.full((39, 400), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((39,), 7.0, device="cuda")
    same_quantized(b, wide[:, 400:800], codes=codes[1:38], scales=scales[1:38])
    assert (codes[[0, 38]] == 99).all() and (scales[[0, 38]] == 7).all()
    one = wide[5:6, 400:800]
    same_quantized(b, one)
    with pytest.raises(b.RazerError):
        b.razer_quant_i8(wide[:, 1:401])                     # rows off their 16 bytes


def exact_product(x, sx, w, sw):
    """Full 64-bit result; the sums are whole numbers below 2^53."""
    return (x.double() @ w.double().t()) * sx.double()[:, None] * sw.double()


def codes_of(rows, K, seed, low=-128):
    return torch.randint(low, 128, (rows, K), generator=torch.Generator().manual_seed(seed), dtype=torch.int8)


def check_product(b, M, N, K, seed=0, x=None, w=None):
    x = codes_of(M, K, seed + 1) if x is None else x
    w = codes_of(N, K, seed + 2) if w is None else w
    g = torch.Generator().manual_seed(seed)
    sx, sw = torch.rand(M, generator=g) + 0.01, (torch.rand(N, generator=g) + 0.01) * 1e-3
    guard = torch.full(((M + 2) * N,), 3.0, dtype=torch.bfloat16, device="cuda")
    y = guard[N:-N].view(M, N)
    b.razer_gemm_i8(x.cuda(), sx.cuda(), w.cuda(), sw.cuda(), y)
    assert (guard[:N] == 3).all() and (guard[-N:] == 3).all()
    want = exact_product(x.cuda(), sx.cuda(), w.cuda(), sw.cuda())
    off = (y.double() - want).abs()
    assert (off <= BAR * want.abs()).all(), (M, N, K, float((off / want.abs().clamp(min=1e-30)).max()))
    again = b.razer_gemm_i8(x.cuda(), sx.cuda(), w.cuda(), sw.cuda())
    assert torch.equal(y, again)
    return y


@pytest.mark.parametrize("M,N,K", [(1, 1, 16), (1, 1, 131056), (2, 3, 48), (1, 128, 128), (1, 129, 144), (5, 333, 2064), (16, 300, 4096), (17, 300, 4096), (32, 127, 272),
                                   (33, 640, 1040), (64, 257, 528), (65, 1000, 656), (128, 130, 2048), (129, 384, 2064), (255, 511, 272), (256, 256, 256),
                                   (257, 513, 1296), (300, 65, 128), (513, 1030, 784), (1, 4096, 4096), (3, 11008, 512), (700, 2304, 400)])
def test_gemm_i8(b, M, N, K):
    check_product(b, M, N, K, seed=M + N + K)


@pytest.mark.parametrize("M", [1, 16, 64, 128, 256, 600])
def test_gemm_i8_largest_sums(b, M):
    """(-128)^2 summed up to the longest K: 2^31 - 2^18, and the same with signs that cancel."""
    K, N = 131056, 40
    x = torch.full((M, K), -128, dtype=torch.int8)
    w = torch.full((N, K), -128, dtype=torch.int8)
    w[1::2, ::2] = 127
    w[2::4] = 127
    check_product(b, M, N, K, x=x, w=w)


def test_gemm_i8_one_hot_finds_every_place(b):
    """x = rows of the unit matrix: every weight comes out alone, so that each code is seen to be read from its own place."""
    N, K = 200, 400
    w = codes_of(N, K, 9)
    x = torch.eye(K, dtype=torch.int8)
    y = b.razer_gemm_i8(x.cuda(), torch.ones(K).cuda(), w.cuda(), torch.ones(N).cuda())
    assert torch.equal(y.float().cpu(), w.t().float())


def test_gemm_i8_scales(b):
    """Zero scales give zeros, a NaN scale its own row or column only."""
    M, N, K = 40, 130, 64
    x, w = codes_of(M, K, 1).cuda(), codes_of(N, K, 2).cuda()
    sx, sw = torch.ones(M).cuda(), torch.ones(N).cuda()
    sx[3], sx[4], sw[7], sw[129] = 0.0, float("nan"), float("nan"), 0.0
    y = b.razer_gemm_i8(x, sx, w, sw)
    assert torch.isnan(y[4]).all() and torch.isnan(y[:, 7]).all() and (y[3, :7] == 0).all() and (y[:4, 129] == 0).all()
    fine = torch.ones((M, N), dtype=torch.bool)
    fine[4], fine[:, 7] = False, False
    assert torch.isfinite(y.cpu()[fine]).all()


def test_gemm_i8_unaligned_output_and_streams(b):
    """y at an odd element, work on another stream, and the same through a captured graph."""
    M, N, K = 19, 80, 192
    x, w = codes_of(M, K, 1).cuda(), codes_of(N, K, 2).cuda()
    sx, sw = torch.rand(M).cuda(), torch.rand(N).cuda()
    want = b.razer_gemm_i8(x, sx, w, sw)
    buf = torch.zeros(M * N + 1, dtype=torch.bfloat16, device="cuda")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        b.razer_gemm_i8(x, sx, w, sw, buf[1:].view(M, N))
    st.synchronize()
    assert torch.equal(buf[1:].view(M, N), want)
    y = torch.zeros_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        codes, scales = b.razer_quant_i8(want)
        b.razer_gemm_i8(x, sx, w, sw, y)
    for _ in range(3):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


@pytest.mark.parametrize("M", [1, 16, 200])
def test_quantize_and_multiply_back_to_back(b, M):
    """Operands that the kernel directly ahead has just written, many times in a row on buffers in turn."""
    N, K = 320, 1024
    g = torch.Generator().manual_seed(M)
    ws = [(0.02 * torch.randn((N, K), generator=g)).cuda() for _ in range(4)]
    xs = [torch.randn((M, K), generator=g).bfloat16().cuda() for _ in range(4)]
    codes, scales = torch.empty((N, K), dtype=torch.int8, device="cuda"), torch.empty(N, device="cuda")
    got = []
    for i in range(32):
        b.razer_quant_i8(ws[i % 4], codes, scales)
        xc, xs_ = b.razer_quant_i8(xs[i % 4])
        got.append(b.razer_gemm_i8(xc, xs_, codes, scales))
    for i in range(32):
        wc, wsc = (torch.from_numpy(a) for a in quantize64(ws[i % 4].double().cpu().numpy()))
        xc, xsc = (torch.from_numpy(a) for a in quantize64(xs[i % 4].double().cpu().numpy()))
        want = exact_product(xc, xsc, wc, wsc)
        assert ((got[i].double().cpu() - want).abs() <= BAR * want.abs()).all(), i


@pytest.mark.parametrize("M,N,K", [(3, 33000, 70000), (33000, 24, 70000), (46400, 46500, 16)])
def test_gemm_i8_beyond_32_bits(b, M, N, K):
    """Operands and a result of more than 2^31 elements: the last rows and columns, and the first, against 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(N)
    x, w = (torch.randint(-128, 128, (r, K), generator=g, dtype=torch.int8, device="cuda") for r in (M, N))
    sx, sw = torch.rand(M, generator=g, device="cuda") + 0.01, torch.rand(N, generator=g, device="cuda") + 0.01
    y = b.razer_gemm_i8(x, sx, w, sw)
    at = lambda n: torch.unique(torch.tensor([0, 1, 2, n // 2, n - 3, n - 2, n - 1], device="cuda").clamp(0, n - 1))  # noqa: E731
    m, n = at(M), at(N)
    want = exact_product(x[m], sx[m], w[n], sw[n])
    assert ((y[m][:, n].double() - want).abs() <= BAR * want.abs()).all()


def test_quant_i8_beyond_32_bits(b):
    M, K = 33000, 70000
    x = torch.full((M, K), 0.5, dtype=torch.bfloat16, device="cuda")
    rows = [0, M // 2, M - 2, M - 1]
    for r in rows:
        x[r] = torch.randn(K, generator=torch.Generator().manual_seed(r)).bfloat16().cuda()
    codes, scales = b.razer_quant_i8(x)
    want_codes, want_scales = quantize64(x[rows].double().cpu().numpy())
    assert np.array_equal(codes[rows].cpu().numpy(), want_codes) and np.array_equal(scales[rows].cpu().numpy(), want_scales)
    assert (codes[1] == 127).all() and (codes[M - 3] == 127).all()
