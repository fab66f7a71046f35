// Rows to 8-bit integers with a scale each: tokens online, weight channels offline (razer_quant_i8).
//
// One pass: a row's values stay in registers from its maximum to its codes.  WARPS warps share a row, VPT 16-byte vectors a thread;
// the host takes the fewest warps that hold the row with VPT <= 4, so that a single token spreads over a whole CTA (latency).  In flight a CTA has its rows: four of up to
// 2 KB, or one of 2 to 64 KB (4096 FP32: 16).  Rows too long for that (over 32 K of bf16, 16 K of FP32) are read twice, the second time
// from L2.  Bound by HBM from some MB on; the arithmetic is about 7 instructions an element (razer_i8.cuh).  11008 rows of 4096 FP32 35.4 us (6.4 TB/s),
// 333 of 11008 bf16 4.5 (2.4 TB/s, the launch is half of it), one of 4096 1.9 in a graph; a call from the host 4.7, two allocations included.
#include "razer_common.cuh"
#include "razer_i8.cuh"
#include "razer_ptx.cuh"

namespace razer {

namespace {

template <bool FP32>
__device__ __forceinline__ uint32_t vec_top(uint32_t top, uint4 v) {
  if (FP32) return max(max(max(top, v.x & 0x7FFFFFFFu), max(v.y & 0x7FFFFFFFu, v.z & 0x7FFFFFFFu)), v.w & 0x7FFFFFFFu);
  return bf16_pair_max(bf16_pair_max(bf16_pair_max(bf16_pair_max(top, v.x), v.y), v.z), v.w);
}

// The codes of a vector: 4 (FP32) or 8 (bf16).
template <bool FP32>
__device__ __forceinline__ void vec_store(uint4 v, const I8Step& t, int8_t* row, long long i) {
  if (FP32) {
    const float x[4] = {__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w)};
    uint32_t c[1];
    i8_round<4>(x, t, c);
    reinterpret_cast<uint32_t*>(row)[i] = c[0];
  } else {
    const float x[8] = {bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y), bf16_lo(v.z), bf16_hi(v.z), bf16_lo(v.w), bf16_hi(v.w)};
    uint32_t c[2];
    i8_round<8>(x, t, c);
    reinterpret_cast<uint2*>(row)[i] = make_uint2(c[0], c[1]);
  }
}

// ROWS rows a CTA, WARPS warps a row.  HELD: the row fits the threads' registers.
template <bool FP32, int WARPS, int ROWS, int VPT, bool HELD>
__global__ void __launch_bounds__(32 * WARPS * ROWS) quant_i8_kernel(const uint4* x, int M, int vecs, long long row_vecs,
                                                                     int8_t* codes, float* scales) {
  constexpr int TPR = 32 * WARPS;
  __shared__ uint32_t tops[WARPS > 1 ? WARPS * ROWS : 1];
  const int at = threadIdx.x % TPR, r = threadIdx.x / TPR;
  const long long m = (long long)blockIdx.x * ROWS + r;
  grid_dep_wait();
  grid_dep_launch();
  const bool live = m < M;
  const uint4* src = x + (live ? m : 0) * row_vecs;
  const int n = live ? vecs : 0;
  uint4 v[VPT];
  uint32_t top = 0;
  if (HELD) {
#pragma unroll
    for (int j = 0; j < VPT; ++j) v[j] = at + j * TPR < n ? src[at + j * TPR] : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < VPT; ++j) top = vec_top<FP32>(top, v[j]);
  } else {
    for (int i0 = at; i0 < n; i0 += VPT * TPR) {
#pragma unroll
      for (int j = 0; j < VPT; ++j) v[j] = i0 + j * TPR < n ? src[i0 + j * TPR] : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int j = 0; j < VPT; ++j) top = vec_top<FP32>(top, v[j]);
    }
  }
  if (!FP32) top = bf16_pair_top(top);
  top = __reduce_max_sync(0xFFFFFFFFu, top);
  if (WARPS > 1) {
    if (threadIdx.x % 32 == 0) tops[threadIdx.x / 32] = top;
    __syncthreads();
    const int lane = threadIdx.x % 32;
    top = __reduce_max_sync(0xFFFFFFFFu, lane < WARPS ? tops[r * WARPS + lane] : 0u);
  }
  if (!live) return;
  const I8Step t = i8_step(i8_scale(top));
  if (at == 0) scales[m] = t.s;
  int8_t* row = codes + m * (FP32 ? 4LL : 8LL) * vecs;
  if (HELD) {
#pragma unroll
    for (int j = 0; j < VPT; ++j)
      if (at + j * TPR < n) vec_store<FP32>(v[j], t, row, at + j * TPR);
  } else {
    for (int i = at; i < n; i += TPR) vec_store<FP32>(src[i], t, row, i);
  }
}

template <bool FP32, int WARPS, int ROWS, int VPT, bool HELD>
int launch_as(const void* x, int M, int vecs, long long row_vecs, int8_t* codes, float* scales, cudaStream_t st) {
  return launch_dependent("quant_i8_kernel launch", quant_i8_kernel<FP32, WARPS, ROWS, VPT, HELD>, ((long long)M + ROWS - 1) / ROWS, 32 * WARPS * ROWS, 0, st,
                          (const uint4*)x, M, vecs, row_vecs, codes, scales);
}

template <bool FP32>
int launch_for(const void* x, int M, int vecs, long long row_vecs, int8_t* codes, float* scales, cudaStream_t st) {
  if (vecs <= 32) return launch_as<FP32, 1, 4, 1, true>(x, M, vecs, row_vecs, codes, scales, st);
  if (vecs <= 128) return launch_as<FP32, 1, 4, 4, true>(x, M, vecs, row_vecs, codes, scales, st);
  if (vecs <= 512) return launch_as<FP32, 4, 1, 4, true>(x, M, vecs, row_vecs, codes, scales, st);
  if (vecs <= 1024) return launch_as<FP32, 8, 1, 4, true>(x, M, vecs, row_vecs, codes, scales, st);
  if (vecs <= 2048) return launch_as<FP32, 16, 1, 4, true>(x, M, vecs, row_vecs, codes, scales, st);
  if (vecs <= 4096) return launch_as<FP32, 32, 1, 4, true>(x, M, vecs, row_vecs, codes, scales, st);
  return launch_as<FP32, 32, 1, 4, false>(x, M, vecs, row_vecs, codes, scales, st);
}

}  // namespace

int launch_quant_i8(const void* x, int x_is_fp32, int M, int K, long long row_stride, int8_t* codes, float* scales, cudaStream_t st) {
  const int per = x_is_fp32 ? 4 : 8;
  return x_is_fp32 ? launch_for<true>(x, M, K / per, row_stride / per, codes, scales, st) : launch_for<false>(x, M, K / per, row_stride / per, codes, scales, st);
}

}  // namespace razer
