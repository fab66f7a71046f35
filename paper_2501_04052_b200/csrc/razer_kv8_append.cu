// New keys and values into the 8-bit cache (razer_kv8_append).
//
// For each page and head that gets tokens: a = the largest new magnitude, s = max(s0, fl32(a / 127)) with s0 the page's scale so far
// (0 where its first token is new); where s > s0 > 0 the page's other codes become the nearest integers to q s0 / s, then the new
// codes are written.  One CTA per (page that may get tokens, head, key or value): its new values stay in registers from their maximum to their
// codes, and a code that moves to the new scale does so by a table of 256.  Which page a CTA has follows from q_start alone: sequence b has the
// slots from q_start[b] / page + 2 b on, which is room enough (n tokens touch at most n / page + 2 pages), so that the grid T / page + 2 B needs
// nothing from the device.  What bounds it: latency for a decode step (a chain of five loads: 64 tokens x 8 heads 3.7 us
// a call), for prompts the same chain in three rounds of CTAs and the bytes (46 MB 13.4 us in a graph, 3.4 TB/s, 14.7 a call from the host).
#include "razer_common.cuh"
#include "razer_i8.cuh"
#include "razer_kv8.cuh"
#include "razer_ptx.cuh"

namespace razer {

namespace {

// 14.3 M values in pages of 64 x 128, in a graph: 128 threads 14.2 us, 256 13.4, 512 19.1
constexpr int append_threads(int D, int page) { return D * page >= 8192 ? 256 : 128; }

template <int D, int PAGE>
__global__ void __launch_bounds__(append_threads(D, PAGE)) kv8_append_kernel(const __grid_constant__ Kv8 c, const __grid_constant__ Kv8Batch s,
                                                                             const __nv_bfloat16* k_new, const __nv_bfloat16* v_new,
                                                                             long long k_stride, long long v_stride) {
  constexpr int THREADS = append_threads(D, PAGE), VECS = D / 8, VPT = (PAGE * VECS + THREADS - 1) / THREADS;   // vectors of 8 values, of a row and of a thread
  constexpr int LOG2 = PAGE == 16 ? 4 : PAGE == 32 ? 5 : PAGE == 64 ? 6 : 7;
  __shared__ uint32_t tops[THREADS / 32];
  __shared__ int8_t moved[256];
  const int slot = blockIdx.x, head = blockIdx.y % c.heads, tid = threadIdx.x;
  const bool value = blockIdx.y >= (unsigned)c.heads;
  grid_dep_wait();
  grid_dep_launch();
  int before = 0;                                            // sequences whose slots begin at or before this one
  for (int b0 = 0; b0 < s.B; b0 += THREADS) {
    const int b = b0 + tid;
    const bool here = b < s.B && (long long)(max(s.q_start[b], 0) >> LOG2) + 2LL * b <= slot;
    before += __syncthreads_count(here);
  }
  if (before == 0) return;
  const int b = before - 1;
  const Kv8Seq q = kv8_seq(s, b);
  const int first = q.len - q.n, block = (max(first, 0) >> LOG2) + slot - ((q.row0 >> LOG2) + 2 * b);
  const long long begin = (long long)block << LOG2;
  if (q.n == 0 || block < 0 || begin >= q.len) return;     // (no block below 0 where q_start does not decrease)
  const int lo = max(first, (int)begin), hi = (int)min((long long)q.len, begin + PAGE);
  if (lo >= hi) return;
  const int page = kv8_page(c, s, b, block);                 // asked for, and looked at when the new values are on their way too
  const int r0 = lo - (int)begin, rows = hi - lo;            // rows of the page
  const long long stride = value ? v_stride : k_stride;
  const __nv_bfloat16* src = (value ? v_new : k_new) + (long long)(q.row0 + lo - first) * stride + (long long)head * D;
  uint4 x[VPT];
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = tid + j * THREADS, r = i / VECS;
    x[j] = r < rows ? *reinterpret_cast<const uint4*>(src + (long long)r * stride + i % VECS * 8) : make_uint4(0, 0, 0, 0);
  }
  if (page < 0) return;
  int8_t* codes = (value ? c.v : c.k) + ((long long)page * c.heads + head) * PAGE * D;
  float* scale = (value ? c.v_scales : c.k_scales) + (long long)page * c.heads + head;
  const float s0 = r0 > 0 ? *scale : 0.0f;
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < VPT; ++j) top = bf16_pair_max(bf16_pair_max(bf16_pair_max(bf16_pair_max(top, x[j].x), x[j].y), x[j].z), x[j].w);
  top = __reduce_max_sync(0xFFFFFFFFu, bf16_pair_top(top));
  if ((tid & 31) == 0) tops[tid >> 5] = top;
  __syncthreads();                                           // also: everyone has read the old scale
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) top = max(top, tops[w]);
  const float fresh = i8_scale(top);
  const bool broken = !(fresh < __uint_as_float(0x7F800000u)) || !(fabsf(s0) < __uint_as_float(0x7F800000u));
  const float now = broken ? __uint_as_float(0x7FC00000u) : fmaxf(s0, fresh);
  const I8Step t = i8_step(now);
  if (tid == 0) *scale = now;
  if (s0 > 0.0f && now > s0) {                               // false where one is NaN
    for (int i = tid; i < 256; i += THREADS) moved[i] = (int8_t)(int)rint((double)(int8_t)i * (double)s0 / (double)now);
    __syncthreads();
    uint32_t* words = reinterpret_cast<uint32_t*>(codes);
    for (int i = tid; i < PAGE * D / 4; i += THREADS) {
      const int r = i / (D / 4);
      if (r >= r0 && r < r0 + rows) continue;
      const uint32_t w = words[i];
      words[i] = (uint32_t)(uint8_t)moved[w & 255] | (uint32_t)(uint8_t)moved[(w >> 8) & 255] << 8 | (uint32_t)(uint8_t)moved[(w >> 16) & 255] << 16 |
                 (uint32_t)(uint8_t)moved[w >> 24] << 24;
    }
  }
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = tid + j * THREADS;
    if (i / VECS >= rows) break;
    const float f[8] = {bf16_lo(x[j].x), bf16_hi(x[j].x), bf16_lo(x[j].y), bf16_hi(x[j].y), bf16_lo(x[j].z), bf16_hi(x[j].z), bf16_lo(x[j].w), bf16_hi(x[j].w)};
    uint32_t o[2];
    i8_round<8>(f, t, o);
    *reinterpret_cast<uint2*>(codes + (long long)r0 * D + i * 8) = make_uint2(o[0], o[1]);
  }
}

template <int D, int PAGE>
int launch_as(const Kv8& c, const Kv8Batch& s, const void* k_new, const void* v_new, long long k_stride, long long v_stride, cudaStream_t st) {
  const long long slots = (long long)(s.T / PAGE) + 2LL * s.B;
  if (slots > 0x7FFFFFFFll) return set_error(RAZER_ERR_UNSUPPORTED, "%d tokens of %d sequences: more pages than a launch has", s.T, s.B);
  return launch_dependent_clusters("kv8_append_kernel launch", kv8_append_kernel<D, PAGE>, dim3((unsigned)slots, 2u * c.heads), 1, append_threads(D, PAGE), 0, st, c, s,
                                   (const __nv_bfloat16*)k_new, (const __nv_bfloat16*)v_new, k_stride, v_stride);
}

template <int D>
int launch_for(const Kv8& c, const Kv8Batch& s, const void* k_new, const void* v_new, long long k_stride, long long v_stride, cudaStream_t st) {
  switch (c.page) {
    case 16: return launch_as<D, 16>(c, s, k_new, v_new, k_stride, v_stride, st);
    case 32: return launch_as<D, 32>(c, s, k_new, v_new, k_stride, v_stride, st);
    case 64: return launch_as<D, 64>(c, s, k_new, v_new, k_stride, v_stride, st);
    default: return launch_as<D, 128>(c, s, k_new, v_new, k_stride, v_stride, st);
  }
}

}  // namespace

int launch_kv8_append(const Kv8& c, const Kv8Batch& s, const void* k_new, const void* v_new, long long k_stride, long long v_stride, cudaStream_t st) {
  return c.D == 64 ? launch_for<64>(c, s, k_new, v_new, k_stride, v_stride, st) : launch_for<128>(c, s, k_new, v_new, k_stride, v_stride, st);
}

}  // namespace razer
