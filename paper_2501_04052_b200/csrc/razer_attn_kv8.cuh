// What the attention kernels over the 8-bit cache share: arguments, the way through the work, the end of a unit.
//
// A unit is a row tile (tq tokens x Gc query heads of one key-value head) of a sequence, an item a tile of tokens of a unit.  The batch's
// items, in the order sequence, row tile, head, tile, are cut into equal runs, one a CTA, whatever the sequences' lengths are; every CTA
// works its run out from q_start and kv_len, so that the host needs neither.  A unit inside a run is finished by its CTA.  Of one that
// several CTAs share each leaves its part (sums with the maxima that they are relative to) in the workspace; the last to arrive adds
// them up in CTA order, and leaves the counter zero.
#pragma once

#include "razer_common.cuh"
#include "razer_kv8.cuh"
#include "razer_tcgen05.cuh"

namespace razer {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct AttnArgs {
  Kv8 c;
  Kv8Batch s;
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  float* lse;
  uint32_t *status, *counters;
  float* parts;
  long long q_stride;
  float scale;
  int G, Gc, chunks, tq;     // query heads per key-value head; per row tile; row tiles of heads; tokens of a row tile
};

__device__ __forceinline__ float power2(int n) { return __int_as_float((n + 127) << 23); }       // -126 <= n <= 127
__device__ __forceinline__ float ex2(float x) {         // 2 ulp; 0 below 2^-126; exact in 0 and -infinity
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Pairs of FP32 numbers, two a instruction.
__device__ __forceinline__ uint64_t pair64(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float low64(uint64_t v) {
  float lo;
  asm("{\n\t.reg .f32 hi;\n\tmov.b64 {%0, hi}, %1;\n\t}" : "=f"(lo) : "l"(v));
  return lo;
}
__device__ __forceinline__ float high64(uint64_t v) {
  float hi;
  asm("{\n\t.reg .f32 lo;\n\tmov.b64 {lo, %0}, %1;\n\t}" : "=f"(hi) : "l"(v));
  return hi;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
template <int N>
__device__ __forceinline__ void threads_meet() { asm volatile("bar.sync 1, %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void group_meet(int group) { asm volatile("bar.sync %0, 128;" ::"r"(2 + group) : "memory"); }
// The factor by which what was summed at maximum `m` counts at maximum `top`; sums of nothing count nothing, NaN stays.
__device__ __forceinline__ float rebase(float m, float l, float top) { return m == -INFINITY && l == 0.0f ? 0.0f : ex2(m - top); }

// A place in a CTA's work: segments, each the part of one unit that falls to it.
struct Walk {
  int b, row0, n, len, tiles, units, unit, tile;
  bool over;                                             // longer than its table: its rows are NaN
  long long left;                                        // items that remain to the CTA
};
// Sequence b and its number of items.
__device__ __forceinline__ long long walk_enter(const AttnArgs& a, int tokens, int b, Walk& w) {
  Kv8Seq q = kv8_seq(a.s, b);
  w.over = kv8_over(a.c, a.s, q.len);
  if (w.over) q.len = q.n;                               // a key for each row, whatever page it is on
  w.b = b, w.row0 = q.row0, w.n = q.n, w.len = q.len;
  w.tiles = max((q.len + tokens - 1) / tokens, 1);
  w.units = (q.n + a.tq - 1) / a.tq * a.c.heads * a.chunks;
  return (long long)w.units * w.tiles;
}
__device__ __forceinline__ int walk_count(const Walk& w) { return (int)min((long long)(w.tiles - w.tile), w.left); }
// On to the next segment, n items further; false at the end.
__device__ __forceinline__ bool walk_advance(const AttnArgs& a, int tokens, Walk& w, int n) {
  w.left -= n;
  if (w.left <= 0) return false;
  w.tile = 0;
  if (++w.unit < w.units) return true;
  w.unit = 0;
  do walk_enter(a, tokens, w.b + 1, w);
  while (w.units == 0);
  return true;
}
// The run of items [begin, end) of the CTA or pair of CTAs `share` of `shares`, `per` to each, and the place where it begins; false if it has none.  All threads; `words`: four words, and
// `sums` one long long a warp, of shared memory.
template <int THREADS>
__device__ __forceinline__ bool attn_share(const AttnArgs& a, int tokens, int* words, long long* sums, long long& begin, long long& end, long long& per, Walk& at,
                                           int share, int shares) {
  constexpr int WARPS = THREADS / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool once = a.s.B <= THREADS;                    // every sequence has a thread: one look at it is enough
  long long total = 0, mine = 0;
  for (int b = threadIdx.x; b < a.s.B; b += THREADS) total += mine = walk_enter(a, tokens, b, at);
  long long base = 0;                                    // items of the sequences before those looked at
  if (!once) {
    for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, o);
    if (lane == 0) sums[warp] = total;
    __syncthreads();
    total = 0;
    for (int w = 0; w < WARPS; ++w) total += sums[w];
  }
#pragma unroll 1
  for (int b0 = 0;; b0 += THREADS) {
    if (!once) mine = b0 + (int)threadIdx.x < a.s.B ? walk_enter(a, tokens, b0 + threadIdx.x, at) : 0;
    long long upto = mine;
    for (int o = 1; o < 32; o <<= 1) {
      const long long v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
      if (lane >= o) upto += v;
    }
    if (!once) __syncthreads();                          // the sums of the round before have been read
    if (lane == 31) sums[warp] = upto;
    __syncthreads();
    long long before = base, all = 0;
    for (int w = 0; w < WARPS; ++w) {
      const long long v = sums[w];
      if (w < warp) before += v;
      all += v;
    }
    base += all;
    if (once) total = all;
    if (b0 == 0) {
      per = (total + shares - 1) / shares;
      begin = per * share;
      end = min(begin + per, total);
      if (begin >= end) return false;
    }
    if (before + upto - mine <= begin && begin < before + upto) {
      words[0] = b0 + threadIdx.x;
      *reinterpret_cast<long long*>(words + 2) = begin - (before + upto - mine);
    }
    if (base > begin) break;
  }
  __syncthreads();
  const long long into = *reinterpret_cast<long long*>(words + 2);
  walk_enter(a, tokens, words[0], at);
  at.unit = (int)(into / at.tiles);
  at.tile = (int)(into - (long long)at.unit * at.tiles);
  at.left = end - begin;
  return true;
}

// Four dimensions of an output row: sums of weights exp2(s + log2 vs - ta) against sum_l of exp2(s - tm).
template <int D>
__device__ __forceinline__ void attn_store(const AttnArgs& a, long long row, int d, float4 sum, float sum_l, float ta, float tm) {
  const bool none = sum_l == 0.0f;
  const float f = none ? 0.0f : (ta == -INFINITY ? 0.0f : ex2(ta - tm)) / sum_l;
  __nv_bfloat162 lo = __floats2bfloat162_rn(none ? 0.0f : sum.x * f, none ? 0.0f : sum.y * f);
  __nv_bfloat162 hi = __floats2bfloat162_rn(none ? 0.0f : sum.z * f, none ? 0.0f : sum.w * f);
  *reinterpret_cast<uint2*>(a.out + row * D + d) = make_uint2(*reinterpret_cast<uint32_t*>(&lo), *reinterpret_cast<uint32_t*>(&hi));
  if (d == 0 && a.lse) a.lse[row] = none ? -INFINITY : (tm + log2f(sum_l)) * LN2;
}

constexpr int ATTN_CTAS = 152;                            // CTAs of a launch at most

// The CTA has left its part of a unit that others share ([R][D] sums, then [R] ta, tm, sum_l; a CTA's first unit in its slot 0, its last in
// slot 1); the last of them to come here finishes it.  THREADS threads (threads_meet); `flag`: a word of shared memory, `scratch`: (ATTN_CTAS + 3) R floats.
// Code that runs once is held short: what a CTA does not have in its instruction cache costs it some 15 cycles an instruction (16 parts put together by
// code unrolled eight times 8900 cycles).
template <int D, int R, int THREADS, int PART_FLOATS>
__device__ __forceinline__ void attn_combine(const AttnArgs& a, const Walk& at, int qt, int h, int chunk, long long unit_begin, long long per, int* flag, float* scratch) {
  const int c_first = (int)(unit_begin / per), parts = (int)((unit_begin + at.tiles - 1) / per) - c_first + 1;
  threads_meet<THREADS>();
  if (threadIdx.x == 0) {
    // release: the part's stores (ordered before this by the meeting) become visible with the count; acquire: so do the others' to what follows the
    // next meeting
    uint32_t seen;
    asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(seen) : "l"(a.counters + c_first) : "memory");
    *flag = seen == (uint32_t)(parts - 1);
    if (*flag) a.counters[c_first] = 0;                  // ready for the next call
  }
  threads_meet<THREADS>();
  if (!*flag) return;
  const float* p0 = a.parts + ((long long)c_first * 2 + 1) * PART_FLOATS;              // the first CTA's; the others' lie 2 PART_FLOATS apart from the next slot 0 on
  auto part = [&](int c) { return p0 + (c > 0 ? (long long)(2 * c - 1) * PART_FLOATS : 0); };
  const int lane = threadIdx.x & 31;
  float* rows = scratch + ATTN_CTAS * R;                 // [R] ta, tm, sum_l
#pragma unroll 1
  for (int r = threadIdx.x >> 5; r < R; r += THREADS / 32) {
    float ta = -INFINITY, tm = -INFINITY, sum_l = 0.0f;
#pragma unroll 1
    for (int c = lane; c < parts; c += 32) {
      const float* p = part(c) + R * D + r;
      const float ac = __ldcg(p), mc = __ldcg(p + R), lc = __ldcg(p + 2 * R), nm = fmaxf(tm, mc);
      scratch[c * R + r] = ac;
      ta = fmaxf(ta, ac);
      sum_l = rebase(tm, sum_l, nm) * sum_l + rebase(mc, lc, nm) * lc;
      tm = nm;
    }
    float top = tm;
    for (int x = 16; x; x >>= 1) {
      ta = fmaxf(ta, __shfl_xor_sync(0xFFFFFFFFu, ta, x));
      top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
    }
    sum_l *= rebase(tm, sum_l, top);
    for (int x = 16; x; x >>= 1) sum_l += __shfl_xor_sync(0xFFFFFFFFu, sum_l, x);
    for (int c = lane; c < parts; c += 32) {
      const float ac = scratch[c * R + r];
      scratch[c * R + r] = ac == -INFINITY ? 0.0f : ex2(ac - ta);
    }
    if (lane == 0) rows[r] = ta, rows[R + r] = top, rows[2 * R + r] = sum_l;
  }
  threads_meet<THREADS>();
#pragma unroll 1
  for (int x = threadIdx.x; x < R * (D / 4); x += THREADS) {
    const int r = x / (D / 4), d = x % (D / 4) * 4;
    const int i = qt * a.tq + r / a.Gc, hq = chunk * a.Gc + r % a.Gc;
    if (!(r < a.tq * a.Gc && i < at.n && hq < a.G)) continue;
    float4 sum = make_float4(0, 0, 0, 0);
#pragma unroll 4
    for (int c = 0; c < parts; ++c) {
      const float4 v = __ldcg(reinterpret_cast<const float4*>(part(c) + r * D + d));
      const float f = scratch[c * R + r];
      sum.x += f * v.x;
      sum.y += f * v.y;
      sum.z += f * v.z;
      sum.w += f * v.w;
    }
    attn_store<D>(a, (long long)(at.row0 + i) * a.c.heads * a.G + h * a.G + hq, d, sum, rows[2 * R + r], rows[r], rows[R + r]);
  }
}

// A tensor map over a pool of codes: (dimension, token of the page, page and head), boxes of `rows` tokens and `columns` (64 or 128) of their
// dimensions.
static inline int attn_encode_pool(CUtensorMap* map, const void* p, const Kv8& c, int rows, int columns) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return set_error(RAZER_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
  const cuuint64_t dims[3] = {(cuuint64_t)c.D, (cuuint64_t)c.page, (cuuint64_t)c.pages * c.heads};
  const cuuint64_t strides[2] = {(cuuint64_t)c.D, (cuuint64_t)c.D * c.page};
  const cuuint32_t box[3] = {(cuuint32_t)columns, (cuuint32_t)rows, 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  const CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         columns == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return set_error(RAZER_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d", (int)r);
  return RAZER_OK;
}

}  // namespace razer
