// Attention over the paged 8-bit cache (razer_attn_kv8).
//
//   s_j = scale * ks[page(j)] * <q, kq_j>   over the keys j <= p of a row at position p
//   out = sum_j exp(s_j) vs[page(j)] vq_j / sum_j exp(s_j),   lse = log sum_j exp(s_j)
//
// One pass over the cache with a running maximum and sum.  A work item is a tile of TK tokens of one (sequence, row tile, key-value
// head), and all items of the batch are cut evenly among the CTAs, whatever the sequences' lengths are: every CTA works its share out
// from q_start and kv_len, so that the host needs neither.  Item i of a CTA belongs to warp i % NW, which has a ring and a softmax of
// its own: it looks the pages up and brings their rows by TMA itself, RING tiles ahead and across the units' ends (one producer warp for all
// took 900 cycles a tile and bounded the kernel at 2.5 TB/s).  The warps meet at the end of a unit.  A unit that several CTAs share is put together
// in CTA order by the last of them to arrive (counters that reset themselves, parts in the workspace).
//
// Both products run with the cache as operand A (16 tokens x 16 dimensions, then 16 dimensions x 16 tokens) and the rows of queries as
// the eight columns of B, so that a decode step of up to 8 query heads a key-value head wastes nothing, and O takes 32 registers for 8 rows.
// Codes become f16 exactly: byte ^ 0x80 under an exponent of 2^10 is 1152 + code, and a packed subtraction leaves the code.  Queries go to
// f16 too, each row by its own power of two (largest magnitude in [2^14, 2^15): what falls below the f16 range is less than 2^-38 of it).
// Probabilities p <= 1 are held as f16 times 2^14, 11 significant bits where bf16 would keep 8 and 38 binades; the value scales
// enter there, relative to the largest one met so far.
#include "razer_common.cuh"
#include "razer_kv8.cuh"
#include "razer_tcgen05.cuh"

#include <cuda_fp16.h>

namespace razer {

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float P_ONE = 16384.0f;                        // what a probability of 1 is held as

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

template <int D_, int NB_>
struct AttnCfg {
  static constexpr int D = D_, NB = NB_, ROWS = 8 * NB_;
  static constexpr int NW = 8, RING = 3;                 // warps, tiles of each warp's ring
  static constexpr int THREADS = 32 * NW;
  static constexpr int TK = D_ == 64 ? 64 : 32;          // tokens of a tile
  static constexpr int MT = TK / 16;
  static constexpr int TILE_BYTES = TK * D;
  static constexpr int STAGE_BYTES = 2 * TILE_BYTES;
  static constexpr int STAGES = RING * NW;
  static constexpr int HALF = D / 2;                     // columns of O that the warps put together at a time
  static constexpr int PITCH = HALF + 4;
  static constexpr int O_RING = 0;
  static constexpr int O_META = STAGES * STAGE_BYTES;                    // [STAGES][MT] key and value scale
  static constexpr int O_Q = O_META + STAGES * MT * 8;                   // [D / 16][NB][32 lanes] two registers of B
  static constexpr int O_JOIN = O_Q + (D / 16) * NB * 256;               // [NW][8][PITCH]
  static constexpr int O_STAT = O_JOIN + NW * 8 * PITCH * 4;             // [NW][ROWS] maximum, then sum; [NW] value scale
  static constexpr int O_ROW = (O_STAT + (2 * NW * ROWS + NW) * 4 + 7) / 8 * 8;   // [ROWS] score factor in two parts; [ROWS] visible keys
  static constexpr int O_BAR = (O_ROW + 3 * ROWS * 4 + 15) / 16 * 16;
  static constexpr int O_MISC = O_BAR + STAGES * 8;                     // words: see below
  static constexpr int SMEM_BYTES = 1024 + O_MISC + 128;
  static constexpr int PART_FLOATS = ROWS * (D + 2);                     // a part: O, maxima, sums
};

__device__ __forceinline__ uint32_t half_pair(uint32_t bytes02) {        // codes in bytes 0 and 2 -> f16 pair
  const uint32_t h = (bytes02 & 0x00FF00FFu) ^ 0x64806480u;
  const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&h), __half2half2(__ushort_as_half(0x6480)));
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float power2(int n) { return __int_as_float((n + 127) << 23); }       // -126 <= n <= 127
__device__ __forceinline__ float ex2(float x) {         // 2 ulp; 0 below 2^-126; exact in 0 and -infinity
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
template <int N>
__device__ __forceinline__ void threads_meet() { asm volatile("bar.sync 1, %0;" ::"n"(N) : "memory"); }
// The factor by which what was summed at maximum `m` counts at maximum `top`; sums of nothing count nothing, NaN stays.
__device__ __forceinline__ float rebase(float m, float l, float top) {
  return m == -INFINITY && l == 0.0f ? 0.0f : ex2(m - top);
}
// Row r of a 16-row tile of A is token spread(r) of the tile's 16: rows 2j and 2j + 1 are four apart, so that the 16-byte reads of
// a quarter warp meet no bank twice in either product (64 dimensions: values twice).
__device__ __forceinline__ int spread(int r) { return (r & 8) | ((r & 1) ? ((r & 6) ^ 4) | 1 : (r & 6)); }

// A place in a CTA's work: segments, each the part of one unit that falls to it.
struct Walk {
  int b, row0, n, len, tiles, units, unit, tile;
  long long left;                                        // items that remain to the CTA
};

template <int D, int NB>
__global__ void __launch_bounds__(AttnCfg<D, NB>::THREADS, 1) attn_kv8_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                                                                   const __grid_constant__ AttnArgs a) {
  using C = AttnCfg<D, NB>;
  constexpr int NW = C::NW, TK = C::TK, MT = C::MT, ROWS = C::ROWS, ST = C::STAGES;
  extern __shared__ uint8_t attn_smem[];
  uint8_t* sm = attn_smem + ((1024 - (smem_u32(attn_smem) & 1023)) & 1023);
  const uint32_t sb = smem_u32(sm);
  float2* meta = reinterpret_cast<float2*>(sm + C::O_META);
  float* stat_m = reinterpret_cast<float*>(sm + C::O_STAT);
  float* stat_l = stat_m + NW * ROWS;
  float* stat_v = stat_l + NW * ROWS;
  float* row_scale = reinterpret_cast<float*>(sm + C::O_ROW);
  int* row_keys = reinterpret_cast<int*>(row_scale + 2 * ROWS);
  const uint32_t bar_full = sb + C::O_BAR;
  volatile uint32_t* abort_flag = reinterpret_cast<uint32_t*>(sm + C::O_MISC);
  int* misc = reinterpret_cast<int*>(sm + C::O_MISC);    // 0 abort, 1 a flag that nobody sets, 2 sequence, 3 last to arrive, 4.. warps' sums (long long)
  long long* sums = reinterpret_cast<long long*>(misc + 6);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < ST; ++i) {
      mbar_init(bar_full + 8 * i, 1);
    }
    misc[0] = misc[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
  }
  grid_dep_wait();
  grid_dep_launch();

  // ---- this CTA's share: items in the order sequence, row tile, head, tile
  const int heads = a.c.heads * a.chunks;
  auto weigh = [&](int b, Kv8Seq& q, int& tiles) -> long long {
    q = kv8_seq(a.s, b);
    if (kv8_over(a.c, a.s, q.len)) q.len = q.n;          // its rows will be NaN: a key for each, whatever page it is on
    tiles = max((q.len + TK - 1) / TK, 1);
    return (long long)((q.n + a.tq - 1) / a.tq) * heads * tiles;
  };
  long long total = 0;
  {
    Kv8Seq q;
    int tiles;
    for (int b = threadIdx.x; b < a.s.B; b += C::THREADS) total += weigh(b, q, tiles);
    for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, o);
    if (lane == 0) sums[warp] = total;
    __syncthreads();
    total = 0;
    for (int w = 0; w < NW; ++w) total += sums[w];
  }
  const long long per = (total + gridDim.x - 1) / gridDim.x;
  const long long begin = per * blockIdx.x, end = min(begin + per, total);
  if (begin >= end) return;                              // nobody has a barrier or a copy in flight yet
  Walk at;
  {
    long long base = 0;                                  // items of the sequences before this round's
    Kv8Seq q;
    int tiles;
    for (int b0 = 0;; b0 += C::THREADS) {
      const int b = b0 + threadIdx.x;
      const long long mine = b < a.s.B ? weigh(b, q, tiles) : 0;
      long long upto = mine;
      for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
        if (lane >= o) upto += v;
      }
      __syncthreads();                                   // sums[] of the round before has been read
      if (lane == 31) sums[warp] = upto;
      __syncthreads();
      long long before = base;
      for (int w = 0; w < warp; ++w) before += sums[w];
      for (int w = 0; w < NW; ++w) base += sums[w];
      if (before + upto - mine <= begin && begin < before + upto) {
        misc[2] = b;
        *reinterpret_cast<long long*>(misc + 4) = begin - (before + upto - mine);
      }
      if (base > begin) break;
    }
    __syncthreads();
    at.b = misc[2];
    const long long into = *reinterpret_cast<long long*>(misc + 4);
    weigh(at.b, q, at.tiles);
    at.row0 = q.row0, at.n = q.n, at.len = q.len;
    at.units = (q.n + a.tq - 1) / a.tq * heads;
    at.unit = (int)(into / at.tiles);
    at.tile = (int)(into - (long long)at.unit * at.tiles);
    at.left = end - begin;
  }
  const long long per_items = per;
  auto count = [](const Walk& at) { return (int)min((long long)(at.tiles - at.tile), at.left); };
  auto advance = [&](Walk& at, int n) {                            // on to the next segment, n items further; false at the end
    at.left -= n;
    if (at.left <= 0) return false;
    at.tile = 0;
    if (++at.unit < at.units) return true;
    at.unit = 0;
    do {
      Kv8Seq q;
      weigh(++at.b, q, at.tiles);
      at.row0 = q.row0, at.n = q.n, at.len = q.len;
      at.units = (q.n + a.tq - 1) / a.tq * heads;
    } while (at.units == 0);
    return true;
  };
  // keys that the last row of the unit's row tile sees
  auto unit_keys = [&](const Walk& at, int qt) { return max(at.len - at.n + min((qt + 1) * a.tq, at.n), 0); };
  auto fail = [&](uint32_t code) {
    *abort_flag = 1;
    atomicCAS(a.status, 0u, code);
  };

  // ---- the warp's own loads, ahead of its sums: place in the work, the segment's tiles, the next of them for this warp
  Walk ld = at;
  const int rows_of_box = min(a.c.page, TK), boxes = TK / rows_of_box;
  int ld_base = 0, ld_i = warp, ld_n = 0, ld_tile = 0, ld_keys = 0, ld_head = 0;   // the CTA's items before the segment; tile ld_i of its ld_n
  bool ld_more = true;
  auto segment = [&]() {
    const int qt = ld.unit / heads;
    ld_head = (ld.unit - qt * heads) / a.chunks;
    ld_keys = unit_keys(ld, qt);
    ld_tile = ld.tile;
    ld_n = max(min(ld.tile + count(ld), (ld_keys + TK - 1) / TK) - ld.tile, 0);
  };
  auto settle = [&]() {                                  // to a segment that has the tile
    while (ld_i >= ld_n) {
      ld_i -= ld_n;
      if (!advance(ld, count(ld))) { ld_more = false; return; }
      segment();
    }
  };
  int ld_page = 0;                                       // lane i: the page of the next tile's box i
  auto look_up = [&]() {
    const int tok = (ld_tile + ld_i) * TK + lane * rows_of_box;
    ld_page = ld_more && lane < boxes && tok < ld_keys ? kv8_page(a.c, a.s, ld.b, tok >> a.c.page_log2) : -1;
  };
  int ld_count = 0;                                      // tiles asked for
  float new_k = 0.0f, new_v = 0.0f;                      // lane i: scales of box i of the last of them, on their way
  // Asks for the next tile, and puts down the scales of the one before, which have come by now.
  auto load_next = [&]() {
    if (ld_count > 0) {
      const int before = warp * C::RING + (ld_count - 1) % C::RING, from = lane * 16 / rows_of_box;
      const float k1 = __shfl_sync(0xFFFFFFFFu, new_k, from & 31), v1 = __shfl_sync(0xFFFFFFFFu, new_v, from & 31);
      if (lane < MT) meta[before * MT + lane] = make_float2(k1, v1);
    }
    if (!ld_more) return;
    const int stage = warp * C::RING + ld_count % C::RING, tok0 = (ld_tile + ld_i) * TK;
    const uint32_t bar = bar_full + 8 * stage;
    const int live = min(boxes, (ld_keys - tok0 - 1) / rows_of_box + 1);         // boxes with a visible key
    if (lane == 0) mbar_expect_tx(bar, (uint32_t)(live * rows_of_box * D * 2));
    __syncwarp();
    if (lane < live) {
      const int z = max(ld_page, 0) * a.c.heads + ld_head, y = (tok0 + lane * rows_of_box) & (a.c.page - 1);
      const uint32_t to = sb + C::O_RING + stage * C::STAGE_BYTES + (uint32_t)(lane * rows_of_box * D);
      tma_load_3d(to, &map_k, 0, y, z, bar);
      tma_load_3d(to + C::TILE_BYTES, &map_v, 0, y, z, bar);
      new_k = new_v = __uint_as_float(0x7FC00000u);
      if (ld_page >= 0) {
        new_k = __ldg(a.c.k_scales + (long long)ld_page * a.c.heads + ld_head);
        new_v = __ldg(a.c.v_scales + (long long)ld_page * a.c.heads + ld_head);
      }
    }
    __syncwarp();
    ++ld_count;
    ld_i += NW;
    settle();
    look_up();
  };
  segment();
  settle();
  look_up();
  for (int i = 0; i < C::RING; ++i) load_next();

  const int g = lane >> 2, t4 = lane & 3;
  int item = 0, used = 0;                                // the CTA's items before this segment; the warp's own so far
  for (;;) {
    const int n_items = count(at), qt = at.unit / heads, hc = at.unit - qt * heads, h = hc / a.chunks, chunk = hc - h * a.chunks;
    const int keys = unit_keys(at, qt), first_tile = at.tile, last = min(at.tile + n_items, (keys + TK - 1) / TK);
    // ---- the rows of queries: f16, in the order of B's fragments; row r is token r / Gc, head r % Gc of the row tile
    {
      threads_meet<32 * NW>();                                  // the unit before is done with what follows
      for (int r = warp; r < ROWS; r += NW) {
        const int i = qt * a.tq + r / a.Gc, hq = chunk * a.Gc + r % a.Gc;
        const bool real = r < a.tq * a.Gc && i < at.n && hq < a.G;
        float x[D / 32];                                 // D / 32 consecutive values a lane
        float top = 0.0f;
        bool broken = false;
        const __nv_bfloat16* src = a.q + (long long)(at.row0 + i) * a.q_stride + (long long)(h * a.G + hq) * D + lane * (D / 32);
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
          x[j] = real ? __bfloat162float(src[j]) : 0.0f;
          broken |= !(fabsf(x[j]) < INFINITY);
          top = fmaxf(top, fabsf(x[j]));
        }
        top = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top)));
        broken = __any_sync(0xFFFFFFFFu, broken || kv8_over(a.c, a.s, __ldg(a.s.kv_len + at.b)));
        // 2^e <= top < 2^(e + 1); the row times 2^(14 - e).  In two factors: the whole one may be beyond FP32's range.
        const int e = top > 0.0f && !broken ? ilogbf(top) : 0;
        const float up0 = power2((14 - e) / 2), up1 = power2(14 - e - (14 - e) / 2);
        if (lane == 0) {
          row_scale[2 * r] = broken ? __uint_as_float(0x7FC00000u) : a.scale * LOG2E * power2(e / 2);
          row_scale[2 * r + 1] = power2(e - e / 2 - 14);
          row_keys[r] = real ? max(at.len - at.n + i + 1, 0) : 0;
        }
        // dimension d = 16 c + 4 w + byte of the 16-byte chunk c: chunk c is lane t = c % 4 of steps 4 (c / 4) + w; bytes 0, 2 are the
        // pair of register 0, bytes 1, 3 that of register 1
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
          const int d = lane * (D / 32) + j, c16 = d >> 4, w = (d >> 2) & 3, byte = d & 3;
          const int step = 4 * (c16 >> 2) + w, dst_lane = (r & 7) * 4 + (c16 & 3);
          __half* to = reinterpret_cast<__half*>(sm + C::O_Q + ((step * NB + (r >> 3)) * 32 + dst_lane) * 8);
          to[(byte & 1) * 2 + (byte >> 1)] = __float2half_rn(broken ? 0.0f : x[j] * up0 * up1);
        }
      }
      threads_meet<32 * NW>();
    }
    float o[D / 16][NB][4], m[NB][2], l[NB][2], svm = 0.0f;
    float2 rs[NB][2];                                    // (in two parts, since a row's power of two may leave FP32's normal range)
    int see[NB][2], see_all = 0x7FFFFFFF;                // keys that every row sees
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int j = 0; j < D / 16; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[j][nb][i] = 0.0f;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 8 * nb + 2 * t4 + e;
        m[nb][e] = -INFINITY;
        l[nb][e] = 0.0f;
        rs[nb][e] = *reinterpret_cast<const float2*>(row_scale + 2 * r);
        see[nb][e] = row_keys[r];
      }
    }
    for (int r = 0; r < ROWS; ++r) see_all = min(see_all, row_keys[r] > 0 || r < a.tq * a.Gc ? row_keys[r] : 0x7FFFFFFF);
    const uint32_t q_at = sb + C::O_Q + lane * 8;

    const int n_stages = max(last - first_tile, 0);
    for (int i = (warp - item % NW + NW) % NW; i < n_stages; i += NW) {
      const int stage = warp * C::RING + used % C::RING, tok0 = (first_tile + i) * TK;
      if (!mbar_wait(bar_full + 8 * stage, (uint32_t)((used / C::RING) & 1), abort_flag)) fail(1);
      ++used;
      __syncwarp();
      const uint32_t kt = sb + C::O_RING + stage * C::STAGE_BYTES, vt = kt + C::TILE_BYTES;
      // ---- S = K Q^T
      float s[MT][NB][4];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[mt][nb][e] = 0.0f;
      }
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          uint4 w[2];
#pragma unroll
          for (int hh = 0; hh < 2; ++hh) {
            const int row = 16 * mt + 8 * hh + spread(g), ch = t4 + 4 * c;
            const int sw = D == 64 ? (ch ^ ((row >> 1) & 3)) : (ch ^ (row & 7));
            w[hh] = lds128(kt + row * D + sw * 16);
          }
          const uint32_t w0[4] = {w[0].x, w[0].y, w[0].z, w[0].w}, w1[4] = {w[1].x, w[1].y, w[1].z, w[1].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t a0 = half_pair(w0[k]), a2 = half_pair(w0[k] >> 8), a1 = half_pair(w1[k]), a3 = half_pair(w1[k] >> 8);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              const uint2 bq = lds64(q_at + ((4 * c + k) * NB + nb) * 256);
              mma_f16(s[mt][nb], a0, a1, a2, a3, bq.x, bq.y);
            }
          }
        }
      }
      // ---- softmax: columns are rows of queries
      float sk[MT], sv[MT], svn = svm;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const float2 f = meta[stage * MT + mt];
        const bool any = tok0 + 16 * mt < keys;          // beyond, the scale belongs to no token that anyone sees
        sk[mt] = any ? f.x : 0.0f;
        sv[mt] = any ? f.y : 0.0f;
        svn = fmaxf(svn, fabsf(sv[mt]));
      }
      const bool edge = tok0 + TK > see_all;
      const float shrink = svn > 0.0f && svn != svm ? svm / svn : 1.0f;
      svm = svn;
      float rel[MT];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) rel[mt] = sv[mt] == 0.0f ? 0.0f : P_ONE * (sv[mt] / svn);
      uint32_t pb[MT][NB][2];
      bool moved = shrink != 1.0f;
      float alpha[NB][2];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float v = s[mt][nb][e] * (sk[mt] * rs[nb][e & 1].x) * rs[nb][e & 1].y;
            if (edge && tok0 + 16 * mt + 8 * (e >> 1) + spread(g) >= see[nb][e & 1]) v = -INFINITY;
            s[mt][nb][e] = v;
            top[e & 1] = fmaxf(top[e & 1], v);
          }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) top[e] = fmaxf(top[e], __shfl_xor_sync(0xFFFFFFFFu, top[e], x));
          const float mn = fmaxf(m[nb][e], top[e]), ms = mn == -INFINITY ? 0.0f : mn;
          alpha[nb][e] = ex2(m[nb][e] - ms);
          moved |= mn != m[nb][e];
          m[nb][e] = mn;
          top[e] = ms;
          l[nb][e] *= alpha[nb][e];
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          float w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = ex2(s[mt][nb][e] - top[e & 1]);
            l[nb][e & 1] += p;
            w[e] = p * rel[mt];
            if (edge && s[mt][nb][e] == -INFINITY) w[e] = 0.0f;          // a scale that is NaN is not the hidden rows' affair
          }
          pb[mt][nb][0] = transpose8(pack_half(w[0], w[1]));
          pb[mt][nb][1] = transpose8(pack_half(w[2], w[3]));
        }
      }
      if (__any_sync(0xFFFFFFFFu, moved)) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[j][nb][e] *= alpha[nb][e & 1] * shrink;
      }
      // ---- O += V^T P: lane g has dimensions (D / 8) g .. of tokens spread(2 t), spread(2 t + 1) and those + 8
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        uint32_t w[4][D / 32];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int row = 16 * mt + spread(2 * t4 + (x & 1) + 8 * (x >> 1));
          if (D == 64) {
            const uint2 v = lds64(vt + row * D + (((g >> 1) ^ ((row >> 1) & 3)) << 4) + (g & 1) * 8);
            w[x][0] = v.x, w[x][1] = v.y;
          } else {
            const uint4 v = lds128(vt + row * D + ((g ^ (row & 7)) << 4));
            w[x][0] = v.x, w[x][1] = v.y, w[x][2 % (D / 32)] = v.z, w[x][3 % (D / 32)] = v.w;
          }
        }
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {               // dimensions 2 j and 2 j + 1 of the lane's
          const uint32_t sel = (j & 1) ? 0x7632u : 0x5410u;
          const uint32_t lo = __byte_perm(w[0][j >> 1], w[1][j >> 1], sel), hi = __byte_perm(w[2][j >> 1], w[3][j >> 1], sel);
          const uint32_t a0 = half_pair(lo), a1 = half_pair(lo >> 8), a2 = half_pair(hi), a3 = half_pair(hi >> 8);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) mma_f16(o[j][nb], a0, a1, a2, a3, pb[mt][nb][0], pb[mt][nb][1]);
        }
      }
      __syncwarp();                                      // the tile has been read
      load_next();
    }
    item += n_stages;

    // ---- the warps' parts together
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[nb][e] += __shfl_xor_sync(0xFFFFFFFFu, l[nb][e], x);
        if (g == 0) {
          stat_m[warp * ROWS + 8 * nb + 2 * t4 + e] = m[nb][e];
          stat_l[warp * ROWS + 8 * nb + 2 * t4 + e] = l[nb][e];
        }
      }
    if (lane == 0) stat_v[warp] = svm;
    threads_meet<32 * NW>();
    const bool whole = first_tile == 0 && n_items == at.tiles;
    const int slot = first_tile > 0 ? 0 : 1;             // a CTA's first unit may have begun before it, its last may go on after it
    float* part = a.parts + ((long long)blockIdx.x * 2 + slot) * C::PART_FLOATS;
    float* join = reinterpret_cast<float*>(sm + C::O_JOIN);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float f[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 8 * nb + 2 * t4 + e;
        float top = -INFINITY;
        for (int w = 0; w < NW; ++w) top = fmaxf(top, stat_m[w * ROWS + r]);
        f[e] = rebase(m[nb][e], l[nb][e], top) * (svm / P_ONE);
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if ((g >> 2) == half) {
#pragma unroll
          for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) join[(warp * 8 + 2 * t4 + (e & 1)) * C::PITCH + (g & 3) * (D / 8) + 2 * j + (e >> 1)] = o[j][nb][e] * f[e & 1];
        }
        threads_meet<32 * NW>();
        for (int x = threadIdx.x; x < 8 * C::HALF; x += 32 * NW) {
          const int rr = x / C::HALF, col = x % C::HALF, r = 8 * nb + rr;
          float top = -INFINITY, sum = 0.0f, total_l = 0.0f;
          for (int w = 0; w < NW; ++w) top = fmaxf(top, stat_m[w * ROWS + r]);
          for (int w = 0; w < NW; ++w) {
            sum += join[(w * 8 + rr) * C::PITCH + col];
            const float lw = stat_l[w * ROWS + r];
            total_l += rebase(stat_m[w * ROWS + r], lw, top) * lw;
          }
          const int d = half * C::HALF + col;
          if (whole) {
            const int i = qt * a.tq + r / a.Gc, hq = chunk * a.Gc + r % a.Gc;
            if (r < a.tq * a.Gc && i < at.n && hq < a.G) {
              const long long row = (long long)(at.row0 + i) * a.c.heads * a.G + h * a.G + hq;
              a.out[row * D + d] = __float2bfloat16_rn(total_l == 0.0f ? 0.0f : sum / total_l);
              if (d == 0 && a.lse) a.lse[row] = total_l == 0.0f ? -INFINITY : (top + log2f(total_l)) * LN2;
            }
          } else {
            __stcg(part + r * D + d, sum);
            if (d == 0) {
              __stcg(part + ROWS * D + r, top);
              __stcg(part + ROWS * D + ROWS + r, total_l);
            }
          }
        }
        threads_meet<32 * NW>();
      }
    }
    if (!whole) {
      // ---- the unit's CTAs: this one, those before it down to the unit's first item, those after up to its last
      const long long here = begin + (end - begin - at.left), unit_begin = here - first_tile, unit_end = unit_begin + at.tiles;
      const int c_first = (int)(unit_begin / per_items), c_last = (int)((unit_end - 1) / per_items);
      __threadfence();
      threads_meet<32 * NW>();
      if (threadIdx.x == 0) {
        uint32_t seen;
        asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(seen) : "l"(a.counters + c_first) : "memory");
        misc[3] = seen == (uint32_t)(c_last - c_first);
        if (misc[3]) a.counters[c_first] = 0;            // ready for the next call
      }
      threads_meet<32 * NW>();
      if (misc[3]) {
        __threadfence();
        // part of CTA c: its first unit (slot 0), except in the unit's first CTA
        for (int x = threadIdx.x; x < ROWS * (D / 4); x += 32 * NW) {
          const int r = x / (D / 4), d = x % (D / 4) * 4;
          const int i = qt * a.tq + r / a.Gc, hq = chunk * a.Gc + r % a.Gc;
          if (!(r < a.tq * a.Gc && i < at.n && hq < a.G)) continue;
          float top = -INFINITY, total_l = 0.0f;
          float4 sum = make_float4(0, 0, 0, 0);
          for (int c = c_first; c <= c_last; ++c) top = fmaxf(top, __ldcg(a.parts + ((long long)c * 2 + (c == c_first)) * C::PART_FLOATS + ROWS * D + r));
          for (int c = c_first; c <= c_last; ++c) {
            const float* p = a.parts + ((long long)c * 2 + (c == c_first)) * C::PART_FLOATS;
            const float mc = __ldcg(p + ROWS * D + r), lc = __ldcg(p + ROWS * D + ROWS + r), f = rebase(mc, lc, top);
            const float4 v = __ldcg(reinterpret_cast<const float4*>(p + r * D + d));
            total_l += f * lc;
            sum.x += f * v.x;
            sum.y += f * v.y;
            sum.z += f * v.z;
            sum.w += f * v.w;
          }
          const long long row = (long long)(at.row0 + i) * a.c.heads * a.G + h * a.G + hq;
          const float inv = 1.0f / total_l;
          const bool none = total_l == 0.0f;
          __nv_bfloat162 lo = __floats2bfloat162_rn(none ? 0.0f : sum.x * inv, none ? 0.0f : sum.y * inv);
          __nv_bfloat162 hi = __floats2bfloat162_rn(none ? 0.0f : sum.z * inv, none ? 0.0f : sum.w * inv);
          *reinterpret_cast<uint2*>(a.out + row * D + d) = make_uint2(*reinterpret_cast<uint32_t*>(&lo), *reinterpret_cast<uint32_t*>(&hi));
          if (d == 0 && a.lse) a.lse[row] = none ? -INFINITY : (top + log2f(total_l)) * LN2;
        }
      }
    }
    if (!advance(at, n_items)) break;
  }
  // after a wait that gave up: copies still in flight must land before the CTA's shared memory is released
  if (*abort_flag)
    for (int f = max(ld_count - C::RING, 0); f < ld_count; ++f)
      mbar_wait(bar_full + 8 * (warp * C::RING + f % C::RING), (uint32_t)((f / C::RING) & 1), (volatile uint32_t*)(misc + 1));
}

// A tensor map over a pool of codes: (dimension, token of the page, page and head).
int encode_pool(CUtensorMap* map, const void* p, const Kv8& c, int rows) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return set_error(RAZER_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
  const cuuint64_t dims[3] = {(cuuint64_t)c.D, (cuuint64_t)c.page, (cuuint64_t)c.pages * c.heads};
  const cuuint64_t strides[2] = {(cuuint64_t)c.D, (cuuint64_t)c.D * c.page};
  const cuuint32_t box[3] = {(cuuint32_t)c.D, (cuuint32_t)rows, 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  const CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         c.D == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return set_error(RAZER_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d", (int)r);
  return RAZER_OK;
}

template <int D, int NB>
int launch_as(AttnArgs& a, cudaStream_t st) {
  using C = AttnCfg<D, NB>;
  static_assert(C::SMEM_BYTES <= 232448, "shared memory of a CTA");
  a.Gc = a.G < C::ROWS ? a.G : C::ROWS;
  a.chunks = (a.G + a.Gc - 1) / a.Gc;
  a.tq = C::ROWS / a.Gc;
  CUtensorMap map_k, map_v;
  const int rows = a.c.page < C::TK ? a.c.page : C::TK;
  RAZER_TRY(encode_pool(&map_k, a.c.k, a.c, rows));
  RAZER_TRY(encode_pool(&map_v, a.c.v, a.c, rows));
  static std::atomic<uint64_t> allowed{0};
  RAZER_TRY(allow_smem((const void*)attn_kv8_kernel<D, NB>, C::SMEM_BYTES, allowed));
  return launch_dependent("attn_kv8_kernel launch", attn_kv8_kernel<D, NB>, sm_count(), C::THREADS, C::SMEM_BYTES, st, map_k, map_v, a);
}

}  // namespace

size_t attn_kv8_workspace_bytes(int D) {
  return WS_ZERO_BYTES + (size_t)sm_count() * 2 * (D == 64 ? AttnCfg<64, 4>::PART_FLOATS : AttnCfg<128, 4>::PART_FLOATS) * sizeof(float);
}

int launch_attn_kv8(const Kv8& c, const Kv8Batch& s, const void* q, long long q_stride, int q_heads, float scale, void* out, float* lse, void* ws,
                    cudaStream_t st) {
  AttnArgs a;
  a.c = c;
  a.s = s;
  a.q = (const __nv_bfloat16*)q;
  a.out = (__nv_bfloat16*)out;
  a.lse = lse;
  a.status = (uint32_t*)ws;
  a.counters = (uint32_t*)((char*)ws + WS_STATUS_BYTES);
  a.parts = (float*)((char*)ws + WS_ZERO_BYTES);
  a.q_stride = q_stride;
  a.scale = scale;
  a.G = q_heads / c.heads;
  const long long rows = ((long long)s.T + s.B - 1) / s.B * a.G;       // of a sequence, in the mean
  const int nb = rows <= 8 ? 1 : rows <= 16 ? 2 : 4;
  if (c.D == 64) return nb == 1 ? launch_as<64, 1>(a, st) : nb == 2 ? launch_as<64, 2>(a, st) : launch_as<64, 4>(a, st);
  return nb == 1 ? launch_as<128, 1>(a, st) : nb == 2 ? launch_as<128, 2>(a, st) : launch_as<128, 4>(a, st);
}

}  // namespace razer
