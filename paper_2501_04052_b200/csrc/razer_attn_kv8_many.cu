// Attention over the paged 8-bit cache for many rows of queries a key-value head (prompts and their chunks): 256 at a time.
//
// Two row tiles of 128 share every tile of 128 tokens.  Four warps turn its codes into f16 (exact: byte ^ 0x80 under an exponent of 2^10 is
// 1152 + code, and a packed subtraction leaves the code; 5 instructions for 4 codes, paid once for 256 rows) in the layout of the MMA's B
// operand, one warp issues
//   S = Q K^T  (128 x 128, FP32 in TMEM)   and   O += P V  (P from TMEM, over S)
// for the two tiles in turn, so that one tile's products run under the other one's softmax.  Two threads have a row, 64 columns
// each, and tell each other the maximum through shared memory (with one thread a row the softmax was a chain of 4100 cycles a tile that nothing
// hid).  O stays in TMEM; it is brought to a new maximum only when that has grown by more than 2^8, so that after a unit's first tiles next to
// never.  Queries are f16 with a power of two of their row's own (largest magnitude in [2^14, 2^15)), probabilities f16 times 2^6
// (11 significant bits, at most 2^14 before the maximum follows, down to 2^-30); value scales enter the probabilities relative to the largest met.
// What bounds it: the exponentials (16 a cycle: 2048 cycles a tile of 256 x 128) and the MMAs (2048) alike, then the softmax's issue.
// Row tiles of a sequence are taken in the order first, last, second, last but one ..., so that equal runs of them are about equal work under the
// causal mask.  Work is cut among the CTAs as razer_attn_kv8.cuh says.
#include "razer_attn_kv8.cuh"

#include <cuda_fp16.h>

namespace razer {

namespace {

constexpr float P_ONE = 64.0f;                           // what a probability of 1 is held as
constexpr float LAG = 8.0f;                              // how far (log2) a maximum may run ahead of the one that sums are relative to

template <int D_>
struct ManyCfg {
  static constexpr int D = D_, R = 256, TK = 128;
  static constexpr int SOFT = 512, THREADS = 704, W_CODES = 16, W_LOAD = 20, W_MMA = 21;   // warps 0-7, 8-15: softmax of a row tile each; 16-19: codes to f16
  static constexpr int HALF_BYTES = TK * D * 2, TILE_BYTES = TK * D;
  static constexpr int O_Q = 0;                                        // [tile][block][128 rows][128 bytes]
  static constexpr int O_K = 2 * HALF_BYTES;                           // two buffers [block][128 tokens][128 bytes]
  static constexpr int O_V = O_K + 2 * HALF_BYTES;
  static constexpr int O_CODES = O_V + 2 * HALF_BYTES;                 // keys, values: [128 tokens][D]
  static constexpr int O_META = O_CODES + 2 * TILE_BYTES;              // [4][8] {key scale, log2 of the value scale}, [4] the largest of the latter
  static constexpr int O_BAR = O_META + 4 * 72;
  static constexpr int N_BAR = 2 + 2 + 2 + 2 + 2 + 2 + 2 + 2 + 2 + 2 + 1;
  static constexpr int O_MISC = O_BAR + 8 * N_BAR;                     // (256 bytes)
  static constexpr int O_TOP = O_MISC + 256;                           // [tile][half][128 rows]: maxima, at the end sums
  static constexpr int SMEM_BYTES = O_TOP + 2048;
  static constexpr int PART_FLOATS = R * (D + 3);                      // [D][R] O, [R] ta, tm, sum
};

__device__ __forceinline__ uint32_t half_pair(uint32_t bytes02) {        // codes in bytes 0 and 2 -> f16 pair
  const uint32_t h = (bytes02 & 0x00FF00FFu) ^ 0x64806480u;
  const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&h), __half2half2(__ushort_as_half(0x6480)));
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void tc_ld32(uint32_t taddr, uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
        "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]),
        "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(taddr)
      : "memory");
  tc_wait_ld();
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
// f16 MMAs, A from shared memory or TMEM
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 ad, bd;\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "mov.b64 ad, {%1, %3};\n\t"
      "mov.b64 bd, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], ad, bd, %4, p;\n\t}" ::"r"(d),
      "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 bd;\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "mov.b64 bd, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], bd, %4, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate)
      : "memory");
}

template <int D>
__global__ void __launch_bounds__(704, 1) attn_kv8_many_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                                                               const __grid_constant__ AttnArgs a) {
  using C = ManyCfg<D>;
  constexpr int TK = C::TK, R = C::R;
  // Swizzled tiles want 1024-byte boundaries.  Dynamic shared memory begins on one where a kernel has no other; a launch where it does not would say so.
  extern __shared__ __align__(1024) uint8_t attn_many_smem[];
  uint8_t* sm = attn_many_smem;
  const uint32_t sb = smem_u32(sm);
  if (sb & 1023) {
    if (threadIdx.x == 0) atomicCAS(a.status, 0u, 12u);
    return;
  }
  // codes of keys / values in and read; f16 buffers ready and free; queries ready; S, P; O of a unit
  const uint32_t bar = sb + C::O_BAR;
  const uint32_t bar_in = bar, bar_read = bar + 16, bar_kready = bar + 32, bar_kfree = bar + 48, bar_vready = bar + 64, bar_vfree = bar + 80, bar_q = bar + 96,
                 bar_s = bar + 112, bar_p = bar + 128, bar_o = bar + 144, bar_drain = bar + 160;
  int* misc = reinterpret_cast<int*>(sm + C::O_MISC);                    // abort, never set, share (4 words), TMEM, last; sums from word 16
  volatile uint32_t* abort_flag = reinterpret_cast<uint32_t*>(misc);
  volatile uint32_t* never = reinterpret_cast<uint32_t*>(misc + 1);
  float2* meta = reinterpret_cast<float2*>(sm + C::O_META);
  float* meta_top = reinterpret_cast<float*>(meta + 32);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_in + 8 * i, 1);
      mbar_init(bar_read + 8 * i, 4);                    // a warp arrives by one lane: 32 arrivals of a warp take their turns
      mbar_init(bar_kready + 8 * i, 4);
      mbar_init(bar_kfree + 8 * i, 1);
      mbar_init(bar_vready + 8 * i, 4);
      mbar_init(bar_vfree + 8 * i, 1);
      mbar_init(bar_q + 8 * i, 8);
      mbar_init(bar_s + 8 * i, 1);
      mbar_init(bar_p + 8 * i, 8);
      mbar_init(bar_o + 8 * i, 1);
    }
    mbar_init(bar_drain, 1);
    misc[0] = misc[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
  }
  if (warp == C::W_MMA) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(misc + 6)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  grid_dep_wait();
  grid_dep_launch();
  long long begin, end, per;
  Walk at;
  const bool work = attn_share<C::THREADS>(a, TK, misc + 2, reinterpret_cast<long long*>(misc + 16), begin, end, per, at);
  tc_fence_after();
  const uint32_t tmem = (uint32_t)misc[6], tmem_o = tmem + 256;        // S and P: 128 columns a row tile; O behind
  auto fail = [&](uint32_t code) {
    *abort_flag = 1;
    atomicCAS(a.status, 0u, code);
  };
  // A segment.  Units of a sequence: head by head, row tiles from both ends.
  struct Seg { int n_items, qt, h, chunk, keys, first, last; };
  auto segment = [&](const Walk& at) {
    Seg g;
    g.n_items = walk_count(at);
    const int qts = (at.n + a.tq - 1) / a.tq, hc = at.unit / qts, k = at.unit - hc * qts;
    g.qt = (k & 1) ? qts - 1 - k / 2 : k / 2;
    g.h = hc / a.chunks;
    g.chunk = hc - g.h * a.chunks;
    g.keys = max(at.len - at.n + min((g.qt + 1) * a.tq, at.n), 0);
    g.first = at.tile;
    g.last = max(min(at.tile + g.n_items, (g.keys + TK - 1) / TK), g.first);
    return g;
  };

  if (!work) {
  } else if (warp == C::W_LOAD) {
    // ===================== pages, scales, codes =====================
    const int boxes = TK >> a.c.page_log2;                       // pages of a tile
    int item = 0, asked_v = 0;                                   // tiles whose keys, values were asked for
    bool alive = true;
    do {
      const Seg g = segment(at);
      int have = -64, id = -1, id_next = -1;                     // first of the 32 blocks that the lanes hold; the lane's page of these and of the next 32
      float ks = 0, lg = 0;
      auto page_of = [&](int block) { return ((long long)block << a.c.page_log2) < g.keys ? kv8_page(a.c, a.s, at.b, block) : -1; };
      for (int t = g.first; t < g.last; ++t, ++item) {
        const int block0 = t * boxes;
        if (block0 + boxes > have + 32) {
          id = block0 == have + 32 ? id_next : page_of(block0 + lane);
          have = block0;
          id_next = page_of(have + 32 + lane);
          float vs = ks = __uint_as_float(0x7FC00000u);
          if (id >= 0) {
            ks = __ldg(a.c.k_scales + (long long)id * a.c.heads + g.h);
            vs = __ldg(a.c.v_scales + (long long)id * a.c.heads + g.h);
          }
          lg = vs >= 0.0f && vs < INFINITY ? log2f(vs) : __uint_as_float(0x7FC00000u);   // -infinity for 0
          if (ks < 0.0f) ks = __uint_as_float(0x7FC00000u);
        }
        const int live = min(boxes, ((g.keys - t * TK - 1) >> a.c.page_log2) + 1);
        const int page = __shfl_sync(0xFFFFFFFFu, id, (block0 - have + lane) & 31);
        // scales by sixteen tokens, as the softmax wants them
        const int from = ((lane & 7) * 16) >> a.c.page_log2;
        float k1 = __shfl_sync(0xFFFFFFFFu, ks, (block0 - have + from) & 31), v1 = __shfl_sync(0xFFFFFFFFu, lg, (block0 - have + from) & 31);
        if (from >= live) k1 = 0.0f, v1 = -INFINITY;             // no token that anyone sees
        float most = v1;
        for (int o = 1; o < 8; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
        if (!(most > -INFINITY)) most = -INFINITY;
        if (item > 0) {                                          // the codes before have been read
          if (!mbar_wait(bar_read, (uint32_t)((item - 1) & 1), abort_flag)) fail(1), alive = false;
          alive = __all_sync(0xFFFFFFFFu, alive);
          if (!alive) break;
        }
        if (lane < 8) meta[(item & 3) * 8 + lane] = make_float2(k1, v1);
        if (lane == 0) meta_top[item & 3] = most;
        __syncwarp();
        auto bring = [&](const CUtensorMap* map, int which) {
          if (lane == 0) mbar_expect_tx(bar_in + 8 * which, (uint32_t)((live << a.c.page_log2) * D));
          __syncwarp();
          if (lane < live)
            tma_load_3d(sb + C::O_CODES + which * C::TILE_BYTES + (uint32_t)((lane << a.c.page_log2) * D), map, 0, 0, max(page, 0) * a.c.heads + g.h, bar_in + 8 * which);
          __syncwarp();
        };
        bring(&map_k, 0);
        if (item > 0) {
          if (!mbar_wait(bar_read + 8, (uint32_t)((item - 1) & 1), abort_flag)) fail(2), alive = false;
          alive = __all_sync(0xFFFFFFFFu, alive);
          if (!alive) { ++item; break; }
        }
        bring(&map_v, 1);
        ++asked_v;
      }
      if (!alive) break;
      if (!walk_advance(a, TK, at, g.n_items)) break;
    } while (true);
    // copies in flight must land before shared memory is released
    if (item > 0) mbar_wait(bar_in, (uint32_t)((item - 1) & 1), never);
    if (asked_v > 0) mbar_wait(bar_in + 8, (uint32_t)((asked_v - 1) & 1), never);
  } else if (warp >= C::W_CODES && warp < C::W_LOAD) {
    // ===================== codes to f16: a thread a token =====================
    const int tok = threadIdx.x - C::SOFT;
    const uint32_t row_in = sb + C::O_CODES + tok * D;
    int item = 0;
    do {
      const Seg g = segment(at);
      for (int t = g.first; t < g.last; ++t, ++item) {
        const int buf = item & 1;
#pragma unroll 1
        for (int which = 0; which < 2; ++which) {
          const uint32_t free_bar = (which ? bar_vfree : bar_kfree) + 8 * buf, ready = (which ? bar_vready : bar_kready) + 8 * buf;
          if (!mbar_wait(bar_in + 8 * which, (uint32_t)(item & 1), abort_flag)) fail(3);
          if (item >= 2 && !mbar_wait(free_bar, (uint32_t)((item >> 1) & 1) ^ 1u, abort_flag)) fail(4);
          const uint32_t to = sb + (which ? C::O_V : C::O_K) + buf * C::HALF_BYTES + tok * 128;
#pragma unroll
          for (int c = 0; c < D / 16; ++c) {
            const uint32_t ch = D == 64 ? c ^ ((tok >> 1) & 3) : c ^ (tok & 7);
            const uint4 w = lds128(row_in + which * C::TILE_BYTES + ch * 16);
            // f16 order inside four: dimensions 0, 2, 1, 3
            const uint32_t at16 = to + (c >> 2) * (TK * 128), c0 = 2 * (c & 3);
            sts128(at16 + ((c0 ^ (tok & 7)) << 4), half_pair(w.x), half_pair(w.x >> 8), half_pair(w.y), half_pair(w.y >> 8));
            sts128(at16 + (((c0 + 1) ^ (tok & 7)) << 4), half_pair(w.z), half_pair(w.z >> 8), half_pair(w.w), half_pair(w.w >> 8));
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(ready);
            mbar_arrive(bar_read + 8 * which);
          }
        }
      }
      if (!walk_advance(a, TK, at, g.n_items)) break;
    } while (!*abort_flag);
  } else if (warp == C::W_MMA) {
    // ===================== MMAs =====================
    if (elect_one()) {
      constexpr uint32_t hi = (1024u >> 4) | (1u << 14) | (2u << 29);                              // rows of 128 bytes in the 128-byte swizzle
      constexpr uint32_t id_s = (1u << 4) | ((uint32_t)(TK >> 3) << 17) | (8u << 24);              // FP32 sums, f16 x f16
      constexpr uint32_t id_o = (1u << 4) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | (8u << 24);  // B (values) dimension-major
      auto lo = [](uint32_t addr, uint32_t lead) { return (addr >> 4) | (lead << 16); };           // lead: from one 64-dimension block to the next
      int item = 0, units = 0;
      bool alive = true;
      auto wait = [&](uint32_t b, int phase, uint32_t code) {
        if (alive && !mbar_wait(b, (uint32_t)(phase & 1), abort_flag)) { fail(code); alive = false; }
        return alive;
      };
      auto products = [&](int i, int t, bool fresh) {              // O_t += P_t V of tile i
        if (!wait(bar_p + 8 * t, i, 5) || (t == 0 && !wait(bar_vready + 8 * (i & 1), i >> 1, 6))) return;
        tc_fence_after();
        const uint32_t v = sb + C::O_V + (i & 1) * C::HALF_BYTES;
#pragma unroll
        for (int k = 0; k < TK / 16; ++k) mma_ts(tmem_o + 128 * t, tmem + 128 * t + 64 * (k / 4) + 8 * (k % 4), lo(v + k * 2048, TK * 128 / 16), hi, id_o, !fresh || k > 0);
      };
      for (;;) {
        const Seg g = segment(at);
        if (g.last > g.first) {
          for (int j = g.first; alive && j < g.last; ++j, ++item) {
            const int buf = item & 1;
            if (!wait(bar_kready + 8 * buf, item >> 1, 7)) break;
            for (int t = 0; t < 2 && alive; ++t) {
              if (j > g.first) products(item - 1, t, j - 1 == g.first);
              else wait(bar_q + 8 * t, units, 8);
              if (!alive) break;
              tc_fence_after();
              const uint32_t k0 = sb + C::O_K + buf * C::HALF_BYTES, q0 = sb + C::O_Q + t * C::HALF_BYTES;
#pragma unroll
              for (int k = 0; k < D / 16; ++k) {
                const uint32_t off = (k >> 2) * (TK * 128) + (k & 3) * 32;
                mma_ss(tmem + 128 * t, lo(q0 + off, 1), lo(k0 + off, 1), hi, id_s, k > 0);
              }
              tc_commit(bar_s + 8 * t);
            }
            if (!alive) break;
            tc_commit(bar_kfree + 8 * buf);
            if (j > g.first) tc_commit(bar_vfree + 8 * (buf ^ 1));
          }
          for (int t = 0; t < 2 && alive; ++t) {
            products(item - 1, t, g.last - 1 == g.first);
            if (alive) tc_commit(bar_o + 8 * t);
          }
          if (alive) tc_commit(bar_vfree + 8 * ((item - 1) & 1));
          ++units;
        }
        if (!alive || !walk_advance(a, TK, at, g.n_items)) break;
      }
      tc_commit(bar_drain);
    }
    __syncwarp();
    mbar_wait(bar_drain, 0, never);
    __syncwarp();
  } else if (warp < C::W_CODES) {
    // ===================== softmax: two threads a row =====================
    const int t = warp >> 3, half = (warp >> 2) & 1, row = 128 * t + 32 * (warp & 3) + lane;   // of the unit
    float* top_mine = reinterpret_cast<float*>(sm + C::O_TOP) + (2 * t + half) * 128 + (row & 127);
    const float* top_other = reinterpret_cast<float*>(sm + C::O_TOP) + (2 * t + (half ^ 1)) * 128 + (row & 127);
    auto row_meet = [&]() { asm volatile("bar.sync %0, 256;" ::"r"(2 + t) : "memory"); };
    const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16, t_s = tmem + lanes + 128 * t, t_o = tmem_o + lanes + 128 * t + half * (D / 2);
    int item = 0, units = 0;
    for (;;) {
      const Seg g = segment(at);
      const int i = g.qt * a.tq + row / a.Gc, hq = g.chunk * a.Gc + row % a.Gc;
      const bool real = row < a.tq * a.Gc && i < at.n && hq < a.G;
      const int see = real ? max(at.len - at.n + i + 1, 0) : 0x7FFFFFFF;
      float m = -INFINITY, l = 0.0f, lg_ref = -INFINITY, f1 = 0.0f, f2 = 0.0f;
      if (g.last > g.first) {
        // ---- the row of queries, half of it a thread
        uint32_t top = 0;
        const uint4* src = reinterpret_cast<const uint4*>(a.q + (long long)(at.row0 + i) * a.q_stride + (long long)(g.h * a.G + hq) * D) + half * (D / 16);
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
          const uint4 x = real ? src[c] : make_uint4(0, 0, 0, 0);
          top = __vmaxu2(__vmaxu2(top, __vmaxu2(x.x & 0x7FFF7FFFu, x.y & 0x7FFF7FFFu)), __vmaxu2(x.z & 0x7FFF7FFFu, x.w & 0x7FFF7FFFu));
        }
        top = max(top >> 16, top & 0xFFFFu) << 16;
        *top_mine = __uint_as_float(top);
        row_meet();
        top = max(top, __float_as_uint(*top_other));
        row_meet();                                                                    // both have read
        const bool bad = top >= 0x7F800000u || kv8_over(a.c, a.s, __ldg(a.s.kv_len + at.b));
        const int e = top > 0 && !bad ? ilogbf(__uint_as_float(top)) : 0;
        // to [2^14, 2^15), turned round where the scale is negative, so that the largest score stays the largest
        const float up0 = (a.scale < 0.0f ? -1.0f : 1.0f) * power2((14 - e) / 2), up1 = power2(14 - e - (14 - e) / 2);
        f1 = bad ? __uint_as_float(0x7FC00000u) : fabsf(a.scale) * LOG2E * power2(e / 2);
        f2 = power2(e - e / 2 - 14);
        const uint32_t to = sb + C::O_Q + t * C::HALF_BYTES + (row & 127) * 128;
#pragma unroll
        for (int c0 = 0; c0 < D / 16; ++c0) {
          const int c = half * (D / 16) + c0;
          const uint4 x = real && !bad ? src[c0] : make_uint4(0, 0, 0, 0);             // (again, from L1)
          uint32_t w[4];
#pragma unroll
          for (int k = 0; k < 2; ++k) {                                               // four dimensions, in the order 0, 2, 1, 3
            const uint32_t p0 = k ? x.z : x.x, p1 = k ? x.w : x.y;
            w[2 * k] = pack_half(__uint_as_float(p0 << 16) * up0 * up1, __uint_as_float(p1 << 16) * up0 * up1);
            w[2 * k + 1] = pack_half(__uint_as_float(p0 & 0xFFFF0000u) * up0 * up1, __uint_as_float(p1 & 0xFFFF0000u) * up0 * up1);
          }
          sts128(to + (c >> 3) * (TK * 128) + (((c & 7) ^ (row & 7)) << 4), w[0], w[1], w[2], w[3]);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_q + 8 * t);
        for (int j = g.first; j < g.last; ++j, ++item) {
          const int tok0 = j * TK;
          const bool edge = __any_sync(0xFFFFFFFFu, tok0 + TK > see);
          if (!mbar_wait(bar_kready + 8 * (item & 1), (uint32_t)((item >> 1) & 1), abort_flag)) fail(9);   // the scales are in place
          const float lg_top = meta_top[item & 3];
          float c[4], lg[4];                                                           // of the half's four times sixteen columns
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float2 sc = meta[(item & 3) * 8 + 4 * half + q];
            c[q] = sc.x * f1;
            lg[q] = sc.y;
          }
          const int first = tok0 + 64 * half;
          if (!mbar_wait(bar_s + 8 * t, (uint32_t)(item & 1), abort_flag)) fail(10);
          __syncwarp();
          tc_fence_after();
          // ---- the tile's maximum: of sixteen scores before their page's scale, which is not negative
          float most = -INFINITY;
          bool usual = true;                                                           // factors of the scores that one FP32 number holds
#pragma unroll
          for (int q = 0; q < 4; q += 2) {
            uint32_t v[32];
            tc_ld32(t_s + 64 * half + 16 * q, v);
            if (edge) {
#pragma unroll
              for (int x = 0; x < 32; ++x) v[x] = first + 16 * q + x < see ? v[x] : 0xFF800000u;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
              for (int x = 0; x < 16; ++x) top[x & 1] = fmaxf(top[x & 1], __uint_as_float(v[16 * h + x]));
              const float cf = c[q + h] * f2, topmost = fmaxf(top[0], top[1]);
              usual = usual && (cf == 0.0f ? c[q + h] == 0.0f : fabsf(cf) > 1e-30f);
              if (topmost > -INFINITY) most = fmaxf(most, topmost * c[q + h]);
            }
          }
          most = most == -INFINITY ? most : most * f2;
          *top_mine = most;
          row_meet();                                  // (the next write comes behind the next S, which comes behind both halves' arrivals below)
          most = fmaxf(most, *top_other);
          float fm = 1.0f;
          bool move = false;
          if (most > m + LAG) {                                                        // (or the first)
            fm = ex2(m - most);
            l *= fm;
            m = most;
            move = true;
          }
          if (lg_top > lg_ref) {
            fm *= ex2(lg_ref - lg_top);
            lg_ref = lg_top;
            move = true;
          }
          if (j > g.first && __any_sync(0xFFFFFFFFu, move)) {                         // (the last product with the values is over: S came behind it)
#pragma unroll 1
            for (int q = 0; q < D / 64; ++q) {
              uint32_t v[32];
              tc_ld32(t_o + 32 * q, v);
#pragma unroll
              for (int x = 0; x < 32; ++x) v[x] = __float_as_uint(__uint_as_float(v[x]) * fm);
              tc_st32(t_o + 32 * q, v);
            }
          }
          // ---- probabilities, each half's over its own scores: exp2(s cf - m), times the value scale of the page over the largest
          const float m0 = m == -INFINITY ? 0.0f : m, lg0 = lg_ref == -INFINITY ? 0.0f : lg_ref;
          if (!edge && __all_sync(0xFFFFFFFFu, usual)) {
            uint64_t sum = 0;                                                          // of even and odd columns
            const uint64_t minus_m = pair64(-m0, -m0);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              uint32_t v[16], p[8];
              tc_ld16(t_s + 64 * half + 16 * q, v);
              tc_wait_ld();
              const float cf = c[q] * f2, rel = ex2(lg[q] - lg0) * P_ONE;
              const uint64_t cf2 = pair64(cf, cf), rel2 = pair64(rel, rel);
#pragma unroll
              for (int x = 0; x < 8; ++x) {
                const uint64_t z = fma2(pair64(__uint_as_float(v[2 * x]), __uint_as_float(v[2 * x + 1])), cf2, minus_m);
                const uint64_t e = pair64(ex2(low64(z)), ex2(high64(z)));
                sum = add2(sum, e);
                const uint64_t w = mul2(e, rel2);
                p[x] = pack_half(low64(w), high64(w));
              }
              tc_st8(t_s + 64 * half + 8 * q, p);
            }
            l += low64(sum) + high64(sum);
          } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              uint32_t v[16], p[8];
              tc_ld16(t_s + 64 * half + 16 * q, v);
              tc_wait_ld();
              const float rel = ex2(lg[q] - lg0) * P_ONE;
#pragma unroll
              for (int x = 0; x < 16; x += 2) {
                float e[2], w[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  const bool seen = first + 16 * q + x + k < see;                      // a scale that is NaN is not the hidden rows' affair
                  e[k] = seen ? ex2(__fmaf_rn(__uint_as_float(v[x + k]) * c[q], f2, -m0)) : 0.0f;
                  w[k] = seen ? e[k] * rel : 0.0f;
                }
                l += e[0] + e[1];
                p[x / 2] = pack_half(w[0], w[1]);
              }
              tc_st8(t_s + 64 * half + 8 * q, p);
            }
          }
          tc_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_p + 8 * t);
        }
        if (!mbar_wait(bar_o + 8 * t, (uint32_t)(units & 1), abort_flag)) fail(11);
        __syncwarp();
        tc_fence_after();
        ++units;
        *top_mine = l;
        row_meet();
        l += *top_other;
      }
      // ---- the end of the unit.  lg_ref may be -infinity: nothing but values of scale 0 was met, and O is 0
      const bool whole = g.first == 0 && g.n_items == at.tiles, any = g.last > g.first;
      const float ta = lg_ref == -INFINITY ? -INFINITY : m + lg_ref;
      const long long out_row = (long long)(at.row0 + i) * a.c.heads * a.G + g.h * a.G + hq;
      float* part = a.parts + ((long long)blockIdx.x * 2 + (g.first > 0 ? 0 : 1)) * C::PART_FLOATS;
#pragma unroll 1
      for (int q = 0; q < D / 64; ++q) {
        const int d0 = half * (D / 2) + 32 * q;
        uint32_t v[32];
        if (any) tc_ld32(t_o + 32 * q, v);
#pragma unroll
        for (int x = 0; x < 32; ++x) v[x] = any ? __float_as_uint(__uint_as_float(v[x]) * (1.0f / P_ONE)) : 0u;
        if (whole) {
          if (real) {
#pragma unroll
            for (int x = 0; x < 32; x += 4)                                            // columns 0, 2, 1, 3 of four
              attn_store<D>(a, out_row, d0 + x, make_float4(__uint_as_float(v[x]), __uint_as_float(v[x + 2]), __uint_as_float(v[x + 1]), __uint_as_float(v[x + 3])), l, ta, m);
          }
        } else {
#pragma unroll
          for (int x = 0; x < 32; ++x) __stcg(part + (d0 + x) * R + row, __uint_as_float(v[x]));
        }
      }
      tc_fence_before();
      if (!whole) {
        if (half == 0) {
          __stcg(part + D * R + row, ta);
          __stcg(part + D * R + R + row, m);
          __stcg(part + D * R + 2 * R + row, l);
        }
        // the last of the unit's CTAs to get here adds the parts up, half a row a thread
        const long long unit_begin = begin + (end - begin - at.left) - g.first;
        const int c_first = (int)(unit_begin / per), parts = (int)((unit_begin + at.tiles - 1) / per) - c_first + 1;
        threads_meet<C::SOFT>();
        if (threadIdx.x == 0) {
          uint32_t seen;
          asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(seen) : "l"(a.counters + c_first) : "memory");
          misc[7] = seen == (uint32_t)(parts - 1);
          if (misc[7]) a.counters[c_first] = 0;
        }
        threads_meet<C::SOFT>();
        if (misc[7]) {
          auto at_part = [&](int c) { return a.parts + ((long long)(c_first + c) * 2 + (c == 0)) * C::PART_FLOATS + row; };
          float top_a = -INFINITY, top_m = -INFINITY, sum_l = 0.0f;
          for (int c = 0; c < parts; ++c) {
            const float *p = at_part(c) + D * R, ac = __ldcg(p), mc = __ldcg(p + R), lc = __ldcg(p + 2 * R), nm = fmaxf(top_m, mc);
            top_a = fmaxf(top_a, ac);
            sum_l = rebase(top_m, sum_l, nm) * sum_l + rebase(mc, lc, nm) * lc;
            top_m = nm;
          }
#pragma unroll 1
          for (int d = half * (D / 2); d < (half + 1) * (D / 2); d += 8) {
            float sum[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) sum[x] = 0.0f;
#pragma unroll 2
            for (int c = 0; c < parts; ++c) {
              const float* p = at_part(c);
              const float ac = __ldcg(p + D * R), f = ac == -INFINITY ? 0.0f : ex2(ac - top_a);
#pragma unroll
              for (int x = 0; x < 8; ++x) sum[x] += f * __ldcg(p + (d + x) * R);
            }
            if (real) {
              attn_store<D>(a, out_row, d, make_float4(sum[0], sum[2], sum[1], sum[3]), sum_l, top_a, top_m);
              attn_store<D>(a, out_row, d + 4, make_float4(sum[4], sum[6], sum[5], sum[7]), sum_l, top_a, top_m);
            }
          }
        }
        threads_meet<C::SOFT>();                                                           // misc[7] has been read
      }
      if (!walk_advance(a, TK, at, g.n_items)) break;
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == C::W_MMA) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

template <int D>
int launch_as(AttnArgs& a, cudaStream_t st) {
  using C = ManyCfg<D>;
  static_assert(C::SMEM_BYTES <= 232448, "shared memory of a CTA");
  a.Gc = a.G < C::R ? a.G : C::R;
  a.chunks = (a.G + a.Gc - 1) / a.Gc;
  a.tq = C::R / a.Gc;
  CUtensorMap map_k, map_v;
  RAZER_TRY(attn_encode_pool(&map_k, a.c.k, a.c, a.c.page));
  RAZER_TRY(attn_encode_pool(&map_v, a.c.v, a.c, a.c.page));
  static std::atomic<uint64_t> allowed{0};
  RAZER_TRY(allow_smem((const void*)attn_kv8_many_kernel<D>, C::SMEM_BYTES, allowed));
  return launch_dependent("attn_kv8_many_kernel launch", attn_kv8_many_kernel<D>, sm_count() < ATTN_CTAS ? sm_count() : ATTN_CTAS, C::THREADS, C::SMEM_BYTES, st, map_k,
                          map_v, a);
}

}  // namespace

size_t attn_many_part_floats(int D) { return D == 64 ? ManyCfg<64>::PART_FLOATS : ManyCfg<128>::PART_FLOATS; }

int launch_attn_many(AttnArgs& a, cudaStream_t st) { return a.c.D == 64 ? launch_as<64>(a, st) : launch_as<128>(a, st); }

}  // namespace razer
