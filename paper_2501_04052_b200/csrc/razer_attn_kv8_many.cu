// Attention over the paged 8-bit cache for many rows of queries a key-value head (prompts and their chunks): 256 at a time.
//
// Two row tiles of 128 share every tile of 128 tokens.  Four warps turn its codes into f16 (exact: byte ^ 0x80 under an exponent of 2^10 is
// 1152 + code, and a packed subtraction leaves the code; 5 instructions for 4 codes, paid once for 256 rows) in the layout of the MMA's B
// operand, one warp issues
//   S = Q K^T  (128 x 64, FP32 in TMEM)   and   O += P V  (P from TMEM, over S)
// in steps of 64 tokens.  S has two buffers a row tile, so that the next scores are there when a softmax is done with the last (with one buffer of 128
// columns a row tile's softmax and products took turns: 6000 cycles a tile).  A thread has a row: maximum and sum take no shuffle, the step's
// scores are read once.  O stays in TMEM; it is brought to a new maximum only when that has grown by more than 2^8, so that after a unit's
// first tiles next to never.  Queries are f16 with a power of two of their row's own (largest magnitude in [2^14, 2^15)), probabilities f16
// times 2^6 (11 significant bits, at most 2^14 before the maximum follows, down to 2^-30); value scales enter the probabilities relative to
// twice the largest that the row has met.  (Of the pages that it sees: one for all rows of a tile would leave a row whose own pages have values 2^33 times
// smaller than those behind its mask without any weight.)  Probabilities in f16 are what the MMA takes beside f16 codes; their roundings are independent and an eighth of that
// of a bf16 output: against 64 bits the chunk below is off by 0.00167 of its norm, by FP32 probabilities by 0.00166, the two apart by 0.00087 where one of them rounds the other
// way.  The sums of the exponentials are FP32 of what was not rounded.
// A pair of CTAs (cta_group::2) takes 512 rows: each converts half of the keys of a step and half of the values' dimensions, so that a tile is
// converted once for both, and the MMAs read half as much of it from either's shared memory.
// What bounds it: 3 ragged sequences of up to 8192 tokens, up to 1000 of them new, 8 x 4 heads of 128, 355 us (746 TFLOP/s) by pairs, 373 without: 2300 to 2500 cycles
// for 256 rows x 64 tokens.  Without the softmax a single CTA takes 2200 (the MMAs of S, half as wide as they are long, 860, those of O 300, and shared memory that these share
// with the conversion, 48 KB), a pair 1600.  The exponentials alone are 1024 (16 a cycle); By pairs XU 43 %, ALU 37 %, tensor 39 % busy, issue slots 49 %: what is left is
// the chain of a step (scores read, maximum, exponentials, probabilities stored, 1900 cycles), of which a scheduler has two to interleave.
// A unit's ends (queries in, sums out, parts joined) are a tenth of the time.
// Row tiles of a sequence are taken in the order first, last, second, last but one ..., so that equal runs of them are about equal work under the
// causal mask.  Work is cut among the CTAs as razer_attn_kv8.cuh says.
#include "razer_attn_kv8.cuh"

#include <cuda_fp16.h>

namespace razer {

namespace {

constexpr float P_ONE = 64.0f;                           // what a probability of 1 is held as
constexpr float LAG = 8.0f;                              // how far (log2) a maximum may run ahead of the one that sums are relative to

// CTAS: one, or a pair that goes through the tiles together, 256 rows each.
template <int D_, int CTAS_>
struct ManyCfg {
  static_assert(CTAS_ == 1 || D_ == 128, "a pair's CTA holds 64 of 128 dimensions of the values");
  static constexpr int D = D_, CTAS = CTAS_, R = 256, TK = 128;
  static constexpr int SOFT = 256, THREADS = 448, W_CODES = 8, W_LOAD = 12, W_MMA = 13;   // warps 0-3, 4-7: softmax of a row tile each; 8-11: codes to f16
  static constexpr int STEP = 64;                                      // tokens of a step
  static constexpr int HALF_BYTES = TK * D * 2;                        // queries of a row tile
  static constexpr int K_ROWS = TK / CTAS, V_DIMS = D / CTAS;          // a CTA's part of a tile: 64 / CTAS keys of each step, and V_DIMS of the values' dimensions
  static constexpr int PART_BYTES = HALF_BYTES / CTAS, TILE_BYTES = TK * D / CTAS;
  static constexpr int KBUF = CTAS;                                    // f16 keys: a pair has the room for two, and its barriers take longer (2400 cycles a step with one)
  static constexpr int O_Q = 0;                                        // [tile][block][128 rows][128 bytes]
  static constexpr int O_K = 2 * HALF_BYTES;                           // [block][128 tokens][128 bytes]
  static constexpr int O_V = O_K + KBUF * PART_BYTES;                         // two buffers: the next tile's are made while products still read the last one's
  static constexpr int STAGES = 2 * CTAS;                                     // of codes: with one, a copy's latency was in every tile (194 us of 458 were that skeleton)
  static constexpr int O_CODES = O_V + 2 * PART_BYTES;                     // keys, values of each stage: [K_ROWS][D], [128 tokens][V_DIMS]
  static constexpr int METAS = 8;                                      // tiles whose scales are held: up to four on their way, three in work
  static constexpr int O_META = O_CODES + 2 * STAGES * TILE_BYTES;     // [METAS][8] {key scale, log2 of the value scale}, [METAS][2] the largest of the latter in a step
  static constexpr int O_BAR = O_META + METAS * 72;
  static constexpr int N_BAR = 4 * STAGES + 8 + 2 + 4 + 4 + 4 + 1;
  static constexpr int O_MISC = O_BAR + 8 * N_BAR;
  static constexpr int SMEM_BYTES = 1024 + O_MISC + 256;
  static constexpr int PART_FLOATS = R * (D + 3);                      // [D][R] O, [R] ta, tm, sum
};

// A Walk and its run's bounds.
struct Held {
  int b, row0, n, len, tiles, units, unit, tile;
  bool over;
  long long left, begin, end, per;
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
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// Two warps that go through a part of their code in turn.
__device__ __forceinline__ void take_turn(int barrier) { asm volatile("bar.sync %0, 64;" ::"r"(barrier) : "memory"); }
__device__ __forceinline__ void give_turn(int barrier) { asm volatile("bar.arrive %0, 64;" ::"r"(barrier) : "memory"); }
// f16 MMAs, A from shared memory or TMEM; of one CTA or by the first of a pair for both.
template <bool PAIR>
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate) {
#define RAZER_MMA_SS(GROUP)                                   \
  asm volatile(                                               \
      "{\n\t.reg .pred p;\n\t.reg .b64 ad, bd;\n\t"           \
      "setp.ne.b32 p, %5, 0;\n\t"                             \
      "mov.b64 ad, {%1, %3};\n\t"                             \
      "mov.b64 bd, {%2, %3};\n\t"                             \
      "tcgen05.mma.cta_group::" GROUP ".kind::f16 [%0], ad, bd, %4, p;\n\t}" ::"r"(d), \
      "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate) \
      : "memory")
  if (PAIR) RAZER_MMA_SS("2");
  else RAZER_MMA_SS("1");
#undef RAZER_MMA_SS
}
template <bool PAIR>
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate) {
#define RAZER_MMA_TS(GROUP)                                   \
  asm volatile(                                               \
      "{\n\t.reg .pred p;\n\t.reg .b64 bd;\n\t"               \
      "setp.ne.b32 p, %5, 0;\n\t"                             \
      "mov.b64 bd, {%2, %3};\n\t"                             \
      "tcgen05.mma.cta_group::" GROUP ".kind::f16 [%0], [%1], bd, %4, p;\n\t}" ::"r"(d), \
      "r"(a), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate)  \
      : "memory")
  if (PAIR) RAZER_MMA_TS("2");
  else RAZER_MMA_TS("1");
#undef RAZER_MMA_TS
}

template <int D, int CTAS>
__global__ void __launch_bounds__(448, 1) attn_kv8_many_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                                                               const __grid_constant__ AttnArgs a) {
  using C = ManyCfg<D, CTAS>;
  constexpr int TK = C::TK, R = C::R;
  constexpr bool PAIR = CTAS == 2;
  const int rank = PAIR ? (int)cluster_rank() : 0, share = blockIdx.x / CTAS, shares = gridDim.x / CTAS;
  extern __shared__ uint8_t attn_smem[];
  uint8_t* sm = attn_smem + ((1024 - (smem_u32(attn_smem) & 1023)) & 1023);
  const uint32_t sb = smem_u32(sm);
  // codes of keys / values in and read; f16 buffers ready and free; queries ready; S, P; products with the values done
  const uint32_t bar = sb + C::O_BAR;
  const uint32_t bar_in = bar, bar_read = bar_in + 16 * C::STAGES, bar_kready = bar_read + 16 * C::STAGES, bar_kfree = bar_kready + 16, bar_vready = bar_kfree + 16,
                 bar_vfree = bar_vready + 16, bar_q = bar_vfree + 16, bar_s = bar_q + 16, bar_p = bar_s + 32, bar_o = bar_p + 32, bar_drain = bar_o + 32;   // in, read: [keys, values][stage]; s, p, o: [row tile][buffer]
  int* misc = reinterpret_cast<int*>(sm + C::O_MISC);                    // abort, never set, share (4 words), TMEM, last; sums from word 16
  volatile uint32_t* abort_flag = reinterpret_cast<uint32_t*>(misc);
  volatile uint32_t* never = reinterpret_cast<uint32_t*>(misc + 1);
  float2* meta = reinterpret_cast<float2*>(sm + C::O_META);
  float* meta_top = reinterpret_cast<float*>(meta + 8 * C::METAS);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2 * C::STAGES; ++i) {
      mbar_init(bar_in + 8 * i, 1);
      mbar_init(bar_read + 8 * i, 4);              // a warp arrives by one lane: 32 arrivals of a warp take their turns
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_kready + 8 * i, PAIR && rank == 0 ? 5 : 4);      // the other CTA's four by one
      mbar_init(bar_kfree + 8 * i, 1);
      mbar_init(bar_vready + 8 * i, PAIR && rank == 0 ? 5 : 4);
      mbar_init(bar_vfree + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_q + 8 * i, 4 * CTAS);
      mbar_init(bar_s + 16 * i, 1);
      mbar_init(bar_s + 16 * i + 8, 1);
      mbar_init(bar_p + 16 * i, 4 * CTAS);
      mbar_init(bar_p + 16 * i + 8, 4 * CTAS);
      mbar_init(bar_o + 16 * i, 1);
      mbar_init(bar_o + 16 * i + 8, 1);
    }
    mbar_init(bar_drain, 1);
    misc[0] = misc[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
  }
  if (warp == C::W_MMA) {
    if (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(misc + 6)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(misc + 6)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  grid_dep_wait();
  grid_dep_launch();
  long long begin, end, per;
  Walk at;
  const bool work = attn_share<C::THREADS>(a, TK, misc + 2, reinterpret_cast<long long*>(misc + 16), begin, end, per, at, share, shares);
  if (PAIR) {                                                          // both CTAs' barriers are ready
    __syncwarp();
    cluster_meet();
  }
  tc_fence_after();
  // A barrier that the MMAs wait for is that of the first CTA.
  auto tell = [&](uint32_t b) {
    if (PAIR) peer_arrive(peer_addr(b, 0));
    else mbar_arrive(b);
  };
  const uint32_t tmem = (uint32_t)misc[6], tmem_o = tmem + 256;        // S and P: two buffers of 64 columns a row tile; O behind
  auto fail = [&](uint32_t code) {
    *abort_flag = 1;
    atomicCAS(a.status, 0u, code);
  };
  // A segment.  Units of a sequence: head by head, row tiles from both ends.
  struct Seg { int n_items, qt, h, chunk, keys, first, last, steps; };
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
    g.steps = g.last > g.first ? min(2 * (g.last - g.first), (g.keys - g.first * TK + C::STEP - 1) / C::STEP) : 0;
    return g;
  };

  if (!work) {
  } else if (warp == C::W_LOAD) {
    // ===================== pages, scales, codes =====================
    const int boxes = TK >> a.c.page_log2;                       // pages of a tile
    const int k_rows = PAIR ? min(a.c.page, 32) : a.c.page, k_boxes = C::K_ROWS / k_rows;        // of the keys: a pair's CTA takes 32 of 64 tokens
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
            ks = a.c.k_scales[(long long)id * a.c.heads + g.h];
            vs = a.c.v_scales[(long long)id * a.c.heads + g.h];
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
        float most = fmaxf(v1, -INFINITY);                       // (NaN counts as none)
        for (int o = 1; o < 4; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
        const int stage = item % C::STAGES, round = item / C::STAGES;
        if (round > 0) {                                         // the codes before have been read
          if (!mbar_wait(bar_read + 8 * stage, (uint32_t)(round & 1) ^ 1u, abort_flag)) fail(1), alive = false;
          alive = __all_sync(0xFFFFFFFFu, alive);
          if (!alive) break;
        }
        if (lane < 8) meta[item % C::METAS * 8 + lane] = make_float2(k1, v1);
        if (lane == 0 || lane == 4) meta_top[item % C::METAS * 2 + (lane >> 2)] = most;
        __syncwarp();
        {
          const uint32_t in = bar_in + 8 * stage;
          // box `lane` of the keys: its first token, of the tile
          const int tok = PAIR ? (lane * k_rows >> 5) * 64 + rank * 32 + ((lane * k_rows) & 31) : lane * k_rows;
          const int of = tok >> a.c.page_log2, k_page = __shfl_sync(0xFFFFFFFFu, id, (block0 - have + of) & 31);
          const bool mine = lane < k_boxes && of < live;
          const int n = __popc(__ballot_sync(0xFFFFFFFFu, mine));
          if (lane == 0) mbar_expect_tx(in, (uint32_t)(n * k_rows * D));
          __syncwarp();
          if (mine)
            tma_load_3d(sb + C::O_CODES + 2 * stage * C::TILE_BYTES + (uint32_t)(lane * k_rows * D), &map_k, 0, tok & (a.c.page - 1), max(k_page, 0) * a.c.heads + g.h, in);
          __syncwarp();
        }
        if (round > 0) {
          if (!mbar_wait(bar_read + 8 * (C::STAGES + stage), (uint32_t)(round & 1) ^ 1u, abort_flag)) fail(2), alive = false;
          alive = __all_sync(0xFFFFFFFFu, alive);
          if (!alive) { ++item; break; }
        }
        {
          const uint32_t in = bar_in + 8 * (C::STAGES + stage);
          if (lane == 0) mbar_expect_tx(in, (uint32_t)((live << a.c.page_log2) * C::V_DIMS));
          __syncwarp();
          if (lane < live)
            tma_load_3d(sb + C::O_CODES + (2 * stage + 1) * C::TILE_BYTES + (uint32_t)((lane << a.c.page_log2) * C::V_DIMS), &map_v, rank * C::V_DIMS, 0,
                        max(page, 0) * a.c.heads + g.h, in);
          __syncwarp();
        }
        ++asked_v;
      }
      if (!alive) break;
      if (!walk_advance(a, TK, at, g.n_items)) break;
    } while (true);
    // copies in flight must land before shared memory is released
    for (int f = max(item - C::STAGES, 0); f < item; ++f) mbar_wait(bar_in + 8 * (f % C::STAGES), (uint32_t)((f / C::STAGES) & 1), never);
    for (int f = max(asked_v - C::STAGES, 0); f < asked_v; ++f) mbar_wait(bar_in + 8 * (C::STAGES + f % C::STAGES), (uint32_t)((f / C::STAGES) & 1), never);
  } else if (warp >= C::W_CODES && warp < C::W_LOAD) {
    // ===================== codes to f16: a thread a token =====================
    const int tok = threadIdx.x - C::SOFT;
    int item = 0;
    do {
      const Seg g = segment(at);
      for (int t = g.first; t < g.last; ++t, ++item) {
        const int stage = item % C::STAGES;
#pragma unroll 1
        for (int which = 0; which < 2; ++which) {
          const int buf = which ? item & 1 : item % C::KBUF;
          const uint32_t ready = (which ? bar_vready : bar_kready) + 8 * buf;
          if (!mbar_wait(bar_in + 8 * (which * C::STAGES + stage), (uint32_t)((item / C::STAGES) & 1), abort_flag)) fail(3);
          if (which == 0 && item >= C::KBUF && !mbar_wait(bar_kfree + 8 * buf, (uint32_t)((item / C::KBUF) & 1) ^ 1u, abort_flag)) fail(4);
          if (which == 1 && item > 1 && !mbar_wait(bar_vfree + 8 * buf, (uint32_t)((item >> 1) & 1) ^ 1u, abort_flag)) fail(4);
          // a thread's part: a token's row, or, of a pair's half as many keys, half of it
          const bool split = PAIR && which == 0;
          const int r = split ? tok & (C::K_ROWS - 1) : tok, c0 = split ? (tok / C::K_ROWS) * (D / 32) : 0, columns = which ? C::V_DIMS : D;
          const uint32_t to = sb + (which ? C::O_V : C::O_K) + buf * C::PART_BYTES + r * 128, row_in = sb + C::O_CODES + (2 * stage + which) * C::TILE_BYTES + r * columns;
          const uint32_t block = which ? TK * 128 : C::K_ROWS * 128;
#pragma unroll
          for (int i = 0; i < C::V_DIMS / 16; ++i) {
            const int c = c0 + i;
            const uint32_t ch = columns == 64 ? c ^ ((r >> 1) & 3) : c ^ (r & 7);
            const uint4 w = lds128(row_in + ch * 16);
            // f16 order inside four: dimensions 0, 2, 1, 3
            const uint32_t at16 = to + (c >> 2) * block, h0 = 2 * (c & 3);
            sts128(at16 + ((h0 ^ (r & 7)) << 4), half_pair(w.x), half_pair(w.x >> 8), half_pair(w.y), half_pair(w.y >> 8));
            sts128(at16 + (((h0 + 1) ^ (r & 7)) << 4), half_pair(w.z), half_pair(w.z >> 8), half_pair(w.w), half_pair(w.w >> 8));
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(ready);
            mbar_arrive(bar_read + 8 * (which * C::STAGES + stage));
          }
        }
      }
      if (!walk_advance(a, TK, at, g.n_items)) break;
    } while (!*abort_flag);
  } else if (warp == C::W_MMA && rank == 0) {
    // ===================== MMAs =====================
    if (elect_one()) {
      constexpr uint32_t hi = (1024u >> 4) | (1u << 14) | (2u << 29);                              // rows of 128 bytes in the 128-byte swizzle
      constexpr uint32_t id_s = (1u << 4) | ((uint32_t)(C::STEP >> 3) << 17) | ((8u * CTAS) << 24);         // FP32 sums, f16 x f16
      constexpr uint32_t id_o = (1u << 4) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((8u * CTAS) << 24);  // B (values) dimension-major
      auto lo = [](uint32_t addr, uint32_t lead) { return (addr >> 4) | (lead << 16); };           // lead: from one 64-dimension block to the next
      auto commit = [&](uint32_t b) {                              // to this barrier of both CTAs
        if (PAIR) commit_pair(b, 3u);
        else tc_commit(b);
      };
      int tiles = 0, done = 0, units = 0;                          // tiles whose keys, values were waited for; steps of the units before
      bool alive = true;
      auto wait = [&](uint32_t b, int phase, uint32_t code) {
        if (alive && !mbar_wait<PAIR>(b, (uint32_t)(phase & 1), abort_flag)) { fail(code); alive = false; }
        return alive;
      };
      for (;;) {
        const Seg g = segment(at);
        if (g.steps > 0) {
          int k_tiles = tiles;
          // scores of step n of the unit, both row tiles or one
          auto scores = [&](int n, int t) {
            const int b = (done + n) & 1;
            const int buf = (tiles + (n >> 1)) % C::KBUF;
            const uint32_t k0 = sb + C::O_K + buf * C::PART_BYTES + (n & 1) * (C::STEP / CTAS * 128), q0 = sb + C::O_Q + t * C::HALF_BYTES, d = tmem + 128 * t + 64 * b;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
              mma_ss<PAIR>(d, lo(q0 + (k >> 2) * (TK * 128) + (k & 3) * 32, 1), lo(k0 + (k >> 2) * (C::K_ROWS * 128) + (k & 3) * 32, 1), hi, id_s, k > 0);
            }
            commit(bar_s + 16 * t + 8 * b);
            if (t == 1 && ((n & 1) || n == g.steps - 1)) commit(bar_kfree + 8 * buf);
          };
          auto keys = [&](int n) {
            if (n & 1) return true;
            const int tile = k_tiles++;
            return wait(bar_kready + 8 * (tile % C::KBUF), tile / C::KBUF, 7);
          };
          for (int n = 0; n < 2 && n < g.steps && alive; ++n) {
            if (!keys(n)) break;
            for (int t = 0; t < 2 && alive; ++t) {
              if (n == 0) wait(bar_q + 8 * t, units, 8);
              tc_fence_after();
              if (alive) scores(n, t);
            }
          }
          for (int n = 0; n < g.steps && alive; ++n) {
            const int b = (done + n) & 1;
            const int tile = tiles + (n >> 1);
            if (!(n & 1) && !wait(bar_vready + 8 * (tile & 1), tile >> 1, 6)) break;
            for (int t = 0; t < 2 && alive; ++t) {
              if (!wait(bar_p + 16 * t + 8 * b, (done + n) >> 1, 5)) break;
              tc_fence_after();
              const uint32_t v = sb + C::O_V + (tile & 1) * C::PART_BYTES + (n & 1) * (C::STEP * 128), pa = tmem + 128 * t + 64 * b;
#pragma unroll
              for (int k = 0; k < C::STEP / 16; ++k) mma_ts<PAIR>(tmem_o + 128 * t, pa + 8 * k, lo(v + k * 2048, TK * 128 / 16), hi, id_o, n > 0 || k > 0);
              commit(bar_o + 16 * t + 8 * b);
              if (n + 2 < g.steps && (t > 0 || keys(n + 2))) {
                tc_fence_after();
                scores(n + 2, t);
              }
            }
            if (alive && ((n & 1) || n == g.steps - 1)) commit(bar_vfree + 8 * (tile & 1));
          }
          tiles += g.last - g.first;
          done += g.steps;
          ++units;
        }
        if (!alive || !walk_advance(a, TK, at, g.n_items)) break;
      }
      if (PAIR) commit_pair(bar_drain, 1u);
      else tc_commit(bar_drain);
    }
    __syncwarp();
    mbar_wait(bar_drain, 0, never);
    __syncwarp();
  } else if (warp == C::W_MMA) {
    // ===================== the second CTA's f16 keys and values, told to the first =====================
    // (By this warp, not by the four that make them: a release of the cluster takes 900 cycles, and two of them a tile were 1700 cycles a step.)
    if (elect_one()) {
      int item = 0;
      bool alive = true;
      do {
        const Seg g = segment(at);
        for (int t = g.first; alive && t < g.last; ++t, ++item)
          for (int which = 0; alive && which < 2; ++which) {
            const uint32_t ready = (which ? bar_vready : bar_kready) + 8 * (item & 1);
            alive = mbar_wait(ready, (uint32_t)((item >> 1) & 1), abort_flag);
            if (alive) peer_arrive(peer_addr(ready, 0));
            else fail(9);
          }
        if (!walk_advance(a, TK, at, g.n_items)) break;
      } while (alive);
    }
    __syncwarp();
  } else if (warp < C::W_CODES) {
    // ===================== softmax: a thread a row =====================
    const int t = warp >> 2, row = 128 * t + 32 * (warp & 3) + lane, urow = rank * R + row;   // of the CTA; of the unit
    const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16, t_s = tmem + lanes + 128 * t, t_o = tmem_o + lanes + 128 * t;
    // Where the threads are in the work lies in shared memory while they go through a unit: all registers are wanted there, and what spills comes
    // from L2, since shared memory takes all of L1.
    volatile Held* held = reinterpret_cast<volatile Held*>(misc + 16);
    auto hold = [&]() {
      threads_meet<C::SOFT>();                                                        // everyone has recalled the one before
      if (threadIdx.x == 0) {
        held->b = at.b, held->row0 = at.row0, held->n = at.n, held->len = at.len, held->tiles = at.tiles, held->units = at.units, held->unit = at.unit, held->tile = at.tile, held->over = at.over;
        held->left = at.left, held->begin = begin, held->end = end, held->per = per;
      }
      threads_meet<C::SOFT>();
    };
    auto recall = [&]() {
      at.b = held->b, at.row0 = held->row0, at.n = held->n, at.len = held->len, at.tiles = held->tiles, at.units = held->units, at.unit = held->unit, at.tile = held->tile, at.over = held->over;
      at.left = held->left, begin = held->begin, end = held->end, per = held->per;
    };
    int tiles = 0, done = 0;                                                          // tiles, steps before the unit
    for (;;) {
      hold();
      float m = -INFINITY, l = 0.0f, lg_ref = -INFINITY;
      int steps, see;
      {
        const Seg g = segment(at);
        const int i = g.qt * a.tq + urow / a.Gc, hq = g.chunk * a.Gc + urow % a.Gc;
        const bool real = urow < a.tq * a.Gc && i < at.n && hq < a.G;
        see = (real ? max(at.len - at.n + i + 1, 0) : 0x7FFFFFFF) - g.first * TK;      // keys from the segment's first on
        steps = g.steps;
      }
      if (steps > 0) {
        float f1, f2;
        {
          // ---- the warp's 32 rows of queries, D / 8 lanes a row, sixteen bytes a lane (a thread a row by itself took 15000 cycles)
          constexpr int LPR = D / 8, RPI = 32 / LPR;                                   // lanes a row, rows an iteration
          const Seg g = segment(at);
          const int piece = lane % LPR, r0 = rank * R + 128 * t + 32 * (warp & 3);
          int mine = 0;                                                                // exponent of the thread's own row; a large one where it is broken
          auto fetch = [&](int it) {
            const int r = r0 + it * RPI + lane / LPR, i = g.qt * a.tq + r / a.Gc, hq = g.chunk * a.Gc + r % a.Gc;
            if (!(r < a.tq * a.Gc && i < at.n && hq < a.G)) return make_uint4(0, 0, 0, 0);
            return *(reinterpret_cast<const uint4*>(a.q + (long long)(at.row0 + i) * a.q_stride + (long long)(g.h * a.G + hq) * D) + piece);
          };
          constexpr int AHEAD = 4;
#pragma unroll 1
          for (int it0 = 0; it0 < 32 / RPI; it0 += AHEAD) {
            uint4 raw[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) raw[u] = fetch(it0 + u);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
              const uint4 x = raw[u];
              uint32_t top = __vmaxu2(__vmaxu2(x.x & 0x7FFF7FFFu, x.y & 0x7FFF7FFFu), __vmaxu2(x.z & 0x7FFF7FFFu, x.w & 0x7FFF7FFFu));
              top = max(top >> 16, top & 0xFFFFu) << 16;
#pragma unroll
              for (int o = 1; o < LPR; o <<= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
              const bool bad = top >= 0x7F800000u || at.over;
              const int e = bad ? 1 << 20 : top > 0 ? ilogbf(__uint_as_float(top)) : 0, es = bad ? 0 : e;
#pragma unroll
              for (int k = 0; k < RPI; ++k) {
                const int other = __shfl_sync(0xFFFFFFFFu, e, k * LPR);
                if (lane == (it0 + u) * RPI + k) mine = other;
              }
              // to [2^14, 2^15), turned round where the scale is negative, so that the largest score stays the largest
              const float up0 = bad ? 0.0f : (a.scale < 0.0f ? -1.0f : 1.0f) * power2((14 - es) / 2), up1 = power2(14 - es - (14 - es) / 2);
              uint32_t w[4];
#pragma unroll
              for (int k = 0; k < 2; ++k) {                                           // four dimensions, in the order 0, 2, 1, 3
                const uint32_t p0 = bad ? 0u : k ? x.z : x.x, p1 = bad ? 0u : k ? x.w : x.y;
                w[2 * k] = pack_half(__uint_as_float(p0 << 16) * up0 * up1, __uint_as_float(p1 << 16) * up0 * up1);
                w[2 * k + 1] = pack_half(__uint_as_float(p0 & 0xFFFF0000u) * up0 * up1, __uint_as_float(p1 & 0xFFFF0000u) * up0 * up1);
              }
              const int r = 32 * (warp & 3) + (it0 + u) * RPI + lane / LPR;            // of the row tile
              sts128(sb + C::O_Q + t * C::HALF_BYTES + r * 128 + (piece >> 3) * (TK * 128) + (((piece & 7) ^ (r & 7)) << 4), w[0], w[1], w[2], w[3]);
            }
          }
          const bool bad = mine == 1 << 20;
          const int e = bad ? 0 : mine;
          f1 = bad ? __uint_as_float(0x7FC00000u) : fabsf(a.scale) * LOG2E * power2(e / 2);
          f2 = power2(e - e / 2 - 14);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) tell(bar_q + 8 * t);
        }
#pragma unroll 1
        for (int n = 0; n < steps; ++n) {
          const int b = (done + n) & 1, tile = tiles + (n >> 1), tok = n * C::STEP;
          const bool edge = __any_sync(0xFFFFFFFFu, tok + C::STEP > see);
          if (!mbar_wait(bar_s + 16 * t + 8 * b, (uint32_t)((done + n) >> 1) & 1u, abort_flag)) fail(10);
          __syncwarp();
          tc_fence_after();
          // The scales were put down before the tile's codes were asked for, and the scores came behind these.  (The barrier of the f16 keys is not for these
          // threads to wait for: it may be two phases further by now, and a parity does not tell.)
          float c[4], lg[4];                                                           // of the step's four times sixteen columns
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float2 sc = meta[tile % C::METAS * 8 + 4 * (n & 1) + q];
            c[q] = sc.x * f1;
            lg[q] = sc.y;
          }
          float lg_top = meta_top[tile % C::METAS * 2 + (n & 1)];                      // the largest that the row sees
          // ---- the step's scores, and their maximum: of sixteen before their page's scale, which is not negative
          uint32_t v[2][32];
          tc_ld32(t_s + 64 * b, v[0]);
          tc_ld32(t_s + 64 * b + 32, v[1]);
          tc_wait_ld();
          if (edge) {
            lg_top = -INFINITY;
#pragma unroll
            for (int q = 0; q < 4; ++q)
              if (tok + 16 * q < see) lg_top = fmaxf(lg_top, lg[q]);
#pragma unroll
            for (int x = 0; x < 64; ++x) v[x / 32][x % 32] = tok + x < see ? v[x / 32][x % 32] : 0xFF800000u;
          }
          float most = -INFINITY;
          bool usual = !edge;                                                          // and factors of the scores that one FP32 number holds
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int x = 0; x < 16; x += 2) top[(x >> 1) & 1] = max3(top[(x >> 1) & 1], __uint_as_float(v[q / 2][16 * (q & 1) + x]), __uint_as_float(v[q / 2][16 * (q & 1) + x + 1]));
            const float cf = c[q] * f2, topmost = fmaxf(top[0], top[1]);
            usual = usual && (cf == 0.0f ? c[q] == 0.0f : fabsf(cf) > 1e-30f);
            if (topmost > -INFINITY) most = fmaxf(most, topmost * c[q]);
          }
          most = most == -INFINITY ? most : most * f2;
          float fm = 1.0f;
          bool move = false;
          if (most > m + LAG) {                                                        // (or the first)
            fm = ex2(m - most);
            l *= fm;
            m = most;
            move = true;
          }
          if (lg_top > lg_ref) {                                                       // to twice the largest, so that a slightly larger one changes nothing
            fm *= ex2(lg_ref - (lg_top + 1.0f));
            lg_ref = lg_top + 1.0f;
            move = true;
          }
          if (n > 0 && __any_sync(0xFFFFFFFFu, move)) {
            // the last product with the values has to be over (the one before it is: these scores came behind it)
            if (!mbar_wait(bar_o + 16 * t + 8 * (b ^ 1), (uint32_t)((done + n - 1) >> 1) & 1u, abort_flag)) fail(11);
            __syncwarp();
            tc_fence_after();
#pragma unroll 1
            for (int q = 0; q < D / 16; ++q) {
              uint32_t o[16];
              tc_ld16(t_o + 16 * q, o);
              tc_wait_ld();
              uint32_t w[8];
#pragma unroll
              for (int x = 0; x < 8; ++x) w[x] = __float_as_uint(__uint_as_float(o[x]) * fm);
              tc_st8(t_o + 16 * q, w);
#pragma unroll
              for (int x = 0; x < 8; ++x) w[x] = __float_as_uint(__uint_as_float(o[8 + x]) * fm);
              tc_st8(t_o + 16 * q + 8, w);
            }
          }
          // The two row tiles' warps of a scheduler take turns with the exponentials: by themselves they go in step in a pair, 1450 cycles for what takes 1000 (388 -> 366 us).
          if (PAIR && (t == 1 || n > 0)) take_turn(2 + 4 * t + (warp & 3));
          // ---- probabilities, over the scores: exp2(s cf - m), times the value scale of the page over the reference
          const float m0 = m == -INFINITY ? 0.0f : m, lg0 = lg_ref == -INFINITY ? 0.0f : lg_ref;
          if (__all_sync(0xFFFFFFFFu, usual)) {
            uint64_t sum = 0;                                                          // of even and odd columns
            const uint64_t minus_m = pair64(-m0, -m0);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              uint32_t p[8];
              const float cf = c[q] * f2, rel = ex2(lg[q] - lg0) * P_ONE;
              const uint64_t cf2 = pair64(cf, cf), rel2 = pair64(rel, rel);
#pragma unroll
              for (int x = 0; x < 8; ++x) {
                const uint64_t z = fma2(pair64(__uint_as_float(v[q / 2][16 * (q & 1) + 2 * x]), __uint_as_float(v[q / 2][16 * (q & 1) + 2 * x + 1])), cf2, minus_m);
                const uint64_t e = pair64(ex2(low64(z)), ex2(high64(z)));
                sum = add2(sum, e);
                const uint64_t w = mul2(e, rel2);
                p[x] = pack_half(low64(w), high64(w));
              }
              tc_st8(t_s + 64 * b + 8 * q, p);
            }
            l += low64(sum) + high64(sum);
          } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              uint32_t p[8];
              const float rel = ex2(lg[q] - lg0) * P_ONE;
#pragma unroll
              for (int x = 0; x < 16; x += 2) {
                float e[2], w[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  const bool seen = tok + 16 * q + x + k < see;                        // a scale that is NaN is not the hidden rows' affair
                  e[k] = seen ? ex2(__fmaf_rn(__uint_as_float(v[q / 2][16 * (q & 1) + x + k]) * c[q], f2, -m0)) : 0.0f;
                  w[k] = seen ? e[k] * rel : 0.0f;
                }
                l += e[0] + e[1];
                p[x / 2] = pack_half(w[0], w[1]);
              }
              tc_st8(t_s + 64 * b + 8 * q, p);
            }
          }
          if (PAIR && (t == 0 || n < steps - 1)) give_turn(2 + 4 * (t ^ 1) + (warp & 3));
          tc_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            // what it tells of is in TMEM and ordered by the fence; a release of the cluster takes 900 cycles
            if (PAIR) peer_arrive_relaxed(peer_addr(bar_p + 16 * t + 8 * b, 0));
            else mbar_arrive(bar_p + 16 * t + 8 * b);
          }
        }
        // The last product; those before it are over with it.  A barrier for each buffer: of one for all steps the phase before would not be known to be over,
        // and a parity tells two neighbouring phases apart, no more.
        if (!mbar_wait(bar_o + 16 * t + 8 * ((done + steps - 1) & 1), (uint32_t)((done + steps - 1) >> 1) & 1u, abort_flag)) fail(12);
        __syncwarp();
        tc_fence_after();
        tiles += (steps + 1) >> 1;
        done += steps;
      }
      recall();
      const Seg g = segment(at);
      const int i = g.qt * a.tq + urow / a.Gc, hq = g.chunk * a.Gc + urow % a.Gc;
      const bool real = urow < a.tq * a.Gc && i < at.n && hq < a.G;
      // ---- the end of the unit.  lg_ref may be -infinity: nothing but values of scale 0 was met, and O is 0
      const bool whole = g.first == 0 && g.n_items == at.tiles, any = g.steps > 0;
      const float ta = lg_ref == -INFINITY ? -INFINITY : m + lg_ref;
      const long long out_row = (long long)(at.row0 + i) * a.c.heads * a.G + g.h * a.G + hq;
      // sixteen columns of O, in the order of the dimensions 0, 2, 1, 3 of four, times f to the output
      auto put = [&](int d, const float (&v)[16], float f, bool none) {
        uint32_t w[8];
#pragma unroll
        for (int x = 0; x < 16; x += 4) {
          const __nv_bfloat162 lo = __floats2bfloat162_rn(none ? 0.0f : v[x] * f, none ? 0.0f : v[x + 2] * f), hi = __floats2bfloat162_rn(none ? 0.0f : v[x + 1] * f, none ? 0.0f : v[x + 3] * f);
          w[x / 2] = *reinterpret_cast<const uint32_t*>(&lo);
          w[x / 2 + 1] = *reinterpret_cast<const uint32_t*>(&hi);
        }
        uint4* to = reinterpret_cast<uint4*>(a.out + out_row * D + d);
        to[0] = make_uint4(w[0], w[1], w[2], w[3]);
        to[1] = make_uint4(w[4], w[5], w[6], w[7]);
      };
      float4* part = reinterpret_cast<float4*>(a.parts + ((long long)blockIdx.x * 2 + (g.first > 0 ? 0 : 1)) * C::PART_FLOATS);   // [D / 4][R] four columns, then the statistics
      {
        const bool none = l == 0.0f;
        const float f = none || ta == -INFINITY ? 0.0f : ex2(ta - m) / l;
        if (whole && real && a.lse) a.lse[out_row] = none ? -INFINITY : (m + log2f(l)) * LN2;
#pragma unroll 2
        for (int q = 0; q < D / 16; ++q) {
          uint32_t o[16];
          float v[16];
          if (any) {
            tc_ld16(t_o + 16 * q, o);
            tc_wait_ld();
          }
#pragma unroll
          for (int x = 0; x < 16; ++x) v[x] = any ? __uint_as_float(o[x]) * (1.0f / P_ONE) : 0.0f;
          if (whole) {
            if (real) put(16 * q, v, f, none);
          } else {
#pragma unroll
            for (int x = 0; x < 4; ++x) __stcg(part + (4 * q + x) * R + row, make_float4(v[4 * x], v[4 * x + 1], v[4 * x + 2], v[4 * x + 3]));
          }
        }
      }
      tc_fence_before();
      if (!whole) {
        float* stat = reinterpret_cast<float*>(part) + D * R;
        __stcg(stat + row, ta);
        __stcg(stat + R + row, m);
        __stcg(stat + 2 * R + row, l);
        // the last of the unit's CTAs to get here adds the parts up, a thread a row
        const long long unit_begin = begin + (end - begin - at.left) - g.first;
        const int c_first = (int)(unit_begin / per), parts = (int)((unit_begin + at.tiles - 1) / per) - c_first + 1;
        threads_meet<C::SOFT>();
        if (threadIdx.x == 0) {
          uint32_t seen;
          asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(seen) : "l"(a.counters + c_first * CTAS + rank) : "memory");
          misc[7] = seen == (uint32_t)(parts - 1);
          if (misc[7]) a.counters[c_first * CTAS + rank] = 0;
        }
        threads_meet<C::SOFT>();
        if (misc[7]) {
          auto part_of = [&](int c) { return a.parts + (((long long)(c_first + c) * CTAS + rank) * 2 + (c == 0)) * C::PART_FLOATS; };
          float top_a = -INFINITY, top_m = -INFINITY, sum_l = 0.0f;
#pragma unroll 1
          for (int c = 0; c < parts; ++c) {
            const float *p = part_of(c) + D * R + row, ac = __ldcg(p), mc = __ldcg(p + R), lc = __ldcg(p + 2 * R), nm = fmaxf(top_m, mc);
            top_a = fmaxf(top_a, ac);
            sum_l = rebase(top_m, sum_l, nm) * sum_l + rebase(mc, lc, nm) * lc;
            top_m = nm;
          }
          const bool none = sum_l == 0.0f;
          const float f = none || top_a == -INFINITY ? 0.0f : ex2(top_a - top_m) / sum_l;
          if (real && a.lse) a.lse[out_row] = none ? -INFINITY : (top_m + log2f(sum_l)) * LN2;
#pragma unroll 1
          for (int d = 0; d < D; d += 16) {
            float sum[16];
#pragma unroll
            for (int x = 0; x < 16; ++x) sum[x] = 0.0f;
#pragma unroll 2
            for (int c = 0; c < parts; ++c) {
              const float* p = part_of(c);
              const float ac = __ldcg(p + D * R + row), fc = ac == -INFINITY ? 0.0f : ex2(ac - top_a);
              float4 v[4];
#pragma unroll
              for (int x = 0; x < 4; ++x) v[x] = __ldcg(reinterpret_cast<const float4*>(p) + (d / 4 + x) * R + row);
#pragma unroll
              for (int x = 0; x < 4; ++x) sum[4 * x] += fc * v[x].x, sum[4 * x + 1] += fc * v[x].y, sum[4 * x + 2] += fc * v[x].z, sum[4 * x + 3] += fc * v[x].w;
            }
            if (real) put(d, sum, f, none);
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
  if (PAIR) {                                                          // the other CTA's MMAs may still read this one's operands, its threads arrive at this one's barriers
    __syncwarp();
    cluster_meet();
    tc_fence_after();
  }
  if (warp == C::W_MMA) {
    if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

template <int D, int CTAS>
int launch_as(AttnArgs& a, cudaStream_t st) {
  using C = ManyCfg<D, CTAS>;
  static_assert(C::SMEM_BYTES <= 232448, "shared memory of a CTA");
  constexpr int ROWS = C::R * CTAS;
  a.Gc = a.G < ROWS ? a.G : ROWS;
  a.chunks = (a.G + a.Gc - 1) / a.Gc;
  a.tq = ROWS / a.Gc;
  CUtensorMap map_k, map_v;
  RAZER_TRY(attn_encode_pool(&map_k, a.c.k, a.c, CTAS == 2 && a.c.page > 32 ? 32 : a.c.page, D));
  RAZER_TRY(attn_encode_pool(&map_v, a.c.v, a.c, a.c.page, C::V_DIMS));
  static std::atomic<uint64_t> allowed{0};
  RAZER_TRY(allow_smem((const void*)attn_kv8_many_kernel<D, CTAS>, C::SMEM_BYTES, allowed));
  const int ctas = (sm_count() < ATTN_CTAS ? sm_count() : ATTN_CTAS) / CTAS * CTAS;
  return launch_dependent_clusters("attn_kv8_many_kernel launch", attn_kv8_many_kernel<D, CTAS>, dim3((unsigned)ctas), CTAS, C::THREADS, C::SMEM_BYTES, st, map_k, map_v, a);
}

}  // namespace

size_t attn_many_part_floats(int D) { return D == 64 ? ManyCfg<64, 1>::PART_FLOATS : ManyCfg<128, 1>::PART_FLOATS; }

int launch_attn_many(AttnArgs& a, bool pairs, cudaStream_t st) {
  if (a.c.D == 64) return launch_as<64, 1>(a, st);
  return pairs ? launch_as<128, 2>(a, st) : launch_as<128, 1>(a, st);
}

}  // namespace razer
