// Attention over the paged 8-bit cache for few rows of queries a key-value head (decoding): up to 32 of them at a time.
//
// The cache goes to the tensor core as it lies: keys and values are operand A of integer MMAs (tcgen05 kind::i8), brought by TMA and
// never converted.  Queries and probabilities are operand B, split into 8-bit digits that are columns of their own:
//   S[token][row, digit] = K Q^T    q = 2^(e - 21) (65536 d2 + 256 d1 + d0), signed digits, e from the row's largest magnitude
//   O[dim][row, digit]   = V^T P    w = exp2(s + log2 vs - top) <= 1 held as 24 bits, three unsigned digits, top the tile's own maximum
// The sums are exact in 32 bits, so that what is rounded is q to 2^-22 of its row's largest (bf16 queries exactly but for those below 2^-14
// of it), w to 2^-25 of the tile's largest, and the FP32 arithmetic between.  One maximum serves both sums, of s + max(log2 vs, the tile's largest - 60): it
// stays above every weight, and within 2^60 of the largest exponential.  Where value scales of a tile lie further apart (a page of zeros too) it may be far above the
// weights that there are; theirs is then found as well.  A tile is 128 tokens: a lane of TMEM each for S, a lane for each
// dimension for O.  Since the digits ride along as columns (32 of S and of O for 8 rows, against 54 cycles that an MMA takes at any
// width up to 64), they cost nothing, and a tile takes a third of the instructions that unpacking codes for mma.sync took.
//
// Roles: a warp each brings keys and values (pages and scales looked up 32 at a time), one prepares the queries of the next unit, one issues
// MMAs, and GROUPS groups of four warps take the tiles in turn: maximum over the tile (a warp reduction a row, then the four warps
// through shared memory), exponentials, digits to shared memory, and O = O f + O_tile in FP32 registers.  Work is cut evenly
// among the CTAs as razer_attn_kv8.cuh says.
//
// What bounds it: the chain of a tile in each softmax group (scores, maxima, the group's meeting, exponentials, digits; every instruction in it counts, while issue slots are 37 %
// busy and HBM 56 % at 8 rows and 26 % at 32), then HBM.  64 sequences of up to 16384 tokens, 8 x 8 heads of 128 (1.28 GB) 201 to 214 us (6.0 to 6.4 TB/s) as long as the clock is up; in
// a loop of some seconds the GPU is at its power limit (1000 W, 1700 instead of 1965 MHz) and the call takes 228 (241 before rows went two to an instruction, packed
// FP32, and maxima by redux.sync).  32 sequences of 4096 tokens: 54 us for 8 rows, 78 for 16, 121 for 32 (83 and 169 before that).  One sequence of 4096 tokens, 8 x 4 heads
// of 64: 11.5 a call, 11.6 in a graph, latency: launch, the look at the batch, 2 to 3 tiles a CTA, the meeting of 16 parts.  Heads of 64: 79 us for 268 MB in pages of 64, 95 in pages
// of 16 (boxes of 1 KB).
#include "razer_attn_kv8.cuh"

namespace razer {

namespace {

constexpr float W_ONE = 16777215.0f;                                   // what a weight of 1 is held as: 24 bits
constexpr float FLOOR = 60.0f;                                         // how far (log2) below the tile's largest value scale a token's counts as in the common maximum

template <int D_, int R_>
struct FewCfg {
  static constexpr int D = D_, R = R_, CHUNKS = R_ / 8;
  static constexpr int TK = 128;
  static constexpr int GROUPS = R_ == 8 ? 3 : 2;                     // registers: 128 a thread with three groups, 168 with two
  static constexpr int W_K = 4 * GROUPS, W_V = W_K + 1, W_Q = W_K + 2, W_MMA = W_K + 3;       // the service warps
  static constexpr int THREADS = 32 * (W_K + 4);
  static constexpr int TILE_BYTES = TK * D, STAGE_BYTES = 2 * TILE_BYTES;
  static constexpr int NS = R_ == 8 ? 32 : 3 * R_, NP = NS;                                // columns of S and of O
  static constexpr int Q_BYTES = NS * D, P_BYTES = NP * TK;
  static constexpr int STAGES = (D_ == 64 ? 2 : 1) * (R_ <= 16 ? 6 : 5);
  static constexpr int TABLES = CHUNKS == 1 ? 2 : 1;
  static constexpr int O_RING = 0;
  static constexpr int O_Q = STAGES * STAGE_BYTES;                     // two buffers, [column][D]
  static constexpr int O_P = (O_Q + 2 * Q_BYTES + 1023) / 1024 * 1024; // [group][column][128]
  static constexpr int JOIN_BYTES = GROUPS * 32 * D > (ATTN_CTAS + 3) * R * 4 ? GROUPS * 32 * D : (ATTN_CTAS + 3) * R * 4;   // [group][8 rows][D] floats, then attn_combine's; over the digits where they have the room:
  static constexpr bool JOIN_ON_P = JOIN_BYTES <= GROUPS * P_BYTES;    // at a unit's end they have been read
  static constexpr int O_JOIN = JOIN_ON_P ? O_P : O_P + GROUPS * P_BYTES;
  static constexpr int O_RED = O_P + GROUPS * P_BYTES + (JOIN_ON_P ? 0 : JOIN_BYTES);   // [group][with the floor, without][2][4 warps][R]
  static constexpr int O_STAT = O_RED + GROUPS * 16 * R * 4;            // [group][R] A, M; [group][4][R] sums
  static constexpr int O_TABLE = O_STAT + GROUPS * 6 * R * 4;          // [warp][TABLES][8][R] what a tile means for each row
  static constexpr int O_ROW = O_TABLE + 4 * GROUPS * TABLES * R * 32; // [2][R] score factor in two parts; [2][R] keys
  static constexpr int O_META = O_ROW + 2 * R * 12;                    // [STAGES][8] {key scale, log2 of the value scale}, [STAGES] {the largest of the latter, whether they lie far apart}
  static constexpr int O_BAR = (O_META + STAGES * 72 + 7) / 8 * 8;
  static constexpr int N_BAR = 3 * STAGES + 3 * GROUPS + 5;
  static constexpr int O_MISC = O_BAR + 8 * N_BAR;                     // words: abort, never set, share (4 words), TMEM, last, broken values by group, sums
  static constexpr int SMEM_BYTES = 1024 + O_MISC + 256;
  static constexpr int S_COLS = NS <= 32 ? 32 : NS <= 64 ? 64 : 128, P_COLS = S_COLS;
  static constexpr int TMEM_COLS = GROUPS * (S_COLS + P_COLS) <= 256 ? 256 : 512;
  static constexpr int PART_FLOATS = R * (D + 3);                      // a part of a unit: O, A, M, sum
};

// The sum of each of eight values over a warp: nine shuffles; lane gets that of value sum8_row.
__device__ __forceinline__ float sum8(const float (&v)[8], int lane) {
  float a[4], b[2];
  const bool h4 = lane & 16, h3 = lane & 8, h2 = lane & 4;
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] = (h4 ? v[4 + i] : v[i]) + __shfl_xor_sync(0xFFFFFFFFu, h4 ? v[i] : v[4 + i], 16);
#pragma unroll
  for (int i = 0; i < 2; ++i) b[i] = (h3 ? a[2 + i] : a[i]) + __shfl_xor_sync(0xFFFFFFFFu, h3 ? a[i] : a[2 + i], 8);
  float c = (h2 ? b[1] : b[0]) + __shfl_xor_sync(0xFFFFFFFFu, h2 ? b[0] : b[1], 4);
  c += __shfl_xor_sync(0xFFFFFFFFu, c, 2);
  return c + __shfl_xor_sync(0xFFFFFFFFu, c, 1);
}
__device__ __forceinline__ int sum8_row(int lane) { return ((lane >> 4) & 1) * 4 + ((lane >> 3) & 1) * 2 + ((lane >> 2) & 1); }

// The largest over a warp (NaN counts as none), in all lanes.
__device__ __forceinline__ float warp_max(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xFFFFFFFF;" : "=f"(r) : "f"(v));
  return r;
}
// Eight numbers of shared memory as four pairs.
__device__ __forceinline__ void pairs8(const float* p, uint64_t (&v)[4]) {
  const ulonglong2 a = reinterpret_cast<const ulonglong2*>(p)[0], b = reinterpret_cast<const ulonglong2*>(p)[1];
  v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
}
// 65536 d2 + 256 d1 + d0 of the rows 2 j and 2 j + 1 of eight: columns d0 of all rows, d1, d2.
__device__ __forceinline__ uint64_t join_digits(const uint32_t (&x)[24], int j) {
  const uint64_t low = pair64((float)((int)x[8 + 2 * j] * 256 + (int)x[2 * j]), (float)((int)x[9 + 2 * j] * 256 + (int)x[2 * j + 1]));
  return fma2(pair64((float)(int)x[16 + 2 * j], (float)(int)x[17 + 2 * j]), pair64(65536.0f, 65536.0f), low);
}

__device__ __forceinline__ void mma_digits(uint32_t d_tmem, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 ad, bd;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "mov.b64 ad, {%1, %2};\n\t"
      "mov.b64 bd, {%3, %4};\n\t"
      "tcgen05.mma.cta_group::1.kind::i8 [%0], ad, bd, %5, p;\n\t}" ::"r"(d_tmem),
      "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tc_ld8(uint32_t taddr, uint32_t* v) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tc_ld4(uint32_t taddr, uint32_t* v) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void sts8(uint32_t addr, uint32_t v) { asm volatile("st.shared.u8 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }

template <int D, int R, int LIVE>
__global__ void __launch_bounds__(FewCfg<D, R>::THREADS, 1) attn_kv8_few_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                                                                                const __grid_constant__ AttnArgs a) {
  using C = FewCfg<D, R>;
  constexpr int LP = LIVE < 8 ? LIVE / 2 : 4;                              // pairs of rows of eight that are worked on
  constexpr int TK = C::TK, ST = C::STAGES, GROUPS = C::GROUPS, CHUNKS = C::CHUNKS, SOFT = 128 * GROUPS;
  extern __shared__ uint8_t attn_smem[];
  uint8_t* sm = attn_smem + ((1024 - (smem_u32(attn_smem) & 1023)) & 1023);
  const uint32_t sb = smem_u32(sm);
  const uint32_t bar_kfull = sb + C::O_BAR, bar_vfull = bar_kfull + 8 * ST, bar_empty = bar_vfull + 8 * ST, bar_sfull = bar_empty + 8 * ST,
                 bar_pfull = bar_sfull + 8 * GROUPS, bar_ofull = bar_pfull + 8 * GROUPS, bar_qfull = bar_ofull + 8 * GROUPS, bar_qempty = bar_qfull + 16, bar_drain = bar_qempty + 16;
  int* misc = reinterpret_cast<int*>(sm + C::O_MISC);
  volatile uint32_t* abort_flag = reinterpret_cast<uint32_t*>(misc);
  volatile uint32_t* never = reinterpret_cast<uint32_t*>(misc + 1);
  uint32_t* broken = reinterpret_cast<uint32_t*>(misc + 8);              // [group] rows that saw a value scale that is none
  float2* meta = reinterpret_cast<float2*>(sm + C::O_META);
  float2* meta_top = meta + 8 * ST;
  float* row_scale = reinterpret_cast<float*>(sm + C::O_ROW);             // [2][2][R] the score factor in two parts
  int* row_keys = reinterpret_cast<int*>(row_scale + 4 * R);              // [2][R]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < ST; ++i) {
      mbar_init(bar_kfull + 8 * i, 1);
      mbar_init(bar_vfull + 8 * i, 1);
      mbar_init(bar_empty + 8 * i, 1);
    }
    for (int i = 0; i < GROUPS; ++i) {
      mbar_init(bar_sfull + 8 * i, 1);
      mbar_init(bar_pfull + 8 * i, 4);                   // a warp arrives by one lane: 32 arrivals of a warp take their turns
      mbar_init(bar_ofull + 8 * i, 1);
      broken[i] = 0;
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_qfull + 8 * i, 1);
      mbar_init(bar_qempty + 8 * i, 1);
    }
    mbar_init(bar_drain, 1);
    misc[0] = misc[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
  }
  if (warp == C::W_MMA) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(misc + 6)), "r"((uint32_t)C::TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  grid_dep_wait();
  grid_dep_launch();
  long long begin, end, per;
  Walk at;
  const bool work = attn_share<C::THREADS>(a, TK, misc + 2, reinterpret_cast<long long*>(misc + 16), begin, end, per, at, blockIdx.x, gridDim.x);   // barriers inside
  tc_fence_after();
  const uint32_t tmem = (uint32_t)misc[6];
  const int heads = a.c.heads * a.chunks;
  auto fail = [&](uint32_t code) {
    *abort_flag = 1;
    atomicCAS(a.status, 0u, code);
  };
  // a segment: tiles first .. last - 1 of a unit that have a key that anyone sees
  struct Seg { int n_items, qt, h, chunk, keys, first, last; };
  auto segment = [&](const Walk& at) {
    Seg g;
    g.n_items = walk_count(at);
    g.qt = at.unit / heads;
    const int hc = at.unit - g.qt * heads;
    g.h = hc / a.chunks;
    g.chunk = hc - g.h * a.chunks;
    g.keys = max(at.len - at.n + min((g.qt + 1) * a.tq, at.n), 0);
    g.first = at.tile;
    g.last = max(min(at.tile + g.n_items, (g.keys + TK - 1) / TK), g.first);
    return g;
  };

  if (!work) {
  } else if (warp == C::W_K || warp == C::W_V) {
    // ===================== keys, values =====================
    const bool value = warp == C::W_V;
    const CUtensorMap* map = value ? &map_v : &map_k;
    const uint32_t bar_full = value ? bar_vfull : bar_kfull, to0 = sb + C::O_RING + (value ? C::TILE_BYTES : 0);
    const int boxes = TK >> a.c.page_log2;                       // pages of a tile
    int item = 0;
    bool alive = true;
    do {
      const Seg g = segment(at);
      // The lanes hold 32 blocks from `have` on: pages and (values' warp) scales, the pages of the next 32, and the scales of those on their way
      int have = (g.first * boxes) & ~31, id, id_next;
      float ks = 0, lg = 0, ks_next = 0, vs_next = 0;            // key scale; log2 of the value scale; both of the next 32
      auto page_of = [&](int block) { return ((long long)block << a.c.page_log2) < g.keys ? kv8_page(a.c, a.s, at.b, block) : -1; };
      auto ask = [&]() {
        ks_next = vs_next = __uint_as_float(0x7FC00000u);
        if (value && id_next >= 0) {
          ks_next = a.c.k_scales[(long long)id_next * a.c.heads + g.h];
          vs_next = a.c.v_scales[(long long)id_next * a.c.heads + g.h];
        }
      };
      auto step = [&]() {
        id = id_next;
        ks = ks_next < 0.0f ? __uint_as_float(0x7FC00000u) : ks_next;
        if (value) lg = vs_next >= 0.0f && vs_next < INFINITY ? log2f(vs_next) : __uint_as_float(0x7FC00000u);   // -infinity for 0
      };
      id_next = page_of(have + lane);
      int id_after = page_of(have + 32 + lane);
      ask();
      step();
      id_next = id_after;
      ask();
      id_after = page_of(have + 64 + lane);
      for (int t = g.first; t < g.last; ++t, ++item) {
        const int block0 = t * boxes, stage = item % ST;
        if (block0 >= have + 32) {
          have += 32;
          step();
          id_next = id_after;
          ask();
          id_after = page_of(have + 64 + lane);
        }
        if (item >= ST && !mbar_wait(bar_empty + 8 * stage, (uint32_t)((item / ST) & 1) ^ 1u, abort_flag)) {
          fail(1);
          alive = false;
        }
        alive = __all_sync(0xFFFFFFFFu, alive);
        if (!alive) break;
        const uint32_t bar = bar_full + 8 * stage;
        const int live = min(boxes, ((g.keys - t * TK - 1) >> a.c.page_log2) + 1);
        const int page = __shfl_sync(0xFFFFFFFFu, id, (block0 - have + lane) & 31);
        if (value) {
          float k1 = __shfl_sync(0xFFFFFFFFu, ks, (block0 - have + lane) & 31), v1 = __shfl_sync(0xFFFFFFFFu, lg, (block0 - have + lane) & 31);
          if (lane >= live) k1 = 0.0f, v1 = -INFINITY;           // no token that anyone sees
          float most = v1;
          for (int o = 1; o < 8; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
          const bool apart = __any_sync(0xFFFFFFFFu, lane < live && v1 < most - FLOOR);      // (live: up to 8; false where all are 0)
          if (!(most > -INFINITY)) most = 0.0f;                  // all of them 0 or broken
          if (lane < 8) meta[stage * 8 + lane] = make_float2(k1, v1);
          if (lane == 0) meta_top[stage] = make_float2(most, apart ? 1.0f : 0.0f);
          __syncwarp();
        }
        if (lane == 0) mbar_expect_tx(bar, (uint32_t)((live << a.c.page_log2) * D));
        __syncwarp();
        if (lane < live)
          tma_load_3d(to0 + stage * C::STAGE_BYTES + (uint32_t)((lane << a.c.page_log2) * D), map, 0, 0, max(page, 0) * a.c.heads + g.h, bar);
        __syncwarp();
      }
      if (!walk_advance(a, TK, at, g.n_items)) break;
    } while (alive);
    // copies in flight must land before shared memory is released
    for (int f = max(item - ST, 0); f < item; ++f) mbar_wait(bar_full + 8 * (f % ST), (uint32_t)((f / ST) & 1), never);
  } else if (warp == C::W_Q) {
    // ===================== queries of the next unit =====================
    for (int n = 0;; ++n) {
      const Seg g = segment(at);
      const int buf = n & 1;
      if (n >= 2 && !mbar_wait(bar_qempty + 8 * buf, (uint32_t)((n >> 1) & 1) ^ 1u, abort_flag)) { fail(2); break; }
      __syncwarp();
      const bool over = at.over;
#pragma unroll 1
      for (int c = 0; c < CHUNKS; ++c) {                          // eight rows at once, four lanes a row, D / 4 dimensions a lane
        const int j = lane >> 2, part = lane & 3, r = 8 * c + j, i = g.qt * a.tq + r / a.Gc, hq = g.chunk * a.Gc + r % a.Gc;
        const bool real = r < a.tq * a.Gc && i < at.n && hq < a.G;
        const uint4* src = reinterpret_cast<const uint4*>(a.q + (long long)(at.row0 + i) * a.q_stride + (long long)(g.h * a.G + hq) * D) + part * (D / 32);
        uint4 raw[D / 32];
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) raw[k] = real ? src[k] : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int k = 0; k < D / 32; ++k)
          top = __vmaxu2(__vmaxu2(top, __vmaxu2(raw[k].x & 0x7FFF7FFFu, raw[k].y & 0x7FFF7FFFu)), __vmaxu2(raw[k].z & 0x7FFF7FFFu, raw[k].w & 0x7FFF7FFFu));
        top = max(top >> 16, top & 0xFFFFu) << 16;
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        const bool bad = top >= 0x7F800000u || over;
        const int e = top > 0 && !bad ? ilogbf(__uint_as_float(top)) : 0;
        const float up0 = power2((21 - e) / 2), up1 = power2(21 - e - (21 - e) / 2);
        if (part == 0) {
          row_scale[2 * buf * R + r] = bad ? __uint_as_float(0x7FC00000u) : a.scale * LOG2E * power2(e / 2);
          row_scale[(2 * buf + 1) * R + r] = power2(e - e / 2 - 21);
          row_keys[buf * R + r] = real ? max(at.len - at.n + i + 1, 0) : 0x7FFFFFFF;
        }
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
          const uint32_t w[4] = {raw[k].x, raw[k].y, raw[k].z, raw[k].w};
#pragma unroll
          for (int b = 0; b < 2; ++b) {                           // four dimensions: a word of each digit
            uint32_t digit[3] = {0, 0, 0};
#pragma unroll
            for (int m = 0; m < 4; ++m) {
              const uint32_t pair = w[2 * b + (m >> 1)];
              int v = bad ? 0 : __float2int_rn(__uint_as_float((m & 1) ? pair & 0xFFFF0000u : pair << 16) * up0 * up1);
#pragma unroll
              for (int q = 0; q < 3; ++q) {
                const int lo = (int)(int8_t)v;
                digit[q] |= (uint32_t)(lo & 255) << (8 * m);
                v = (v - lo) >> 8;
              }
            }
            const int d = part * (D / 4) + 8 * k + 4 * b;
#pragma unroll
            for (int q = 0; q < 3; ++q) {
              const int col = 24 * c + 8 * q + j;
              const uint32_t chunk16 = D == 64 ? (d >> 4) ^ ((col >> 1) & 3) : (d >> 4) ^ (col & 7);
              asm volatile("st.shared.u32 [%0], %1;" ::"r"(sb + C::O_Q + buf * C::Q_BYTES + col * D + chunk16 * 16 + (d & 15)), "r"(digit[q]) : "memory");
            }
          }
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_qfull + 8 * buf);
      if (!walk_advance(a, TK, at, g.n_items)) break;
    }
  } else if (warp == C::W_MMA) {
    // ===================== MMAs =====================
    if (elect_one()) {
      constexpr uint32_t hi_row = D == 64 ? (512u >> 4) | (1u << 14) | (4u << 29) : (1024u >> 4) | (1u << 14) | (2u << 29);   // rows of D bytes in their swizzle
      constexpr uint32_t hi_p = (1024u >> 4) | (1u << 14) | (2u << 29);
      // S32 sums; keys x query digits, both signed; values (dimension-major, M = D) signed x probability digits unsigned
      constexpr uint32_t id_s = (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(C::NS >> 3) << 17) | (8u << 24);
      constexpr uint32_t id_p = (2u << 4) | (1u << 7) | (1u << 15) | ((uint32_t)(C::NP >> 3) << 17) | ((uint32_t)(D >> 4) << 24);
      auto lo = [](uint32_t addr) { return (addr >> 4) | (1u << 16); };
      // Whichever is ready goes first: the product with the values of the oldest tile whose weights are down, else the scores of the next tile, of the
      // next unit too.  (In a fixed order the last products of a unit waited for the next one's keys: 1500 to 2800 cycles a unit.)
      auto ready = [&](uint32_t bar, int phase) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok)
                     : "r"(bar), "r"((uint32_t)(phase & 1))
                     : "memory");
        return ok != 0;
      };
      int item = 0, weighed = 0;                                 // next scores, next product; at most GROUPS apart
      int n = 0;
      Seg s = segment(at);
      int t = s.first;
      bool more = true, queries = false;                         // segments are left; this one's queries are there
      uint32_t idle = 0;
      uint64_t since = 0;
      while (more || weighed < item) {
        if (weighed < item && ready(bar_pfull + 8 * (weighed % GROUPS), weighed / GROUPS) && ready(bar_vfull + 8 * (weighed % ST), weighed / ST)) {
          const int g = weighed % GROUPS, stage = weighed % ST;
          tc_fence_after();
          const uint32_t v = sb + C::O_RING + stage * C::STAGE_BYTES + C::TILE_BYTES, p = sb + C::O_P + g * C::P_BYTES;
#pragma unroll
          for (int k = 0; k < TK / 32; ++k)
            mma_digits(tmem + GROUPS * C::S_COLS + g * C::P_COLS, lo(v + k * 32 * D), hi_row, lo(p + k * 32), hi_p, id_p, k > 0);
          tc_commit(bar_ofull + 8 * g);
          tc_commit(bar_empty + 8 * stage);
          ++weighed;
          idle = 0;
          continue;
        }
        if (more && !queries) queries = ready(bar_qfull + 8 * (n & 1), n >> 1);    // of every segment in turn, one without tiles too
        if (more && queries && t >= s.last) {
          more = walk_advance(a, TK, at, s.n_items);
          if (more) s = segment(at), t = s.first;
          ++n;
          queries = false;
          idle = 0;
          continue;
        }
        if (more && queries && item - weighed < GROUPS && ready(bar_kfull + 8 * (item % ST), item / ST)) {
          const int g = item % GROUPS;
          tc_fence_after();
          const uint32_t k0 = sb + C::O_RING + (item % ST) * C::STAGE_BYTES, q0 = sb + C::O_Q + (n & 1) * C::Q_BYTES;
#pragma unroll
          for (int k = 0; k < D / 32; ++k) mma_digits(tmem + g * C::S_COLS, lo(k0 + k * 32), hi_row, lo(q0 + k * 32), hi_row, id_s, k > 0);
          tc_commit(bar_sfull + 8 * g);
          ++item;
          ++t;
          idle = 0;
          continue;
        }
        // bounded, as every wait is: by the clock, looked at now and then
        if (++idle % 1024 == 0) {
          const uint64_t now = global_ns();
          if (idle == 1024) since = now;
          else if (now - since > WAIT_LIMIT_NS) fail(3);
          if (*abort_flag) break;
        }
      }
      // what was issued has to be over before shared memory and TMEM go: a commit of its own, waited for whatever happened
      tc_commit(bar_drain);
    }
    __syncwarp();
    mbar_wait(bar_drain, 0, never);
    __syncwarp();
  } else {
    // ===================== softmax: group g takes the tiles g, g + GROUPS, ... =====================
    const int group = warp >> 2, quarter = warp & 3, tid = threadIdx.x & 127;         // tid: token of the tile (S), lane of O
    const uint32_t lanes = (uint32_t)(32 * quarter) << 16;
    const uint32_t t_s = tmem + lanes + group * C::S_COLS, t_o = tmem + lanes + GROUPS * C::S_COLS + group * C::P_COLS;
    const uint32_t p_at = sb + C::O_P + group * C::P_BYTES;
    float* red = reinterpret_cast<float*>(sm + C::O_RED) + group * 16 * R;            // [2][2][4][R]
    float* stat = reinterpret_cast<float*>(sm + C::O_STAT);                           // [group][R] A, M; [group][4][R]
    float* stat_a = stat + group * R;
    float* stat_m = stat + GROUPS * R + group * R;
    float* stat_l = stat + 2 * GROUPS * R + group * 4 * R;
    float* join = reinterpret_cast<float*>(sm + C::O_JOIN);
    float* table = reinterpret_cast<float*>(sm + C::O_TABLE) + warp * C::TABLES * R * 8;
    const int dim = D == 64 ? 16 * quarter + (lane & 15) : tid;                       // of O; with M = 64 the dimensions are lanes 0 .. 15 of each quarter
    const bool has_dim = D != 64 || lane < 16;
    int item = 0, mine = 0;                                                           // the CTA's tiles before this segment; the group's own so far
    for (int n = 0;; ++n) {
      const Seg s = segment(at);
      const int buf = n & 1, n_tiles = s.last - s.first;
      uint64_t o[R / 2], l[R / 2];                                                     // of pairs of rows
      float top_a = -INFINITY, top_m = -INFINITY;                          // lane r: what row r's sums are relative to
#pragma unroll
      for (int r = 0; r < R / 2; ++r) o[r] = l[r] = 0;
      if (!mbar_wait(bar_qfull + 8 * buf, (uint32_t)((n >> 1) & 1), abort_flag)) fail(7);
      __syncwarp();
      int see_all = 0x7FFFFFFF;                                                       // keys that every row sees
      for (int r = 0; r < R; ++r)
        if (r < a.tq * a.Gc) see_all = min(see_all, row_keys[buf * R + r]);
      // O of the group's last tile into the running sums; the registers come first, so that the next product may begin
      uint32_t x_o[CHUNKS == 1 ? 24 : 1];
      auto take = [&](int c, const uint32_t (&x)[24], const float* t) {
        uint64_t so_far[4], now[4];
        pairs8(t + 3 * R + 8 * c, so_far);
        pairs8(t + 4 * R + 8 * c, now);
#pragma unroll
        for (int j = 0; j < LP; ++j) o[4 * c + j] = fma2(o[4 * c + j], so_far[j], mul2(now[j], join_digits(x, j)));
      };
      auto load24 = [&](uint32_t t, uint32_t (&x)[24]) {
        if (LP == 4) {
          tc_ld8(t, x);
          tc_ld8(t + 8, x + 8);
          tc_ld8(t + 16, x + 16);
        } else {
          tc_ld4(t, x);
          tc_ld4(t + 8, x + 8);
          tc_ld4(t + 16, x + 16);
        }
        tc_wait_ld();
      };
      auto row_top = [&](const float* red_now) {                                      // of row `lane`, from the four warps
        float top = -INFINITY;
#pragma unroll
        for (int q = 0; q < 4; ++q) top = fmaxf(top, red_now[q * R + lane]);
        return top;
      };
      bool pending = false;                                                           // the last tile's product with the values is not in yet
      auto take_all = [&]() {
        if (!mbar_wait(bar_ofull + 8 * group, (uint32_t)((mine - 1) & 1), abort_flag)) fail(10);
        __syncwarp();
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
          uint32_t x[24];
          load24(t_o + 24 * c, x);
          take(c, x, table + ((mine - 1) % C::TABLES) * R * 8);
        }
        pending = false;
      };
      for (int i = (group - item % GROUPS + GROUPS) % GROUPS; i < n_tiles; i += GROUPS, ++mine) {
        const int stage = (item + i) % ST, tok = (s.first + i) * TK + tid;
        const bool edge = (s.first + i + 1) * TK > see_all;
        float* tab = table + (mine % C::TABLES) * R * 8;
        float* red_now = red + (mine & 1) * 4 * R;
        // the values' barrier first: their warp has the scales
        if (!mbar_wait(bar_vfull + 8 * stage, (uint32_t)(((item + i) / ST) & 1), abort_flag)) fail(9);
        const float2 sc = meta[stage * 8 + (tid >> a.c.page_log2)];
        const float2 most = meta_top[stage];
        const float lg_top = most.x, lg = sc.y, lg_max = fmaxf(lg, lg_top - FLOOR);   // (a NaN becomes the floor)
        if (!mbar_wait(bar_sfull + 8 * group, (uint32_t)(mine & 1), abort_flag)) fail(8);
        __syncwarp();
        tc_fence_after();
        uint64_t v[R / 2];
        uint32_t seen = 0xFFFFFFFFu;                                                  // rows that see the token
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
          uint64_t f0[4], f1[4], w[4];
          pairs8(row_scale + 2 * buf * R + 8 * c, f0);
          pairs8(row_scale + (2 * buf + 1) * R + 8 * c, f1);
          uint32_t x[24];
          load24(t_s + 24 * c, x);
#pragma unroll
          for (int j = 0; j < LP; ++j) v[4 * c + j] = mul2(mul2(join_digits(x, j), mul2(pair64(sc.x, sc.x), f0[j])), f1[j]);
          if (edge) {
#pragma unroll
            for (int j = 0; j < LP; ++j) {
              const bool s0 = tok < row_keys[buf * R + 8 * c + 2 * j], s1 = tok < row_keys[buf * R + 8 * c + 2 * j + 1];
              v[4 * c + j] = pair64(s0 ? low64(v[4 * c + j]) : -INFINITY, s1 ? high64(v[4 * c + j]) : -INFINITY);
              if (!s0) seen &= ~(1u << (8 * c + 2 * j));
              if (!s1) seen &= ~(2u << (8 * c + 2 * j));
            }
          }
          float t[8] = {};
#pragma unroll
          for (int j = 0; j < LP; ++j) {
            w[j] = add2(v[4 * c + j], pair64(lg_max, lg_max));
            t[2 * j] = warp_max(low64(w[j]));
            t[2 * j + 1] = warp_max(high64(w[j]));
          }
          if (lane == 0) {
            float4* to = reinterpret_cast<float4*>(red_now + quarter * R + 8 * c);
            to[0] = make_float4(t[0], t[1], t[2], t[3]);
            if (LP == 4) to[1] = make_float4(t[4], t[5], t[6], t[7]);
          }
        }
        if (lg != lg && seen) atomicOr(broken + group, seen);                         // a value scale that is none
        // The last tile's product has read its digits by then, and gives way to this one's once it is in registers: late for eight rows, here for more.
        if (CHUNKS > 1 && pending) take_all();
        const bool apart = __any_sync(0xFFFFFFFFu, most.y != 0.0f);                   // one answer for a warp, whatever its lanes have read after a wait that gave up
        if (apart) {
          // Some value scale here is so much smaller than the largest that the floor may make the maximum, above all weights that there are: theirs as well.  (No meeting of its
          // own: after a wait that gave up warps may have read different things here.)
          const uint64_t own = pair64(lg != lg ? -INFINITY : lg, lg != lg ? -INFINITY : lg);
#pragma unroll
          for (int j = 0; j < R / 8 * LP; ++j) {
            const int r = j / LP * 8 + j % LP * 2;
            const uint64_t w = add2(v[r / 2], own);
            const float t0 = warp_max(low64(w)), t1 = warp_max(high64(w));
            if (lane == 0) red_now[(8 + quarter) * R + r] = t0, red_now[(8 + quarter) * R + r + 1] = t1;
          }
        }
        group_meet(group);
        if (lane < R) {                                                               // what all threads want to know of row `lane`
          const float common = row_top(red_now), top = apart ? row_top(red_now + 8 * R) : common;
          const float mn = fmaxf(top_m, common - lg_top), ms = mn == -INFINITY ? 0.0f : mn;
          const float an = fmaxf(top_a, top), as = an == -INFINITY ? 0.0f : an;
          tab[lane] = -ms;
          tab[R + lane] = top == -INFINITY ? 0.0f : -top;
          tab[2 * R + lane] = ex2(top_m - ms);
          tab[3 * R + lane] = ex2(top_a - as);                                        // O so far
          tab[4 * R + lane] = top == -INFINITY ? 0.0f : ex2(top - as);                // the tile's O
          top_m = mn, top_a = an;
        }
        __syncwarp();
        const float lg_w = lg != lg ? -INFINITY : lg;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
          uint64_t ms[4], top[4], so_far[4];
          uint32_t u[8];
          pairs8(tab + 8 * c, ms);
          pairs8(tab + R + 8 * c, top);
          pairs8(tab + 2 * R + 8 * c, so_far);
#pragma unroll
          for (int j = 0; j < LP; ++j) {
            const uint64_t p = v[4 * c + j], e = add2(p, ms[j]), w = add2(add2(p, pair64(lg_w, lg_w)), top[j]);
            l[4 * c + j] = fma2(l[4 * c + j], so_far[j], pair64(ex2(low64(e)), ex2(high64(e))));
            const uint64_t b = mul2(pair64(ex2(low64(w)), ex2(high64(w))), pair64(W_ONE, W_ONE));
            u[2 * j] = __float2uint_rn(low64(b));
            u[2 * j + 1] = __float2uint_rn(high64(b));
          }
          if (CHUNKS == 1 && pending) {
            if (!mbar_wait(bar_ofull + 8 * group, (uint32_t)((mine - 1) & 1), abort_flag)) fail(10);
            __syncwarp();
            tc_fence_after();
            load24(t_o, reinterpret_cast<uint32_t(&)[24]>(x_o));
          }
#pragma unroll
          for (int j = 0; j < 2 * LP; ++j) {
            const uint32_t to = p_at + (24 * c + j) * TK + (tid ^ (j << 4));
            sts8(to, u[j]);
            sts8(to + 8 * TK, u[j] >> 8);
            sts8(to + 16 * TK, u[j] >> 16);
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_pfull + 8 * group);
        if (CHUNKS == 1 && pending) take(0, reinterpret_cast<uint32_t(&)[24]>(x_o), table + ((mine - 1) % C::TABLES) * R * 8);
        pending = true;
      }
      if (pending) take_all();
      item += n_tiles;

      // ---- the groups' parts together
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) {
        float w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = (j & 1) ? high64(l[4 * c + j / 2]) : low64(l[4 * c + j / 2]);
        const float t = sum8(w, lane);
        if ((lane & 3) == 0) stat_l[quarter * R + 8 * c + sum8_row(lane)] = t;
      }
      if (quarter == 0 && lane < R) stat_a[lane] = top_a, stat_m[lane] = top_m;
      threads_meet<SOFT>();
      const bool whole = s.first == 0 && s.n_items == at.tiles;
      float* part = a.parts + ((long long)blockIdx.x * 2 + (s.first > 0 ? 0 : 1)) * C::PART_FLOATS;
      uint32_t lost = 0;
      for (int g = 0; g < GROUPS; ++g) lost |= broken[g];
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) {
        if (has_dim) {
#pragma unroll
          for (int j = 0; j < 8; ++j) join[(group * 8 + j) * D + dim] = (j & 1) ? high64(o[4 * c + j / 2]) : low64(o[4 * c + j / 2]);
        }
        threads_meet<SOFT>();
        for (int x = threadIdx.x; x < 8 * (D / 4); x += SOFT) {
          const int j = x / (D / 4), d = x % (D / 4) * 4, r = 8 * c + j;
          float ta = -INFINITY, tm = -INFINITY, sum_l = 0.0f;
          float4 sum = make_float4(0, 0, 0, 0);
          for (int g = 0; g < GROUPS; ++g) ta = fmaxf(ta, stat[g * R + r]), tm = fmaxf(tm, stat[GROUPS * R + g * R + r]);
          for (int g = 0; g < GROUPS; ++g) {
            const float4 v = *reinterpret_cast<const float4*>(join + (g * 8 + j) * D + d);
            const float f = stat[g * R + r] == -INFINITY ? 0.0f : ex2(stat[g * R + r] - ta) * (1.0f / W_ONE);
            sum.x += f * v.x, sum.y += f * v.y, sum.z += f * v.z, sum.w += f * v.w;
            const float* q = stat + 2 * GROUPS * R + g * 4 * R + r;
            const float lg = q[0] + q[R] + q[2 * R] + q[3 * R];
            sum_l += rebase(stat[GROUPS * R + g * R + r], lg, tm) * lg;
          }
          if ((lost >> r) & 1u) sum.x = sum.y = sum.z = sum.w = __uint_as_float(0x7FC00000u);
          if (whole) {
            const int i = s.qt * a.tq + r / a.Gc, hq = s.chunk * a.Gc + r % a.Gc;
            if (r < a.tq * a.Gc && i < at.n && hq < a.G) attn_store<D>(a, (long long)(at.row0 + i) * a.c.heads * a.G + s.h * a.G + hq, d, sum, sum_l, ta, tm);
          } else {
            __stcg(reinterpret_cast<float4*>(part + r * D + d), sum);
            if (d == 0) {
              __stcg(part + R * D + r, ta);
              __stcg(part + R * D + R + r, tm);
              __stcg(part + R * D + 2 * R + r, sum_l);
            }
          }
        }
        threads_meet<SOFT>();
      }
      if (!whole) attn_combine<D, R, SOFT, C::PART_FLOATS>(a, at, s.qt, s.h, s.chunk, begin + (end - begin - at.left) - s.first, per, misc + 7, join);
      if (threadIdx.x == 0) {
        for (int g = 0; g < GROUPS; ++g) broken[g] = 0;
        mbar_arrive(bar_qempty + 8 * buf);                                            // queries, factors and statistics of the unit are done with
      }
      threads_meet<SOFT>();
      if (!walk_advance(a, TK, at, s.n_items)) break;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == C::W_MMA) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)C::TMEM_COLS) : "memory");
}

// LIVE: rows of a row tile, R or half of 8: what is computed of a tile's scores and sums goes by it, the columns that the MMAs compute by R.
template <int D, int R, int LIVE = R>
int launch_as(AttnArgs& a, cudaStream_t st) {
  using C = FewCfg<D, R>;
  static_assert(C::SMEM_BYTES <= 232448, "shared memory of a CTA");
  a.Gc = a.G < LIVE ? a.G : LIVE;
  a.chunks = (a.G + a.Gc - 1) / a.Gc;
  a.tq = LIVE / a.Gc;
  CUtensorMap map_k, map_v;
  RAZER_TRY(attn_encode_pool(&map_k, a.c.k, a.c, a.c.page, D));
  RAZER_TRY(attn_encode_pool(&map_v, a.c.v, a.c, a.c.page, D));
  static std::atomic<uint64_t> allowed{0};
  RAZER_TRY(allow_smem((const void*)attn_kv8_few_kernel<D, R, LIVE>, C::SMEM_BYTES, allowed));
  return launch_dependent("attn_kv8_few_kernel launch", attn_kv8_few_kernel<D, R, LIVE>, sm_count() < ATTN_CTAS ? sm_count() : ATTN_CTAS, C::THREADS, C::SMEM_BYTES, st, map_k, map_v, a);
}

}  // namespace

size_t attn_few_part_floats(int D) { return D == 64 ? FewCfg<64, 32>::PART_FLOATS : FewCfg<128, 32>::PART_FLOATS; }

int launch_attn_few(AttnArgs& a, int rows, cudaStream_t st) {
  // Four rows at most (64 sequences of 4096 tokens, 8 x 4 heads): half of eight's work, heads of 64 79 us against 88, of 128 (32 sequences) 55 against 57.
  if (rows <= 4) return a.c.D == 64 ? launch_as<64, 8, 4>(a, st) : launch_as<128, 8, 4>(a, st);
  if (a.c.D == 64) return rows <= 8 ? launch_as<64, 8>(a, st) : rows <= 16 ? launch_as<64, 16>(a, st) : launch_as<64, 32>(a, st);
  return rows <= 8 ? launch_as<128, 8>(a, st) : rows <= 16 ? launch_as<128, 16>(a, st) : launch_as<128, 32>(a, st);
}

}  // namespace razer
