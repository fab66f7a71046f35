// Matrix product in 8-bit integers for sm_100a (tcgen05 kind::i8 + TMEM + TMA):
//   y[m, n] = bf16( fl32(sx[m] sw[n]) * sum_k xq[m, k] wq[n, k] ),   xq [M][K], wq [N][K] int8, the sum exact in 32 bits.
//
// i8_split_kernel: a 128-row weight tile is the MMA's A operand and NT tokens its B operand, both K-major in shared memory in the 128-byte
// swizzle (a row of a stage = 128 codes), accumulated in TMEM as 32-bit integers.  Warp 0 feeds the ring by TMA, warp 1 issues the
// MMAs, warps 2-5 store.  One output tile belongs to a cluster of 1, 2, 4 or 8 CTAs that share its K: with few tokens there are fewer
// tiles than SMs, and every weight byte comes from HBM once whatever the split.  The parts meet in distributed shared memory - integers, so that their
// order does not matter - and each CTA finishes 128 / split of the rows: no workspace, no counters, nothing left between calls.
//
// i8_pair_kernel: two CTAs on 256 weight rows x up to 256 tokens, where the cost model below finds it faster (from 33 tokens on; narrow products of some hundred tokens
// stay with the other).
//
// What bounds them, in a graph (a host loop in brackets, where the power limit lowers the clock): 1 x 11008 x 4096 10.2 us (11.0), 16 x 28672 x 8192 38.8 (40.1,
// 5.9 TB/s): the weights from HBM, and the launch; 333 x 4096 x 11008 17 (21): 64 pairs of CTAs that take in 1.9 MB a CTA at 150 GB/s;
// 2048 x 14336 x 4096 80 (99, 2.4 POP/s): the MMAs, under the power limit.
#include "razer_common.cuh"
#include "razer_tcgen05.cuh"

namespace razer {

namespace {

constexpr int I8_STAGE_K = 128;                    // codes of a row in a stage: one 128-byte swizzle row
constexpr int I8_A_BYTES = TILE_ROWS * I8_STAGE_K;

// Shared-memory descriptor, upper half (K-major, 128-byte swizzle: 1024 bytes from one group of eight rows to the next)
constexpr uint32_t I8_DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);
// D = S32, A and B = signed 8-bit, both K-major
__host__ __device__ constexpr uint32_t i8_idesc(int m, int n) {
  return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ uint32_t i8_desc_lo(uint32_t addr) { return (addr >> 4) | (1u << 16); }

__device__ __forceinline__ void mma_i8(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 ad, bd;\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "mov.b64 ad, {%1, %3};\n\t"
      "mov.b64 bd, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::i8 [%0], ad, bd, %4, p;\n\t}" ::"r"(d_tmem),
      "r"(a_lo), "r"(b_lo), "r"(I8_DESC_HI), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ int4 peer_lds128(uint32_t addr, uint32_t rank) {
  int4 v;
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %4, %5;\n\tld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [a];\n\t}"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(addr), "r"(rank)
               : "memory");
  return v;
}
__device__ __forceinline__ int peer_lds32(uint32_t addr, uint32_t rank) {
  int v;
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.s32 %0, [a];\n\t}" : "=r"(v) : "r"(addr), "r"(rank) : "memory");
  return v;
}

// Sixteen columns (tokens) of a row: sums from TMEM, scaled, rounded, stored.  sx: the columns' scales in shared memory (loaded one by one from global
// memory between the stores they cost 2 us for 16 columns); `count` of the columns are tokens, `live` says whether the row is one.
__device__ __forceinline__ void store_columns(uint32_t taddr, const float* sx, float sw, bool bad, __nv_bfloat16* dst, int N, int count, bool live) {
  uint32_t v[16];
  tc_ld16(taddr, v);
  float f[16];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float4 q = reinterpret_cast<const float4*>(sx)[j];
    f[4 * j] = q.x, f[4 * j + 1] = q.y, f[4 * j + 2] = q.z, f[4 * j + 3] = q.w;
  }
  tc_wait_ld();
  __nv_bfloat16 o[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) o[j] = __float2bfloat16_rn(bad ? __uint_as_float(0x7FC00000u) : (f[j] * sw) * (float)(int)v[j]);
  if (!live) return;
  if (count >= 16) {
#pragma unroll
    for (int j = 0; j < 16; ++j) dst[(size_t)j * N] = o[j];
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if (j < count) dst[(size_t)j * N] = o[j];
  }
}

template <int N>
__device__ __forceinline__ void threads_meet() { asm volatile("bar.sync 1, %0;" ::"n"(N) : "memory"); }

struct I8Args {
  __nv_bfloat16* y;
  const float *sx, *sw;
  int M, N;
  int token_tiles, chunks;     // chunks: stages of the whole K
};

// The sums of a cluster's CTAs over K, [token][128 rows] at `part` of each: CTA `mine` of the `split` adds up and
// stores 128 / split of the rows, four rows a thread (16 bytes of sums, 8 of results), four tokens in flight.
template <int THREADS>
__device__ __forceinline__ void add_parts(const I8Args& a, uint32_t part, int n_tile, int m_tile, int valid, int split, int mine, int t, bool bad) {
  const int quads = TILE_ROWS / 4 / split, r = 4 * (mine * quads + t % quads), n = n_tile + r, step = THREADS / quads;
  if (n >= a.N) return;
  const bool wide = n + 4 <= a.N && a.N % 4 == 0 && (reinterpret_cast<uintptr_t>(a.y) & 7) == 0;
  float sw[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) sw[i] = n + i < a.N ? a.sw[n + i] : 0.0f;
  for (int m0 = t / quads; m0 < valid; m0 += 4 * step) {
    int4 sum[4];
    float sx[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      sum[u] = make_int4(0, 0, 0, 0);
      sx[u] = m0 + u * step < valid ? a.sx[m_tile + m0 + u * step] : 0.0f;
    }
    for (int p = 0; p < split; p += 2) {
      int4 v[2][4];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int u = 0; u < 4; ++u) v[h][u] = peer_lds128(part + (uint32_t)(min(m0 + u * step, valid - 1) * TILE_ROWS + r) * 4, p + h);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int u = 0; u < 4; ++u) sum[u].x += v[h][u].x, sum[u].y += v[h][u].y, sum[u].z += v[h][u].z, sum[u].w += v[h][u].w;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int m = m0 + u * step;
      if (m >= valid) break;
      const int v[4] = {sum[u].x, sum[u].y, sum[u].z, sum[u].w};
      __align__(8) __nv_bfloat16 o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = __float2bfloat16_rn(bad ? __uint_as_float(0x7FC00000u) : (sx[u] * sw[i]) * (float)v[i]);
      __nv_bfloat16* dst = a.y + (size_t)(m_tile + m) * a.N + n;
      if (wide) {
        *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(o);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (n + i < a.N) dst[i] = o[i];
      }
    }
  }
}

template <int NT, int STAGES_>
struct I8Cfg {
  static constexpr int STAGES = STAGES_;
  static constexpr int B_BYTES = NT * I8_STAGE_K;
  static constexpr int STAGE_BYTES = I8_A_BYTES + B_BYTES;
  static constexpr int PART_BYTES = NT * TILE_ROWS * 4;                       // a CTA's sums, over the ring once that is done with
  static constexpr int RING_BYTES = STAGES * STAGE_BYTES > PART_BYTES ? STAGES * STAGE_BYTES : PART_BYTES;
  static constexpr int SMEM_BYTES = 1024 + RING_BYTES + 256 + NT * 4;         // alignment, barriers, scales of the tokens
  static constexpr int TMEM_COLS = NT < 32 ? 32 : NT;
  static constexpr int THREADS = 192;
};

template <int NT, int STAGES, int CTAS>
__global__ void __launch_bounds__(192, CTAS) i8_split_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x,
                                                             const __grid_constant__ I8Args a, int split) {
  using C = I8Cfg<NT, STAGES>;
  extern __shared__ uint8_t i8_smem[];
  const uint32_t base = (smem_u32(i8_smem) + 1023) & ~1023u;
  const uint32_t bars = base + C::RING_BYTES;
  const uint32_t bar_full = bars, bar_empty = bars + 8 * STAGES, bar_acc = bars + 16 * STAGES;
  uint32_t* words = reinterpret_cast<uint32_t*>(i8_smem + (bars - smem_u32(i8_smem)) + 16 * STAGES + 8);
  uint32_t* tmem_slot = words;
  volatile uint32_t* abort_flag = words + 1;       // words + 2: a flag that nobody sets (drain waits)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = split > 1 ? (int)cluster_rank() : 0;
  const int tile = blockIdx.x / split, rt = tile / a.token_tiles, tt = tile - rt * a.token_tiles;
  // never empty: K is split only where every part has two stages
  const int c_begin = (int)((long long)a.chunks * rank / split), c_end = (int)((long long)a.chunks * (rank + 1) / split);

  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(bar_full + 8 * i, 1);
      mbar_init(bar_empty + 8 * i, 1);
    }
    mbar_init(bar_acc, 1);
    words[1] = words[2] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_w) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_x) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"((uint32_t)C::TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  grid_dep_wait();
  grid_dep_launch();

  if (warp == 0) {
    if (elect_one()) {
      int slot = 0, issued = 0;
      uint32_t phase = 0;
      for (int c = c_begin; c < c_end; ++c, ++issued) {
        if (issued >= STAGES && !mbar_wait(bar_empty + 8 * slot, phase ^ 1u, abort_flag)) { *abort_flag = 1; break; }
        const uint32_t st = base + slot * C::STAGE_BYTES, bar = bar_full + 8 * slot;
        mbar_expect_tx(bar, (uint32_t)C::STAGE_BYTES);      // boxes are zero-filled past N, M and K: always whole
        tma_load_2d(st, &tmap_w, c * I8_STAGE_K, rt * TILE_ROWS, bar);
        tma_load_2d(st + I8_A_BYTES, &tmap_x, c * I8_STAGE_K, tt * NT, bar);
        if (++slot == STAGES) { slot = 0; phase ^= 1u; }
      }
      // copies still in flight must land before this CTA's shared memory is used anew or released
      for (int f = issued > STAGES ? issued - STAGES : 0; f < issued; ++f)
        mbar_wait(bar_full + 8 * (f % STAGES), (uint32_t)((f / STAGES) & 1), words + 2);
    }
  } else if (warp == 1) {
    if (elect_one()) {
      int slot = 0;
      uint32_t phase = 0;
      for (int c = c_begin; c < c_end; ++c) {
        if (!mbar_wait(bar_full + 8 * slot, phase, abort_flag)) { *abort_flag = 1; break; }
        tc_fence_after();
        const uint32_t al = i8_desc_lo(base + slot * C::STAGE_BYTES), bl = i8_desc_lo(base + slot * C::STAGE_BYTES + I8_A_BYTES);
#pragma unroll
        for (int k = 0; k < I8_STAGE_K / 32; ++k) mma_i8(tmem, al + 2 * k, bl + 2 * k, i8_idesc(128, NT), (c > c_begin || k > 0) ? 1u : 0u);
        tc_commit(bar_empty + 8 * slot);
        if (++slot == STAGES) { slot = 0; phase ^= 1u; }
      }
      tc_commit(bar_acc);                                   // after a failure too: what was issued is then waited for
    }
    __syncwarp();
    mbar_wait(bar_acc, 0, words + 2);
    __syncwarp();
  }
  float* scales = reinterpret_cast<float*>(i8_smem + (bars + 256 - smem_u32(i8_smem)));
  const int row = 32 * (warp & 3) + lane;
  if (split == 1) {
    if (warp >= 2) {
      for (int i = threadIdx.x - 64; i < NT; i += 128) scales[i] = tt * NT + i < a.M ? a.sx[tt * NT + i] : 0.0f;
      threads_meet<128>();
      if (!mbar_wait(bar_acc, 0, words + 2)) *abort_flag = 1;
      __syncwarp();
      tc_fence_after();
      const bool bad = *abort_flag;
      const int n = rt * TILE_ROWS + row, m0 = tt * NT, valid = min(NT, a.M - m0);
      const float sw = n < a.N ? a.sw[n] : 0.0f;
      __nv_bfloat16* dst = a.y + (size_t)m0 * a.N + n;
#pragma unroll 1
      for (int c = 0; c < valid; c += 16)
        store_columns(tmem + ((uint32_t)(32 * (warp & 3)) << 16) + c, scales + c, sw, bad, dst + (size_t)c * a.N, a.N, valid - c, n < a.N);
      tc_fence_before();
    }
    __syncthreads();
  } else {
    __syncthreads();                                        // the ring is done with: copies have landed, MMAs have read them
    if (warp >= 2) {
      if (!mbar_wait(bar_acc, 0, words + 2)) *abort_flag = 1;
      __syncwarp();
      tc_fence_after();
#pragma unroll 1
      for (int c = 0; c < NT; c += 16) {
        if (c >= a.M - tt * NT) break;
        uint32_t v[16];
        tc_ld16(tmem + ((uint32_t)(32 * (warp & 3)) << 16) + c, v);
        tc_wait_ld();
#pragma unroll
        for (int j = 0; j < 16; ++j)
          asm volatile("st.shared.u32 [%0], %1;" ::"r"(base + (uint32_t)((c + j) * TILE_ROWS + row) * 4), "r"(v[j]) : "memory");
      }
      tc_fence_before();
    }
    __syncwarp();
    cluster_meet();
    if (warp >= 2) {
      bool bad = false;
      for (int p = 0; p < split; ++p) bad |= peer_lds32(smem_u32(words + 1), p) != 0;
      add_parts<128>(a, base, rt * TILE_ROWS, tt * NT, min(NT, a.M - tt * NT), split, rank, threadIdx.x - 64, bad);
    }
    __syncwarp();
    cluster_meet();                                         // nobody leaves while another reads its sums
  }
  tc_fence_after();
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)C::TMEM_COLS) : "memory");
}

// ------------------------------------------------------------------ two CTAs on one tile
__device__ __forceinline__ void mma_i8_pair(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 ad, bd;\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "mov.b64 ad, {%1, %3};\n\t"
      "mov.b64 bd, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::2.kind::i8 [%0], ad, bd, %4, p;\n\t}" ::"r"(d_tmem),
      "r"(a_lo), "r"(b_lo), "r"(I8_DESC_HI), "r"(idesc), "r"(accumulate)
      : "memory");
}
// A box into this CTA's shared memory whose bytes are counted by a barrier of the pair's first CTA.
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(bar)
      : "memory");
}

template <int NT>
struct PairCfg {
  static constexpr int B_BYTES = NT / 2 * I8_STAGE_K;                          // a CTA's half of the tokens
  static constexpr int STAGE_BYTES = I8_A_BYTES + B_BYTES;
  static constexpr int STAGES = 200 * 1024 / STAGE_BYTES;
  static constexpr int ACC_COLS = NT <= 64 ? 64 : NT <= 128 ? 128 : 256;       // of one of two accumulators
  static constexpr int TMEM_COLS = 2 * ACC_COLS;
  static constexpr int SMEM_BYTES = 1024 + STAGES * STAGE_BYTES + 256 + 2 * NT * 4;
  static constexpr int THREADS = 320;
};

// 256 weight rows x NT tokens by two CTAs (cta_group::2): each holds 128 of the rows and half of the tokens, so that an operand byte in shared
// memory serves twice the multiplications (a CTA alone would write and read 192 bytes a cycle at 128 x 256, beyond the 128 there are).
// Persistent, two accumulators in TMEM: the epilogue of a tile runs under the next one's MMAs.  The first CTA of the pair issues.
template <int NT>
__global__ void __launch_bounds__(320, 1) i8_pair_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x,
                                                         const __grid_constant__ I8Args a, int tiles) {
  using C = PairCfg<NT>;
  constexpr int STAGES = C::STAGES;
  extern __shared__ uint8_t i8_smem[];
  const uint32_t base = (smem_u32(i8_smem) + 1023) & ~1023u;
  const uint32_t bars = base + STAGES * C::STAGE_BYTES;
  const uint32_t bar_full = bars, bar_empty = bars + 8 * STAGES, bar_accfull = bars + 16 * STAGES, bar_accempty = bar_accfull + 16, bar_drain = bar_accempty + 16;
  uint32_t* words = reinterpret_cast<uint32_t*>(i8_smem + (bar_drain + 8 - smem_u32(i8_smem)));
  uint32_t* tmem_slot = words;
  volatile uint32_t* abort_flag = words + 1;       // words + 2: a flag that nobody sets (drain waits)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float* scales = reinterpret_cast<float*>(i8_smem + (bars + 256 - smem_u32(i8_smem)));
  const int rank = (int)cluster_rank(), pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(bar_full + 8 * i, 1);
      mbar_init(bar_empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_accfull + 8 * i, 1);
      mbar_init(bar_accempty + 8 * i, 16);         // eight epilogue warps of each CTA
    }
    mbar_init(bar_drain, 1);
    words[1] = words[2] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_w) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_x) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"((uint32_t)C::TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  __syncwarp();
  cluster_meet();                                  // both CTAs' barriers are ready
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  grid_dep_wait();
  grid_dep_launch();

  if (warp == 0) {
    if (elect_one()) {
      int slot = 0, issued = 0;
      uint32_t phase = 0;
      bool alive = true;
      const uint32_t full0 = peer_addr(bar_full, 0);
      for (int tile = pair; alive && tile < tiles; tile += pairs) {
        const int rt = tile / a.token_tiles, tt = tile - rt * a.token_tiles;
        for (int c = 0; c < a.chunks; ++c, ++issued) {
          if (issued >= STAGES && !mbar_wait(bar_empty + 8 * slot, phase ^ 1u, abort_flag)) { *abort_flag = 1; alive = false; break; }
          const uint32_t st = base + slot * C::STAGE_BYTES;
          if (rank == 0) mbar_expect_tx(bar_full + 8 * slot, 2u * C::STAGE_BYTES);
          tma_load_pair(st, &tmap_w, c * I8_STAGE_K, rt * 256 + rank * 128, full0 + 8 * slot);
          tma_load_pair(st + I8_A_BYTES, &tmap_x, c * I8_STAGE_K, tt * NT + rank * (NT / 2), full0 + 8 * slot);
          if (++slot == STAGES) { slot = 0; phase ^= 1u; }
        }
      }
      // Copies in flight must land before shared memory is released: the first CTA's barriers count both CTAs' copies, and the pair parts together.
      if (rank == 0)
        for (int f = issued > STAGES ? issued - STAGES : 0; f < issued; ++f)
          mbar_wait(bar_full + 8 * (f % STAGES), (uint32_t)((f / STAGES) & 1), words + 2);
    }
  } else if (warp == 1 && rank == 0) {
    if (elect_one()) {
      int slot = 0, turn = 0;
      uint32_t phase = 0;
      bool alive = true;
      for (int tile = pair; alive && tile < tiles; tile += pairs, ++turn) {
        const int acc = turn & 1;
        if (turn >= 2 && !mbar_wait(bar_accempty + 8 * acc, (uint32_t)(turn >> 1 & 1) ^ 1u, abort_flag)) { *abort_flag = 1; break; }
        tc_fence_after();
        const uint32_t d = tmem + acc * C::ACC_COLS;
        for (int c = 0; c < a.chunks; ++c) {
          if (!mbar_wait(bar_full + 8 * slot, phase, abort_flag)) { *abort_flag = 1; alive = false; break; }
          tc_fence_after();
          const uint32_t al = i8_desc_lo(base + slot * C::STAGE_BYTES), bl = i8_desc_lo(base + slot * C::STAGE_BYTES + I8_A_BYTES);
#pragma unroll
          for (int k = 0; k < I8_STAGE_K / 32; ++k) mma_i8_pair(d, al + 2 * k, bl + 2 * k, i8_idesc(256, NT), (c > 0 || k > 0) ? 1u : 0u);
          commit_pair(bar_empty + 8 * slot, 3u);
          if (++slot == STAGES) { slot = 0; phase ^= 1u; }
        }
        if (alive) commit_pair(bar_accfull + 8 * acc, 3u);
      }
      commit_pair(bar_drain, 1u);
    }
    __syncwarp();
    mbar_wait(bar_drain, 0, words + 2);
    __syncwarp();
  } else if (warp >= 2) {
    const int row = 32 * (warp & 3) + lane;
    const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
    const uint32_t empty0 = peer_addr(bar_accempty, 0);
    int turn = 0;
    for (int tile = pair; tile < tiles; tile += pairs, ++turn) {
      const int rt = tile / a.token_tiles, tt = tile - rt * a.token_tiles, acc = turn & 1;
      const int n = rt * 256 + rank * 128 + row, m0 = tt * NT, valid = min(NT, a.M - m0);
      float* sx = scales + acc * NT;                        // of two, so that one meeting a tile is enough
      for (int i = threadIdx.x - 64; i < NT; i += 256) sx[i] = m0 + i < a.M ? a.sx[m0 + i] : 0.0f;
      const float sw = n < a.N ? a.sw[n] : 0.0f;
      threads_meet<256>();
      if (!mbar_wait(bar_accfull + 8 * acc, (uint32_t)(turn >> 1 & 1), abort_flag)) *abort_flag = 1;
      const bool bad = __any_sync(0xFFFFFFFFu, *abort_flag != 0);
      tc_fence_after();
      __nv_bfloat16* dst = a.y + (size_t)m0 * a.N + n;
#pragma unroll 1
      for (int c = 16 * ((warp - 2) >> 2); c < valid; c += 32)       // two warps to a quarter of the rows take the columns in turn
        store_columns(tmem + lanes + acc * C::ACC_COLS + c, sx + c, sw, bad, dst + (size_t)c * a.N, a.N, valid - c, n < a.N);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) peer_arrive(empty0 + 8 * acc);
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  __syncwarp();
  cluster_meet();                                  // the other CTA may still read this one's operands or arrive at its barriers
  tc_fence_after();
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)C::TMEM_COLS) : "memory");
}

int encode_codes(CUtensorMap* map, const void* p, int rows, int K, int box_rows) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return set_error(RAZER_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
  const cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)K};
  const cuuint32_t box[2] = {(cuuint32_t)I8_STAGE_K, (cuuint32_t)box_rows};
  const cuuint32_t estr[2] = {1, 1};
  const CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return set_error(RAZER_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d", (int)r);
  return RAZER_OK;
}

template <int NT, int STAGES, int CTAS>
int launch_split(const int8_t* x, const int8_t* w, const I8Args& a, int K, int split, cudaStream_t st) {
  using C = I8Cfg<NT, STAGES>;
  CUtensorMap tmap_w, tmap_x;
  RAZER_TRY(encode_codes(&tmap_w, w, a.N, K, TILE_ROWS));
  RAZER_TRY(encode_codes(&tmap_x, x, a.M, K, NT));
  static std::atomic<uint64_t> allowed{0};
  RAZER_TRY(allow_smem((const void*)i8_split_kernel<NT, STAGES, CTAS>, C::SMEM_BYTES, allowed));
  const long long tiles = (long long)((a.N + TILE_ROWS - 1) / TILE_ROWS) * a.token_tiles;
  if (tiles * split > 0x7FFFFFFFll) return set_error(RAZER_ERR_UNSUPPORTED, "M=%d N=%d: more tiles than a launch has", a.M, a.N);
  return launch_dependent_clusters("i8_split_kernel launch", i8_split_kernel<NT, STAGES, CTAS>, dim3((unsigned)(tiles * split)), split, C::THREADS,
                                   C::SMEM_BYTES, st, tmap_w, tmap_x, a, split);
}

template <int NT>
int launch_pair(const int8_t* x, const int8_t* w, const I8Args& a, int K, cudaStream_t st) {
  using C = PairCfg<NT>;
  static_assert(C::SMEM_BYTES <= 232448, "shared memory of a CTA");
  CUtensorMap tmap_w, tmap_x;
  RAZER_TRY(encode_codes(&tmap_w, w, a.N, K, 128));
  RAZER_TRY(encode_codes(&tmap_x, x, a.M, K, NT / 2));
  static std::atomic<uint64_t> allowed{0};
  RAZER_TRY(allow_smem((const void*)i8_pair_kernel<NT>, C::SMEM_BYTES, allowed));
  const long long tiles = (long long)((a.N + 255) / 256) * a.token_tiles, pairs = sm_count() / 2;
  if (tiles > 0x7FFFFFFFll) return set_error(RAZER_ERR_UNSUPPORTED, "M=%d N=%d: too many tiles", a.M, a.N);
  return launch_dependent_clusters("i8_pair_kernel launch", i8_pair_kernel<NT>, dim3((unsigned)(2 * (tiles < pairs ? tiles : pairs))), 2, C::THREADS,
                                   C::SMEM_BYTES, st, tmap_w, tmap_x, a, (int)tiles);
}

// Which kernel, how many tokens a tile, how many CTAs on a tile's K: the least of what the candidates are modelled to take, in microseconds, from
// sweeps over sizes (M 1 .. 2048, N and K 1024 .. 28672, weights from HBM, launches in a graph).  A launch takes 2.8 (split) or 3.6 (pairs) with its
// first loads; an SM takes in at most 175 GB/s with one CTA's 64-byte-a-cycle ring (150 beside the MMAs of a pair), all together
// 19 TB/s out of L2, and the weights come at 6.3 TB/s from HBM; the MMAs of a stage of a pair take 1.07 ns a token, 1.3 where they go on for
// several tiles and the clock gives way; the end of a tile 8 ns a token.  A cluster's meetings cost 1.1.  Measured, both kernels at their best: 128 x 4096 x 4096 9.9 (split) and 7.9 (pairs), 256 x 8192 x
// 8192 25 and 18.5, 64 x 8192 x 8192 14.6 and 16.2, 1 x 1024 x 8192 5.4 with K split eight ways and 9.2 without.
struct I8Plan {
  bool pair;
  int nt, split;
};
I8Plan i8_plan(int M, int N, int K) {
  const int chunks = (K + I8_STAGE_K - 1) / I8_STAGE_K, sms = sm_count();
  const float hbm = (float)N * K / 6.3e6f;
  I8Plan best = {false, 16, 1};
  float least = 0.0f;
  auto consider = [&](bool pair, int nt, int split, float us) {
    if (least == 0.0f || us < least) least = us, best = {pair, nt, split};
  };
  {
    const int nt = M <= 16 ? 16 : M <= 32 ? 32 : 64;
    const long long tiles = (long long)((N + 127) / 128) * ((M + nt - 1) / nt);
    const float stage = I8_A_BYTES + nt * 128.0f;
    for (int split = 1; split <= 8 && (split == 1 || (tiles * split <= sms && chunks >= 2 * split)); split *= 2) {
      const float ctas = (float)(tiles * split), waves = tiles <= sms ? 1.0f : (float)((tiles + 2 * sms - 1) / (2 * sms));
      const float at_once = ctas < 2.0f * sms ? ctas : 2.0f * sms;
      const float chunk = fmaxf(stage / 175e3f * (tiles > sms ? 2.0f : 1.0f), at_once * stage / 19e6f);
      consider(false, nt, split, 2.8f + 0.008f * nt + (split > 1 ? 1.1f + 0.02f * nt : 0.0f) + fmaxf(hbm, waves * (float)((chunks + split - 1) / split) * chunk));
    }
  }
  for (int nt = 64; M > 32 && nt <= 256; nt += 32) {
    const long long tiles = (long long)((N + 255) / 256) * ((M + nt - 1) / nt), pairs = sms / 2;
    const float stage = I8_A_BYTES + nt * 64.0f;
    auto pace = [&](float ctas) { return fmaxf((tiles > pairs ? 1.3e-3f : 1.07e-3f) * nt, fmaxf(stage / 150e3f, ctas * stage / 19e6f)); };
    const float rest = (float)(tiles % pairs);
    const float us = 3.6f + 0.008f * nt + fmaxf(hbm, chunks * ((float)(tiles / pairs) * pace((float)sms) + (rest > 0.0f ? pace(2.0f * rest) : 0.0f)));
    consider(true, nt, 1, us);
  }
  return best;
}

}  // namespace

int launch_gemm_i8(const int8_t* x, const float* sx, const int8_t* w, const float* sw, int M, int N, int K, void* y, cudaStream_t st) {
  I8Args a;
  a.y = (__nv_bfloat16*)y;
  a.sx = sx;
  a.sw = sw;
  a.M = M;
  a.N = N;
  a.chunks = (K + I8_STAGE_K - 1) / I8_STAGE_K;
  const I8Plan p = i8_plan(M, N, K);
  a.token_tiles = (M + p.nt - 1) / p.nt;
  if (p.pair) {
    switch (p.nt) {
      case 64: return launch_pair<64>(x, w, a, K, st);
      case 96: return launch_pair<96>(x, w, a, K, st);
      case 128: return launch_pair<128>(x, w, a, K, st);
      case 160: return launch_pair<160>(x, w, a, K, st);
      case 192: return launch_pair<192>(x, w, a, K, st);
      case 224: return launch_pair<224>(x, w, a, K, st);
      default: return launch_pair<256>(x, w, a, K, st);
    }
  }
  // As many stages as an SM holds for one CTA to each, half of them where there are more CTAs than SMs (1 x 4096 x 11008 12.7 us against 17.9 with
  // the short ring; 16 x 28672 x 8192, 224 tiles, 39.6 against 38.9).
  const long long ctas = (long long)((N + TILE_ROWS - 1) / TILE_ROWS) * a.token_tiles * p.split;
  const bool deep = ctas <= sm_count();
  switch (p.nt) {
    case 16: return deep ? launch_split<16, 12, 1>(x, w, a, K, p.split, st) : launch_split<16, 6, 2>(x, w, a, K, p.split, st);
    case 32: return deep ? launch_split<32, 11, 1>(x, w, a, K, p.split, st) : launch_split<32, 5, 2>(x, w, a, K, p.split, st);
    default: return deep ? launch_split<64, 9, 1>(x, w, a, K, p.split, st) : launch_split<64, 4, 2>(x, w, a, K, p.split, st);
  }
}

}  // namespace razer
