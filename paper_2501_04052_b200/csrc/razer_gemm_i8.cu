// Matrix product in 8-bit integers for sm_100a (tcgen05 kind::i8 + TMEM + TMA):
//   y[m, n] = bf16( fl32(sx[m] sw[n]) * sum_k xq[m, k] wq[n, k] ),   xq [M][K], wq [N][K] int8, the sum exact in 32 bits.
//
// i8_split_kernel: a 128-row weight tile is the MMA's A operand and NT tokens its B operand, both K-major in shared memory in the 128-byte
// swizzle (a row of a stage = 128 codes), accumulated in TMEM as 32-bit integers.  Warp 0 feeds the ring by TMA, warp 1 issues the
// MMAs, warps 2-5 store.  One output tile belongs to a cluster of 1, 2, 4 or 8 CTAs that share its K: with few tokens there are fewer
// tiles than SMs, and every weight byte comes from HBM once whatever the split.  The parts meet in distributed shared memory - integers, so that their
// order does not matter - and each CTA finishes 128 / split of the rows: no workspace, no counters, nothing left between calls.
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
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_meet() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int peer_lds32(uint32_t addr, uint32_t rank) {
  int v;
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.s32 %0, [a];\n\t}" : "=r"(v) : "r"(addr), "r"(rank) : "memory");
  return v;
}

struct I8Args {
  __nv_bfloat16* y;
  const float *sx, *sw;
  int M, N;
  int token_tiles, chunks;     // chunks: stages of the whole K
};

template <int NT, int STAGES_>
struct I8Cfg {
  static constexpr int STAGES = STAGES_;
  static constexpr int B_BYTES = NT * I8_STAGE_K;
  static constexpr int STAGE_BYTES = I8_A_BYTES + B_BYTES;
  static constexpr int PART_BYTES = NT * TILE_ROWS * 4;                       // a CTA's sums, over the ring once that is done with
  static constexpr int RING_BYTES = STAGES * STAGE_BYTES > PART_BYTES ? STAGES * STAGE_BYTES : PART_BYTES;
  static constexpr int SMEM_BYTES = 1024 + RING_BYTES + 256;                  // alignment, barriers
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
  const bool any = c_end > c_begin;
  const int row = 32 * (warp & 3) + lane;
  if (split == 1) {
    if (warp >= 2) {
      if (!mbar_wait(bar_acc, 0, words + 2)) *abort_flag = 1;
      __syncwarp();
      tc_fence_after();
      const bool bad = *abort_flag;
      const int n = rt * TILE_ROWS + row, m0 = tt * NT, valid = min(NT, a.M - m0);
      const float sw = n < a.N ? a.sw[n] : 0.0f;
      __nv_bfloat16* dst = a.y + (size_t)m0 * a.N + n;
#pragma unroll 1
      for (int c = 0; c < NT; c += 16) {
        if (c >= valid) break;
        uint32_t v[16];
        tc_ld16(tmem + ((uint32_t)(32 * (warp & 3)) << 16) + c, v);
        tc_wait_ld();
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          if (c + j < valid && n < a.N) {
            const float r = bad ? __uint_as_float(0x7FC00000u) : (a.sx[m0 + c + j] * sw) * (float)(int)v[j];
            *dst = __float2bfloat16_rn(r);
          }
          dst += a.N;
        }
      }
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
          asm volatile("st.shared.u32 [%0], %1;" ::"r"(base + (uint32_t)((c + j) * TILE_ROWS + row) * 4), "r"(any ? v[j] : 0u) : "memory");
      }
      tc_fence_before();
    }
    __syncwarp();
    cluster_meet();
    if (warp >= 2) {
      const int rows = TILE_ROWS / split, t = threadIdx.x - 64;
      const int r = rank * rows + t % rows, n = rt * TILE_ROWS + r, m0 = tt * NT, valid = min(NT, a.M - m0);
      bool bad = false;
      for (int p = 0; p < split; ++p) bad |= peer_lds32(smem_u32(words + 1), p) != 0;
      if (n < a.N) {
        const float sw = a.sw[n];
        for (int m = t / rows; m < valid; m += split) {
          int sum = 0;
          for (int p = 0; p < split; ++p) sum += peer_lds32(base + (uint32_t)(m * TILE_ROWS + r) * 4, p);
          const float v = bad ? __uint_as_float(0x7FC00000u) : (a.sx[m0 + m] * sw) * (float)sum;
          a.y[(size_t)(m0 + m) * a.N + n] = __float2bfloat16_rn(v);
        }
      }
    }
    __syncwarp();
    cluster_meet();                                         // nobody leaves while another reads its sums
  }
  tc_fence_after();
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)C::TMEM_COLS) : "memory");
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

}  // namespace

int launch_gemm_i8(const int8_t* x, const float* sx, const int8_t* w, const float* sw, int M, int N, int K, void* y, cudaStream_t st) {
  I8Args a;
  a.y = (__nv_bfloat16*)y;
  a.sx = sx;
  a.sw = sw;
  a.M = M;
  a.N = N;
  a.chunks = (K + I8_STAGE_K - 1) / I8_STAGE_K;
  const int nt = M <= 16 ? 16 : M <= 32 ? 32 : M <= 64 ? 64 : M <= 128 ? 128 : 256;
  a.token_tiles = (M + nt - 1) / nt;
  const long long tiles = (long long)((N + TILE_ROWS - 1) / TILE_ROWS) * a.token_tiles;
  const int sms = sm_count(), ctas = nt <= 64 ? 2 : 1;
  int split = 1;
  while (split < 8 && tiles * split * 2 <= (long long)sms * ctas && a.chunks >= 4 * split) split *= 2;
  switch (nt) {
    case 16: return launch_split<16, 6, 2>(x, w, a, K, split, st);
    case 32: return launch_split<32, 5, 2>(x, w, a, K, split, st);
    case 64: return launch_split<64, 4, 2>(x, w, a, K, split, st);
    case 128: return launch_split<128, 6, 1>(x, w, a, K, split, st);
    default: return launch_split<256, 4, 1>(x, w, a, K, split, st);
  }
}

}  // namespace razer
