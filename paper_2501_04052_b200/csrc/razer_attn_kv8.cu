// Attention over the paged 8-bit cache (razer_attn_kv8): which kernel takes a call.
#include "razer_attn_kv8.cuh"

namespace razer {

size_t attn_few_part_floats(int D);
int launch_attn_few(AttnArgs& a, int rows, cudaStream_t st);
size_t attn_many_part_floats(int D);
int launch_attn_many(AttnArgs& a, bool pairs, cudaStream_t st);

size_t attn_kv8_workspace_bytes(int D) {
  const size_t few = attn_few_part_floats(D), many = attn_many_part_floats(D);
  return WS_ZERO_BYTES + (size_t)sm_count() * 2 * (few > many ? few : many) * sizeof(float);
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
  // By the rows of queries that a sequence has for a key-value head, in the mean (which ones the device alone knows; either kernel takes any).  8 key-value
  // heads x 8, 32 sequences of 4096 tokens, pages of 64, microseconds with few / many rows: 8 rows 54 / 193, 16 78 / 196, 32 121 / 199,
  // 48 217 / 200 (the tile of 32 taken twice), 128 408 / 202.  Pairs of CTAs
  // (heads of 128) from 1024 rows on where a row tile of 512 is at most 128 tokens, so that the causal mask wastes little of it, many rows / pairs: 3 ragged
  // sequences of 8192 with 4 x 1000 rows 373 / 355, 8192 rows over 32768 tokens 1231 / 1081, 2400 rows over 4000 87 / 83, 1024 over 8192 82 / 80; 512 over
  // 8192 70 / 72, 510 over 4096 73 / 81, 2048 tokens among themselves with one query head 109 / 119.  RAZER_ATTN (environment, read once; a test aid): "few",
  // "many" or "pair" takes that one.
  static const char force = [] { const char* e = getenv("RAZER_ATTN"); return e ? e[0] : '\0'; }();
  const long long rows = ((long long)s.T + s.B - 1) / s.B * a.G;
  if (force ? force != 'f' : rows > 32) return launch_attn_many(a, force ? force == 'p' : rows >= 1024 && a.G >= 4, st);
  return launch_attn_few(a, rows > 32 ? 32 : (int)rows, st);
}

}  // namespace razer
