// Attention over the paged 8-bit cache (razer_attn_kv8): which kernel takes a call.
#include "razer_attn_kv8.cuh"

namespace razer {

size_t attn_few_part_floats(int D);
int launch_attn_few(AttnArgs& a, int rows, cudaStream_t st);
size_t attn_many_part_floats(int D);
int launch_attn_many(AttnArgs& a, cudaStream_t st);

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
  const long long rows = ((long long)s.T + s.B - 1) / s.B * a.G;       // of a sequence and key-value head, in the mean
  static const int force = getenv("ATTN_MANY") ? atoi(getenv("ATTN_MANY")) : 33;   // XXX
  if (rows >= force) return launch_attn_many(a, st);
  return launch_attn_few(a, rows > 32 ? 32 : (int)rows, st);
}

}  // namespace razer
