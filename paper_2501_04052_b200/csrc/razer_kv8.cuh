// The paged cache of 8-bit keys and values, as its writer and the attention over it see it.
//
// k, v: [pages][heads][page][head_dim] int8; k_scales, v_scales: [pages][heads] FP32, value = scale * code.  A sequence's tokens
// p = 0 .. kv_len - 1 lie in row p % page of page table[p / page].
#pragma once

#include <stdint.h>

namespace razer {

struct Kv8 {
  int8_t *k, *v;
  float *k_scales, *v_scales;
  int pages, page, page_log2, heads, D;
};

// A batch: sequence b's new tokens are rows q_start[b] .. q_start[b + 1] - 1, at its last positions.
struct Kv8Batch {
  const int* table;
  const int* q_start;
  const int* kv_len;
  int width, B, T;
};

// Sequence b's rows and length, made safe: rows inside 0 .. T, no negative counts.
struct Kv8Seq {
  int row0, n, len;
};
// Longer than its table.
__device__ __forceinline__ bool kv8_over(const Kv8& c, const Kv8Batch& s, int len) { return len > s.width << c.page_log2; }
__device__ __forceinline__ Kv8Seq kv8_seq(const Kv8Batch& s, int b) {
  Kv8Seq q;
  const int lo = s.q_start[b], hi = s.q_start[b + 1];
  q.len = max(s.kv_len[b], 0);
  const bool good = lo >= 0 && hi <= s.T && hi >= lo;
  q.row0 = good ? lo : 0;
  q.n = good ? hi - lo : 0;
  return q;
}

// The page of block c of sequence b, or -1 where the table is too narrow for it or names no page.
__device__ __forceinline__ int kv8_page(const Kv8& c, const Kv8Batch& s, int b, int block) {
  if (block >= s.width) return -1;
  const int p = s.table[(long long)b * s.width + block];
  return p >= 0 && p < c.pages ? p : -1;
}

}  // namespace razer
