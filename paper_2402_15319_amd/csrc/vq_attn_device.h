// Device-side helpers of attention over the paged cache.
#pragma once
#include "vq_attn.h"

namespace vq {

// A value of the cache's type, and back with one rounding to nearest even.
template <bool BF16> __device__ __forceinline__ float to_f32(uint16_t u) {
  if constexpr (BF16) return __builtin_bit_cast(float, (uint32_t)u << 16);
  else return (float)__builtin_bit_cast(_Float16, u);
}
template <bool BF16> __device__ __forceinline__ uint16_t from_f32(float f) {
  if constexpr (BF16) return __builtin_bit_cast(uint16_t, (__bf16)f);
  else return __builtin_bit_cast(uint16_t, (_Float16)f);
}

// The sequence that owns new token t: the last one that starts at or before it.
__device__ __forceinline__ int sequence_of(const CacheArgs& c, int t) {
  if (!c.q_start) return t;
  int lo = 0, hi = c.n_seqs;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (c.q_start[mid] <= t) lo = mid; else hi = mid;
  }
  return lo;
}

// Tokens in the cache of sequence s: what the table can list at most.
__device__ __forceinline__ int cached_tokens(const CacheArgs& c, int s) {
  const int n = c.kv_len[s];
  return n < 0 ? 0 : n < c.max_len ? n : c.max_len;
}

// The rows [*first, *last) of sequence s, inside the arrays whatever q_start holds.
__device__ __forceinline__ void rows_of(const CacheArgs& c, int s, int* first, int* last) {
  int a = c.q_start ? c.q_start[s] : s, b = c.q_start ? c.q_start[s + 1] : s + 1;
  a = a < 0 ? 0 : a < c.n_tokens ? a : c.n_tokens;
  b = b < a ? a : b < c.n_tokens ? b : c.n_tokens;
  *first = a;
  *last = b;
}

// Page number j of sequence s, moved into the cache where the table holds another.
__device__ __forceinline__ int page_inside(const CacheArgs& c, int s, int j) {
  const uint32_t p = (uint32_t)c.table[(int64_t)s * c.table_width + j];
  return (int)(p < (uint32_t)c.n_pages ? p : (uint32_t)c.n_pages - 1);
}

}  // namespace vq
