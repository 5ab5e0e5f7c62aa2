// Attention over the paged cache: what the host code (vq_attn_api.hip) hands to the kernels, and the
// launchers of vq_cache.hip, vq_attn_decode.hip and vq_attn_prompt.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/vq.h"

namespace vq {

// The sequences of a launch (include/vq.h: vq_attn_batch), and the cache's shape.
struct CacheArgs {
  const int32_t* q_start;   // NULL: token i is sequence i's
  const int32_t* kv_len;
  const int32_t* table;
  int32_t n_seqs, n_tokens, table_width, max_len;
  int32_t n_pages, page_shift;   // page_size = 1 << page_shift
  int32_t kv_heads;
};

// Element strides of a [token][head][dim] array.
struct Strides { int64_t token, head, dim; };

struct AppendArgs {
  CacheArgs c;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* k_pages;
  uint16_t* v_pages;
  Strides ks, vs;
};

struct AttnArgs {
  CacheArgs c;
  const uint16_t* q;
  const uint16_t* k_pages;
  const uint16_t* v_pages;
  uint16_t* out;
  float* lse;          // NULL: not wanted
  Strides qs, os;
  int32_t heads, group;   // group: query heads that share a key/value head
  float scale_log2;    // scale * log2(e): the kernels work with powers of two
};

// Pages copied by one launch: every pair in every buffer.  No page of a launch is written twice, or read and written.
constexpr int kCopyBuffers = 128, kCopyPairs = 320;
struct CopyArgs {
  uint64_t page_bytes;
  int32_t n_buffers, n_pairs;
  void* buffer[kCopyBuffers];
  int32_t from_to[kCopyPairs][2];
};
static_assert(sizeof(CopyArgs) <= 4096, "kernel arguments");

hipError_t launch_append(const AppendArgs& a, int head_dim, hipStream_t s);
hipError_t launch_copy(const CopyArgs& a, hipStream_t s);
hipError_t launch_attn_decode(const AttnArgs& a, int head_dim, bool bf16, hipStream_t s);
hipError_t launch_attn_prompt(const AttnArgs& a, int head_dim, bool bf16, hipStream_t s);

}  // namespace vq
