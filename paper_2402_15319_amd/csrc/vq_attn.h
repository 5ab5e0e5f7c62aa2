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
  float* k_scales;     // pages in 8 bits: [page][kv head][block]; NULL: pages in 16 bits
  float* v_scales;
  int32_t bf16;        // the type of k and v: bf16, or fp16
};
constexpr int kBlock = 16;   // slots of a head that share a scale

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
  int32_t window, sinks;    // window 0: every token up to a row's own is seen
  const float* k_scales;    // pages in 8 bits: [page][kv head][block of 16 slots]; NULL: pages in 16 bits
  const float* v_scales;
};
constexpr int kEveryToken = 1 << 30;   // a window that no sequence reaches the end of

// How a call of vq_attn_decode is split: a workgroup takes `chunk` tokens of one sequence and up to 16 query heads of one
// key/value head (a tile); where a sequence has several parts, the last of their workgroups to finish joins them.
struct DecodePlan {
  int32_t chunk, parts;   // tokens of a part; parts of the longest sequence
  int32_t tiles, cols;    // tiles of a key/value head's query heads; query heads of a tile at most
  int32_t together;       // tiles of a workgroup: 1, 2 or 3
  int32_t waves;          // of a workgroup: 4 or 8; each takes 32 tokens in turn, 64 of pages in 8 bits
};
constexpr int kJoinCounters = 16384;   // at the start of the workspace: parts that have finished, zero between calls
constexpr int kTileHeads = 16, kTogetherDim = 128;   // several tiles up to this head_dim: two of larger ones do not fit the registers (three of 128 spill 76 bytes)
constexpr int kThreeDim8 = 64;         // three tiles in 8 bits up to this head_dim: of 96 and 128 they spill 36 and 252 bytes
constexpr int kMostParts = 64;         // of a sequence

struct DecodeArgs {
  AttnArgs a;
  DecodePlan plan;
  uint32_t* counter;   // [n_seqs][kv_heads][tiles]
  float* part;         // [n_seqs][kv_heads][tiles][parts][part_floats]
};

// What a part leaves: 16 maxima, 16 sums of weights, and sums over the values for each head of the tile.
__host__ __device__ inline size_t part_floats(const DecodePlan& p, int head_dim) { return 2 * kTileHeads + (size_t)p.cols * head_dim; }

// vq_attn_prompt: (new token, query head) pairs that a workgroup takes, and workgroups of a launch at most, which bounds those of an
// append too (2^32 threads for each dimension of a grid).
constexpr int kPromptRows = 128, kPromptTokens = 64;   // tokens: of a step
constexpr int64_t kPromptMostWorkgroups = 1 << 20;

// How a call of vq_attn_prompt is split: slots for tiles of one sequence's `tokens` new tokens and `heads` query heads of a
// key/value head, 128 (token, head) rows or a few less, and parts of at most so many steps, which one or two teams of four waves take in turn.
struct PromptPlan {
  int64_t slots;
  int32_t steps, parts;
  int32_t heads, tokens, teams;
};
struct PromptArgs {
  AttnArgs a;
  PromptPlan plan;
  uint32_t* counter;   // [slots][heads / plan.heads]
  float* part;         // [slots][heads / plan.heads][parts][prompt_part_floats]
};
inline size_t prompt_part_floats(int head_dim) { return kPromptRows * (4 + (size_t)head_dim); }

// Pages copied by one launch: every pair in every buffer.  No page of a launch is written twice, or read and written.
constexpr int kCopyBuffers = 128, kCopyPairs = 1024, kCopyFew = 64;
template <int PAIRS>
struct CopyArgsOf {
  uint64_t page_bytes;
  uint64_t scales_at;   // bytes from the first page to its scales, of which a page has scale_words
  int32_t n_buffers, n_pairs, pieces, scale_words;   // pieces: workgroups for a page
  void* buffer[kCopyBuffers];
  int32_t from_to[PAIRS][2];
};
typedef CopyArgsOf<kCopyPairs> CopyArgs;
static_assert(sizeof(CopyArgs) <= 16384, "kernel arguments");

hipError_t launch_append(const AppendArgs& a, int head_dim, hipStream_t s);
hipError_t launch_append8(const AppendArgs& a, int head_dim, hipStream_t s);   // pages in 8 bits
hipError_t launch_copy(CopyArgs& a, hipStream_t s);
hipError_t launch_attn_decode(const DecodeArgs& a, int head_dim, bool bf16, hipStream_t s);
hipError_t launch_attn_decode_window(const DecodeArgs& a, int head_dim, bool bf16, hipStream_t s);   // pages in 16 bits
hipError_t launch_attn_decode8(const DecodeArgs& a, int head_dim, bool bf16, hipStream_t s);         // pages in 8 bits, a.window as it is
hipError_t launch_attn_prompt(const PromptArgs& a, int head_dim, bool bf16, hipStream_t s);
hipError_t launch_attn_prompt_256(const PromptArgs& a, bool bf16, hipStream_t s);
hipError_t launch_attn_prompt_window(const PromptArgs& a, int head_dim, bool bf16, hipStream_t s);
hipError_t launch_attn_prompt_window_256(const PromptArgs& a, bool bf16, hipStream_t s);
hipError_t launch_attn_prompt8(const PromptArgs& a, int head_dim, bool bf16, hipStream_t s);
hipError_t launch_attn_prompt8_256(const PromptArgs& a, bool bf16, hipStream_t s);

}  // namespace vq
