// Entry points of attention over the paged cache (include/vq.h): argument checks and the plan of
// every launch, on the host.
#include <math.h>
#include <string.h>

#include "vq_attn.h"

namespace vq {
namespace {

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }

int hip_status(hipError_t e) { return e == hipSuccess ? VQ_OK : VQ_ERR_HIP; }

constexpr float kLog2E = 1.44269504088896f;

int check_attn_desc(const vq_attn_desc* d, bool scaled) {
  if (!d) return VQ_ERR_NULL;
  if (d->heads < 1 || d->kv_heads < 1 || d->head_dim < 1 || d->page_size < 1 || d->n_pages < 1 || d->reserved != 0) return VQ_ERR_BAD_DESC;
  if (d->heads % d->kv_heads != 0) return VQ_ERR_BAD_DESC;
  if (d->heads > 1024) return VQ_ERR_UNSUPPORTED;
  if (d->head_dim != 64 && d->head_dim != 96 && d->head_dim != 128 && d->head_dim != 256) return VQ_ERR_UNSUPPORTED;
  if (d->page_size != 16 && d->page_size != 32 && d->page_size != 64 && d->page_size != 128) return VQ_ERR_UNSUPPORTED;
  if (d->dtype != VQ_F16 && d->dtype != VQ_BF16) return VQ_ERR_UNSUPPORTED;
  if (scaled && !(d->scale > 0.f && d->scale * kLog2E <= 3.402823466e38f)) return VQ_ERR_BAD_ARG;   // a NaN fails both
  return VQ_OK;
}

constexpr int kMostLen = 1 << 29;   // tokens of a sequence: the kernels' token indexes stay within 32 bits with room to spare

// What the host can see of a batch; the arrays' contents are checked by the kernels.
int check_batch_sizes(const vq_attn_desc& d, const vq_attn_batch* b) {
  if (!b) return VQ_ERR_NULL;
  if (b->n_seqs < 1 || b->n_seqs > 65535 || b->n_tokens < 1 || b->table_width < 1 || b->max_len < 0 || b->max_len > kMostLen) return VQ_ERR_BAD_ARG;
  if ((int64_t)b->max_len > (int64_t)b->table_width * d.page_size) return VQ_ERR_BAD_ARG;
  if ((int64_t)b->n_tokens * d.heads / kPromptRows + (int64_t)b->n_seqs * d.heads > kPromptMostWorkgroups) return VQ_ERR_BAD_ARG;
  return VQ_OK;
}

int check_batch(const vq_attn_desc& d, const vq_attn_batch* b, bool one_each) {
  const int st = check_batch_sizes(d, b);
  if (st != VQ_OK) return st;
  if ((one_each || !b->q_start) && b->n_tokens != b->n_seqs) return VQ_ERR_BAD_ARG;
  if (!b->kv_len || !b->page_table) return VQ_ERR_NULL;
  if (!aligned4(b->kv_len) || !aligned4(b->page_table) || !aligned4(b->q_start)) return VQ_ERR_ALIGN;
  return VQ_OK;
}

CacheArgs cache_args(const vq_attn_desc& d, const vq_attn_batch& b, bool one_each) {
  CacheArgs c = {};
  c.q_start = one_each ? nullptr : b.q_start;
  c.kv_len = b.kv_len;
  c.table = b.page_table;
  c.n_seqs = b.n_seqs;
  c.n_tokens = b.n_tokens;
  c.table_width = b.table_width;
  c.max_len = b.max_len;
  c.n_pages = d.n_pages;
  c.page_shift = __builtin_ctz((unsigned)d.page_size);
  c.kv_heads = d.kv_heads;
  return c;
}

constexpr int64_t kMostStride = int64_t(1) << 56;   // elements that an index may step over: offsets in bytes stay within 64 bits

// The strides of a [n_tokens][heads][head_dim] array as the kernels take them (see vq_strides).
int check_strides(const vq_strides* in, int n_tokens, int heads, int head_dim, bool output, Strides* out) {
  if (!in) {
    *out = {(int64_t)heads * head_dim, head_dim, 1};
    return VQ_OK;
  }
  Strides s = {n_tokens > 1 ? in->token : 0, heads > 1 ? in->head : 0, in->dim};
  if (s.token < 0 || s.head < 0 || s.dim < 1) return VQ_ERR_BAD_ARG;
  if (s.token > kMostStride / n_tokens || s.head > kMostStride / heads || s.dim > kMostStride / head_dim) return VQ_ERR_BAD_ARG;
  if (output) {   // no two elements at one place: each stride spans what the smaller ones reach
    struct { int64_t stride, extent; } e[3] = {{s.token, n_tokens}, {s.head, heads}, {s.dim, head_dim}};
    for (int i = 0; i < 2; ++i)
      for (int j = 0; j < 2 - i; ++j)
        if (e[j].stride > e[j + 1].stride) { const auto t = e[j]; e[j] = e[j + 1]; e[j + 1] = t; }
    int64_t reach = 1;   // elements from the first to behind the last
    for (int i = 0; i < 3; ++i) {
      if (e[i].extent == 1) continue;
      if (e[i].stride < reach) return VQ_ERR_BAD_ARG;
      reach += e[i].stride * (e[i].extent - 1);
    }
  }
  *out = s;
  return VQ_OK;
}

// Rows that the kernels take in whole vectors begin at 16 bytes; of others they take an element at a time, from any.
bool aligned_rows(const void* p, const Strides& s) {
  return s.dim == 1 && ((s.token | s.head) & 7) == 0 ? aligned16(p) : ((uintptr_t)p & 1) == 0;
}

constexpr int kPartStep = 128;            // tokens that a workgroup takes at a time
// Workgroups: one for each CU.  The plans count on 256 CUs rather than on the device's: they follow from sizes alone, so that a
// workspace can be asked for without a device.
constexpr int64_t kEnoughUnits = 256;
constexpr int64_t kTogetherUnits = 16;
constexpr int kLongPart = 4096, kShortPart = 1024;
constexpr int kShortValues = 32768;       // of a sequence's keys: no parts up to here

DecodePlan decode_plan(const vq_attn_desc& d, const vq_attn_batch& b) {
  DecodePlan p;
  const int group = d.heads / d.kv_heads;
  p.tiles = (group + kTileHeads - 1) / kTileHeads;
  p.cols = group < kTileHeads ? group : kTileHeads;
  p.together = d.head_dim > kTogetherDim || p.tiles == 1 ? 1 : p.tiles == 2 || p.tiles == 4 ? 2 : 3;
  // Three tiles together read a key/value head once, but leave one workgroup to join all of their parts: with 48 heads to one of 128 and
  // sequences of 4,096 to 8,192, 64 of them take 59 us (a tile to a workgroup 118) and 32 36 (76); with fewer the join is longer than what
  // it saves (16 46 us and 43, 8 50 and 28).
  if ((int64_t)b.n_seqs * d.kv_heads * ((p.tiles + p.together - 1) / p.together) < kTogetherUnits) p.together = 1;
  const int64_t units = (int64_t)b.n_seqs * d.kv_heads * ((p.tiles + p.together - 1) / p.together);
  const int64_t steps = b.max_len > kPartStep ? ((int64_t)b.max_len + kPartStep - 1) / kPartStep : 1;
  int64_t parts = 1;
  p.waves = 4;
  if ((int64_t)b.max_len * d.head_dim <= kShortValues) {
    // One part of 8 waves: a step or two for each of them cost less than the join (a sequence of 256 tokens x 32 heads of 128 6.1
    // us, in two parts of 4 waves 7.7; of 512 8.9 and 8.0; of 512 x 32 heads of 64 5.6 and 7.7).
    p.waves = b.max_len > 32 * p.waves && p.together == 1 ? 8 : 4;
  } else if (units * p.together <= kJoinCounters) {
    // Fewer workgroups than CUs: as many parts as fill the chip once, up to 4,096 tokens each (130,001 tokens x 8 heads: 256
    // workgroups 97 us, 512 100, 1,024 106).  As many without a split: parts of 1,024 tokens, which even out what the lengths differ
    // by (61 sequences of 1 to 8,192: parts of 512 61 us, of 1,024 66; 61 of 4,000 each: parts of 512 194 us, of 1,024
    // 177).  Lengths can differ in the first case too, and only max_len is known here: 31 sequences of 1 to 8,192 x 8 heads have two
    // parts each and take 50 us, 32 of them eight and 58.
    const int64_t most = units < kEnoughUnits ? kLongPart : kShortPart;
    const int64_t enough = (kEnoughUnits + units - 1) / units, least = (steps * kPartStep + most - 1) / most;
    parts = (least + enough - 1) / enough * enough;   // as many for every CU
    parts = parts < kMostParts ? parts : kMostParts;
    parts = parts < steps ? parts : steps;
  }
  const int64_t per = (steps + parts - 1) / parts;   // steps of a part
  p.parts = (int32_t)((steps + per - 1) / per);
  p.chunk = (int32_t)(per * kPartStep);
  return p;
}

constexpr int kLeastSteps = 8;          // of a part
constexpr int64_t kOneTeamUnits = 512, kWideUnits = 448;   // workgroups that the chip runs at once, or nearly: of one team, and of heads of 256

PromptPlan prompt_plan(const vq_attn_desc& d, const vq_attn_batch& b) {
  PromptPlan p;
  // The heads of a tile: as few tiles as sequences of the mean length need; 4, 2 or 1, with 32 successive tokens of a head to a wave, if that
  // takes no more than an eighth more of them.  (Nine prompts of up to 2,500 x 8 key/value heads, 4 heads to each: 98 us with four
  // heads of 32 tokens, 130 with all heads of a token after one another.)
  const int group = d.heads / d.kv_heads, by = group % 4 == 0 ? 4 : group % 2 == 0 ? 2 : 1;
  const int64_t mean = (b.n_tokens + (int64_t)b.n_seqs - 1) / b.n_seqs;
  const auto tiles = [&](int heads) { return group / heads * ((mean + kPromptRows / heads - 1) / (kPromptRows / heads)); };
  p.heads = by;
  int64_t best = tiles(by) * 8;
  for (int h = 1; h <= group && h <= kPromptRows; ++h)
    if (group % h == 0 && tiles(h) * 9 < best) {
      p.heads = h;
      best = tiles(h) * 9;
    }
  // Where there are few tokens for each sequence, no more than twice as many: their rows then lie in one wave or two (one token behind 2,911 x
  // 8 heads to one: 20 us, 26 with the heads 16 rows apart).
  p.tokens = (int32_t)(2 * mean < kPromptRows / p.heads ? 2 * mean : kPromptRows / p.heads);
  p.slots = b.n_tokens / p.tokens + b.n_seqs;
  const int64_t units = p.slots * (d.heads / p.heads), steps = b.max_len > 0 ? ((int64_t)b.max_len + kPromptTokens - 1) / kPromptTokens : 1;
  // Two workgroups of one team share a compute unit and run a step each in about 2.1 us; one alone takes 1.3 us a step.  Where there is but
  // one for each compute unit, or where two are gone through long before the last, two teams take a tile's steps in turn.  Theirs is one
  // barrier, which keeps both at the same work and costs a long prompt 14 %.  Three workgroups on heads of 64 share a compute unit: those keep
  // one team where parts are long.  (`lone`: 32 heads of 128, prompts of 768 and 1,024: 24.6 and 29.3 us with one team, 20.4 and 24.9 with two;
  // two chunks behind 12,000 tokens, heads of 64: 72 us with one, 96 with two.  `few`: 32 heads of 128, 1,500, 1,800 and 2,048 tokens: 41.5, 49.4
  // and 57.4 with one, 37.3, 48.8 and 55.4 with two; of 64 25.2 and 21.9 at 1,500.  Its lines of 24 and 32 steps enclose what was
  // measured first, and are not where one team becomes the faster: 32 heads and 1,100 tokens take 30.4 us with one and would take 27.3, 16
  // heads and 3,000 67.7 and 57.5, but 8 heads and 4,500 67.8 and 74.1.)
  const int64_t full = (b.n_tokens + (int64_t)p.tokens - 1) / p.tokens * (d.heads / p.heads);   // tiles, but for those that a sequence does not fill
  const bool lone = full <= 256 && steps >= 8 && (steps <= 32 || d.head_dim > 64), few = full <= 512 && steps >= 24 && steps <= 32;
  p.teams = d.head_dim <= 128 && (lone || few) ? 2 : 1;
  // Parts, where they bring the workgroups near to what the chip runs at once (heads of 256 have one workgroup to a compute unit, and of
  // longer parts: 16 heads, 1,500 and 2,048 tokens 67 and 88 us whole, 51 and 80 in two parts).
  const int64_t enough = p.teams == 2 ? kEnoughUnits : d.head_dim > 128 ? kWideUnits : kOneTeamUnits;
  int64_t parts = units < enough ? (enough + units / 2) / units : 1;
  while (parts > 1 && parts * parts > steps) --parts;   // to join a part takes about as long as a step
  int64_t per = (steps + parts - 1) / parts;
  per = per < kLeastSteps ? kLeastSteps : per;
  p.steps = (int32_t)per;
  p.parts = (int32_t)((steps + per - 1) / per);
  return p;
}

// The most parts that vq_attn_decode leaves in all tiles together, over batches of no more than n_seqs sequences of up to max_len tokens: those
// of decode_plan above, with the tiles and the units that such a batch has at most.
int64_t decode_most_parts(const vq_attn_desc& d, int64_t n_seqs, int64_t max_len) {
  if (max_len * d.head_dim <= kShortValues) return 0;
  vq_attn_batch b = {};
  b.n_seqs = b.n_tokens = 65535;   // enough for several tiles to a workgroup, where there are several
  b.max_len = 1;
  const DecodePlan p = decode_plan(d, b);
  const auto least = [](int64_t tokens) { return tokens < 1 ? 1 : tokens; };
  const int64_t steps = (max_len + kPartStep - 1) / kPartStep, most = steps < kMostParts ? steps : kMostParts;
  const int64_t wide = d.kv_heads * (int64_t)((p.tiles + p.together - 1) / p.together), tiles = n_seqs * d.kv_heads * p.tiles;
  // Fewer than kEnoughUnits units: parts of kLongPart tokens, and up to kEnoughUnits / units - 1 more for as many on every CU.
  const int64_t few = tiles < (kEnoughUnits - 1) * p.together ? tiles : (kEnoughUnits - 1) * p.together;
  const int64_t by_length = few * least((steps * kPartStep + kLongPart - 1) / kLongPart) + (kEnoughUnits - 1) * p.together;
  int64_t parts = few * most < by_length ? few * most : by_length;
  if (n_seqs * wide >= kEnoughUnits) {
    const int64_t many = tiles < kJoinCounters ? tiles : kJoinCounters, each = least((steps * kPartStep + kShortPart - 1) / kShortPart);
    const int64_t of_many = many * (each < most ? each : most);
    parts = of_many > parts ? of_many : parts;
  }
  return parts;
}

// The same of vq_attn_prompt: a call has parts where its units are fewer than `enough`, and then up to enough + units / 2 of them; its
// units are at most those of tiles of 64 rows and two tiles of one row's heads for each sequence.
int64_t prompt_most_parts(const vq_attn_desc& d, int64_t n_seqs, int64_t n_tokens, int64_t max_len) {
  const int64_t steps = (max_len + kPromptTokens - 1) / kPromptTokens, enough = d.head_dim > 128 ? kWideUnits : kOneTeamUnits;
  const int64_t of_steps = (steps + kLeastSteps - 1) / kLeastSteps, of_join = (int64_t)sqrt((double)steps);   // steps below 2^24: exact
  const int64_t each = of_steps < of_join ? of_steps : of_join;
  if (each <= 1) return 0;
  int64_t units = n_tokens * d.heads / 64 + 2 * n_seqs * d.heads;
  units = units < enough ? units : enough;
  const int64_t all = enough + enough / 2;
  return units * each < all ? units * each : all;
}

// Bytes of the workspace: the counters and what the parts leave, for this batch and every one of no more sequences, new tokens and
// tokens in a sequence.  (What a batch itself needs does not grow with it: fewer workgroups are split into more parts.)
size_t workspace(const vq_attn_desc& d, const vq_attn_batch& b) {
  const int64_t decode = decode_most_parts(d, b.n_seqs < b.n_tokens ? b.n_seqs : b.n_tokens, b.max_len);
  const int64_t prompt = prompt_most_parts(d, b.n_seqs, b.n_tokens, b.max_len);
  if (decode == 0 && prompt == 0) return 16;
  DecodePlan tile = {};
  tile.cols = d.heads / d.kv_heads < kTileHeads ? d.heads / d.kv_heads : kTileHeads;
  const size_t of_decode = (size_t)decode * part_floats(tile, d.head_dim), of_prompt = (size_t)prompt * prompt_part_floats(d.head_dim);
  return (kJoinCounters + (of_decode > of_prompt ? of_decode : of_prompt)) * sizeof(float);
}

int attn_impl(const vq_attn_desc* desc, const vq_attn_batch* batch, const void* q, const vq_strides* q_strides, const void* k_pages,
              const void* v_pages, void* out, const vq_strides* out_strides, float* lse_f32, void* workspace, size_t workspace_bytes,
              void* stream, bool decode) {
  int st = check_attn_desc(desc, true);
  if (st != VQ_OK) return st;
  st = check_batch(*desc, batch, decode);
  if (st != VQ_OK) return st;
  if (!q || !k_pages || !v_pages || !out || !workspace) return VQ_ERR_NULL;
  if (!aligned16(k_pages) || !aligned16(v_pages) || !aligned16(workspace) || !aligned4(lse_f32)) return VQ_ERR_ALIGN;
  if (q == out || k_pages == out || v_pages == out) return VQ_ERR_BAD_ARG;
  DecodeArgs both = {};
  AttnArgs& a = both.a;
  st = check_strides(q_strides, batch->n_tokens, desc->heads, desc->head_dim, false, &a.qs);
  if (st != VQ_OK) return st;
  st = check_strides(out_strides, batch->n_tokens, desc->heads, desc->head_dim, true, &a.os);
  if (st != VQ_OK) return st;
  if (!aligned_rows(q, a.qs) || !aligned_rows(out, a.os)) return VQ_ERR_ALIGN;
  if (workspace_bytes < vq::workspace(*desc, *batch)) return VQ_ERR_BAD_ARG;
  a.c = cache_args(*desc, *batch, decode);
  a.q = (const uint16_t*)q;
  a.k_pages = (const uint16_t*)k_pages;
  a.v_pages = (const uint16_t*)v_pages;
  a.out = (uint16_t*)out;
  a.lse = lse_f32;
  a.heads = desc->heads;
  a.group = desc->heads / desc->kv_heads;
  a.scale_log2 = desc->scale * kLog2E;
  const bool bf16 = desc->dtype == VQ_BF16;
  if (!decode) {
    const PromptArgs prompt = {a, prompt_plan(*desc, *batch), (uint32_t*)workspace, (float*)workspace + kJoinCounters};
    return hip_status(launch_attn_prompt(prompt, desc->head_dim, bf16, (hipStream_t)stream));
  }
  both.plan = decode_plan(*desc, *batch);
  both.counter = (uint32_t*)workspace;
  both.part = (float*)workspace + kJoinCounters;
  return hip_status(launch_attn_decode(both, desc->head_dim, bf16, (hipStream_t)stream));
}

}  // namespace
}  // namespace vq

using namespace vq;

extern "C" {

int vq_cache_bytes(const vq_attn_desc* desc, size_t* bytes) {
  const int st = check_attn_desc(desc, false);
  if (st != VQ_OK) return st;
  if (!bytes) return VQ_ERR_NULL;
  *bytes = (size_t)desc->n_pages * desc->kv_heads * desc->page_size * desc->head_dim * 2;
  return VQ_OK;
}

int vq_cache_append(const vq_attn_desc* desc, const vq_attn_batch* batch, const void* k, const vq_strides* k_strides, const void* v,
                    const vq_strides* v_strides, void* k_pages, void* v_pages, void* stream) {
  int st = check_attn_desc(desc, false);
  if (st != VQ_OK) return st;
  st = check_batch(*desc, batch, false);
  if (st != VQ_OK) return st;
  if (!k || !v || !k_pages || !v_pages) return VQ_ERR_NULL;
  if (!aligned16(k_pages) || !aligned16(v_pages)) return VQ_ERR_ALIGN;
  if (k_pages == v_pages || k == k_pages || k == v_pages || v == k_pages || v == v_pages) return VQ_ERR_BAD_ARG;
  AppendArgs a = {};
  st = check_strides(k_strides, batch->n_tokens, desc->kv_heads, desc->head_dim, false, &a.ks);
  if (st != VQ_OK) return st;
  st = check_strides(v_strides, batch->n_tokens, desc->kv_heads, desc->head_dim, false, &a.vs);
  if (st != VQ_OK) return st;
  if (!aligned_rows(k, a.ks) || !aligned_rows(v, a.vs)) return VQ_ERR_ALIGN;
  a.c = cache_args(*desc, *batch, false);
  a.k = (const uint16_t*)k;
  a.v = (const uint16_t*)v;
  a.k_pages = (uint16_t*)k_pages;
  a.v_pages = (uint16_t*)v_pages;
  return hip_status(launch_append(a, desc->head_dim, (hipStream_t)stream));
}

int vq_cache_copy(const vq_attn_desc* desc, int n_buffers, void* const* buffers, int n_pairs, const int32_t* from_to, void* stream) {
  const int st = check_attn_desc(desc, false);
  if (st != VQ_OK) return st;
  if (n_buffers < 1 || n_buffers > 65536 || n_pairs < 1 || n_pairs > (1 << 30)) return VQ_ERR_BAD_ARG;
  if (!buffers || !from_to) return VQ_ERR_NULL;
  for (int i = 0; i < n_buffers; ++i) {
    if (!buffers[i]) return VQ_ERR_NULL;
    if (!aligned16(buffers[i])) return VQ_ERR_ALIGN;
  }
  for (size_t i = 0; i < 2 * (size_t)n_pairs; ++i)
    if (from_to[i] < 0 || from_to[i] >= desc->n_pages) return VQ_ERR_BAD_ARG;
  // Launches of one stream follow one another, so what depends on an earlier pair starts a new one.  The pages of a launch
  // are held in a small hash table (open addressing, at most half full): 1 read, 2 written.
  constexpr int kSlots = 4096;
  static_assert(kSlots >= 4 * kCopyPairs, "half full at most");
  CopyArgs a;
  a.reserved = 0;
  a.page_bytes = (uint64_t)desc->kv_heads * desc->page_size * desc->head_dim * 2;
  for (int first = 0; first < n_pairs;) {
    int32_t page[kSlots];
    uint8_t use[kSlots];
    memset(use, 0, sizeof(use));
    const auto slot = [&](int32_t p) {
      uint32_t h = ((uint32_t)p * 2654435761u) >> 20;
      while (use[h] && page[h] != p) h = (h + 1) & (kSlots - 1);
      return h;
    };
    int n = 0, i = first;
    for (; i < n_pairs && n < kCopyPairs; ++i) {
      const int32_t from = from_to[2 * (size_t)i], to = from_to[2 * (size_t)i + 1];
      if (from == to) continue;
      if (use[slot(to)] || use[slot(from)] == 2) break;
      const uint32_t f = slot(from);
      page[f] = from;
      use[f] = 1;
      const uint32_t t = slot(to);
      page[t] = to;
      use[t] = 2;
      a.from_to[n][0] = from;
      a.from_to[n][1] = to;
      ++n;
    }
    first = i;
    if (n == 0) continue;   // pages onto themselves only
    a.n_pairs = n;
    for (int b = 0; b < n_buffers; b += kCopyBuffers) {
      a.n_buffers = n_buffers - b < kCopyBuffers ? n_buffers - b : kCopyBuffers;
      memcpy(a.buffer, buffers + b, (size_t)a.n_buffers * sizeof(void*));
      if (launch_copy(a, (hipStream_t)stream) != hipSuccess) return VQ_ERR_HIP;
    }
  }
  return VQ_OK;
}

int vq_attn_workspace_bytes(const vq_attn_desc* desc, const vq_attn_batch* batch, size_t* bytes) {
  int st = check_attn_desc(desc, false);
  if (st != VQ_OK) return st;
  st = check_batch_sizes(*desc, batch);
  if (st != VQ_OK) return st;
  if (!bytes) return VQ_ERR_NULL;
  *bytes = vq::workspace(*desc, *batch);
  return VQ_OK;
}

int vq_attn_decode(const vq_attn_desc* desc, const vq_attn_batch* batch, const void* q, const vq_strides* q_strides, const void* k_pages,
                   const void* v_pages, void* out, const vq_strides* out_strides, float* lse_f32, void* workspace, size_t workspace_bytes,
                   void* stream) {
  return attn_impl(desc, batch, q, q_strides, k_pages, v_pages, out, out_strides, lse_f32, workspace, workspace_bytes, stream, true);
}

int vq_attn_prompt(const vq_attn_desc* desc, const vq_attn_batch* batch, const void* q, const vq_strides* q_strides, const void* k_pages,
                   const void* v_pages, void* out, const vq_strides* out_strides, float* lse_f32, void* workspace, size_t workspace_bytes,
                   void* stream) {
  return attn_impl(desc, batch, q, q_strides, k_pages, v_pages, out, out_strides, lse_f32, workspace, workspace_bytes, stream, false);
}

}  // extern "C"
