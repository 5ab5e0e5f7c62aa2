// The host logic of attention over the paged cache with stand-ins for the kernel launchers, for a build with sanitizers
// (tests/test_attn_host.py): every launch's arguments are checked against what the kernels assume of them; copies of pages are carried out
// on host memory, a launch's pairs in reverse order, and compared with one pair after another.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <vector>

#include "../../paper_2402_15319_amd/csrc/vq_attn.h"

#define REQUIRE(cond)                                                                       \
  do {                                                                                      \
    if (!(cond)) {                                                                          \
      std::fprintf(stderr, "%s:%d: %s violated\n", __FILE__, __LINE__, #cond);              \
      std::abort();                                                                         \
    }                                                                                       \
  } while (0)

namespace vq {
long long g_launches = 0;
size_t g_workspace = 0;

void check_cache(const CacheArgs& c) {
  REQUIRE(c.n_seqs >= 1 && c.n_tokens >= 1 && c.table_width >= 1 && c.kv_heads >= 1 && c.n_pages >= 1);
  REQUIRE(c.page_shift >= 4 && c.page_shift <= 7);
  REQUIRE(c.max_len >= 0 && c.max_len <= ((long long)c.table_width << c.page_shift));
  REQUIRE(c.kv_len && c.table && (c.q_start || c.n_seqs == c.n_tokens));
}

hipError_t launch_append(const AppendArgs& a, int head_dim, hipStream_t) {
  ++g_launches;
  check_cache(a.c);
  REQUIRE(head_dim % 32 == 0 && head_dim <= 256);
  REQUIRE((a.c.n_tokens / 64 + 2ll * a.c.n_seqs) * a.c.kv_heads * 512 <= 4294967295ll);
  return hipSuccess;
}

hipError_t launch_copy(CopyArgs& a, hipStream_t) {
  ++g_launches;
  REQUIRE(a.n_pairs >= 1 && a.n_pairs <= kCopyPairs && a.n_buffers >= 1 && a.n_buffers <= kCopyBuffers && a.page_bytes % 16 == 0);
  for (int b = 0; b < a.n_buffers; ++b)   // in another order than the pairs': they must not depend on one another
    for (int i = a.n_pairs - 1; i >= 0; --i)
      std::memcpy((char*)a.buffer[b] + a.from_to[i][1] * a.page_bytes, (char*)a.buffer[b] + a.from_to[i][0] * a.page_bytes, a.page_bytes);
  return hipSuccess;
}

void check_attn(const AttnArgs& a, int head_dim) {
  ++g_launches;
  check_cache(a.c);
  REQUIRE(head_dim % 32 == 0 && head_dim <= 256);
  REQUIRE(a.q && a.k_pages && a.v_pages && a.out && a.scale_log2 > 0 && a.group >= 1 && a.heads == a.group * a.c.kv_heads);
}

hipError_t launch_attn_decode(const DecodeArgs& d, int head_dim, bool, hipStream_t) {
  const AttnArgs& a = d.a;
  const DecodePlan& p = d.plan;
  check_attn(a, head_dim);
  REQUIRE(!a.c.q_start && a.c.n_seqs == a.c.n_tokens);
  // every token in a part, every query head in a tile, no part that the longest sequence leaves empty
  REQUIRE(p.chunk >= 128 && p.chunk % 128 == 0 && p.parts >= 1 && p.parts <= kMostParts && (long long)p.chunk * p.parts >= a.c.max_len);
  REQUIRE(p.waves == 4 || (p.waves == 8 && p.parts == 1));
  REQUIRE(p.parts == 1 || (long long)p.chunk * (p.parts - 1) < a.c.max_len);
  REQUIRE((long long)p.chunk + a.c.max_len < 2147483647 - 1024);
  REQUIRE(p.cols >= 1 && p.cols <= kTileHeads && p.tiles * kTileHeads >= a.group && p.cols == (a.group < kTileHeads ? a.group : kTileHeads));
  REQUIRE(p.together >= 1 && p.together <= 3 && (p.together == 1 || (head_dim <= kTogetherDim && p.waves == 4 && p.tiles > 1)));
  if (p.parts > 1) {   // the workspace holds the counters and every part
    const long long units = (long long)a.c.n_seqs * a.c.kv_heads * p.tiles;
    REQUIRE(units <= kJoinCounters);
    const size_t end = (size_t)((char*)d.part - (char*)d.counter) + (size_t)units * p.parts * part_floats(p, head_dim) * 4;
    REQUIRE((char*)d.part - (char*)d.counter >= kJoinCounters * 4 && end <= g_workspace);
  }
  return hipSuccess;
}

hipError_t launch_attn_prompt(const PromptArgs& d, int head_dim, bool, hipStream_t) {
  const AttnArgs& a = d.a;
  const PromptPlan& p = d.plan;
  check_attn(a, head_dim);
  // a slot for every tile, every step in a part, no part that the longest sequence leaves empty
  REQUIRE(p.heads >= 1 && a.group % p.heads == 0 && p.tokens >= 1 && p.heads * p.tokens <= kPromptRows);
  REQUIRE(p.slots == a.c.n_tokens / p.tokens + a.c.n_seqs);
  const long long wide = a.heads / p.heads;
  REQUIRE(p.slots * wide * 256 < 4294967296ll);
  REQUIRE(p.steps >= 1 && p.parts >= 1 && p.parts <= 65535 && (long long)p.steps * p.parts * kPromptTokens >= a.c.max_len);
  REQUIRE(p.parts == 1 || (long long)p.steps * (p.parts - 1) * kPromptTokens < a.c.max_len);
  REQUIRE(p.teams == 1 || (p.teams == 2 && head_dim <= 128));
  if (p.parts > 1) {
    REQUIRE(p.slots * wide <= kJoinCounters);
    const size_t end = (size_t)((char*)d.part - (char*)d.counter) + (size_t)p.slots * wide * p.parts * prompt_part_floats(head_dim) * 4;
    REQUIRE((char*)d.part - (char*)d.counter >= kJoinCounters * 4 && end <= g_workspace);
  }
  REQUIRE((long long)a.c.n_tokens + a.c.n_seqs + kPromptRows < 2147483647);
  return hipSuccess;
}
}  // namespace vq

static void* at(uintptr_t i) { return reinterpret_cast<void*>(i << 20); }   // never read

static void copies(std::mt19937& rng) {
  vq_attn_desc d = {1, 1, 64, 16, 1, VQ_F16, 0.f, 0};
  for (int round = 0; round < 60; ++round) {
    d.n_pages = 2 + rng() % (round < 40 ? 30 : round < 50 ? 900 : 6000);
    const int n_buffers = round % 20 == 0 ? 1 + vq::kCopyBuffers + rng() % 3 : 1 + rng() % 3, n_pairs = 1 + rng() % (round < 40 ? 60 : 3000);
    const size_t page = 64 * 16;   // 16-bit values
    std::vector<std::vector<uint16_t>> got(n_buffers, std::vector<uint16_t>(d.n_pages * page)), want;
    for (auto& b : got)
      for (size_t i = 0; i < b.size(); ++i) b[i] = (uint16_t)rng();
    want = got;
    std::vector<int32_t> pairs;
    for (int i = 0; i < n_pairs; ++i) {
      pairs.push_back(rng() % d.n_pages);
      pairs.push_back(rng() % d.n_pages);
      for (auto& b : want) std::memmove(&b[pairs.back() * page], &b[pairs[2 * i] * page], page * 2);
    }
    std::vector<void*> raw;
    for (auto& b : got) {
      void* p = std::aligned_alloc(16, b.size() * 2);
      std::memcpy(p, b.data(), b.size() * 2);
      raw.push_back(p);
    }
    REQUIRE(vq_cache_copy(&d, n_buffers, raw.data(), n_pairs, pairs.data(), nullptr) == VQ_OK);
    for (int b = 0; b < n_buffers; ++b) {
      REQUIRE(std::memcmp(raw[b], want[b].data(), want[b].size() * 2) == 0);
      std::free(raw[b]);
    }
  }
}

static void calls(std::mt19937& rng) {
  const int dims[] = {64, 96, 128, 256}, pages[] = {16, 32, 64, 128};
  auto log_int = [&](int most) { return 1 + (int)(rng() % (1u << (1 + rng() % 31)) % (unsigned)most); };
  for (int i = 0; i < 20000; ++i) {
    vq_attn_desc d = {};
    d.kv_heads = log_int(1024);
    d.heads = d.kv_heads * log_int(1024 / d.kv_heads);
    d.head_dim = dims[rng() % 4];
    d.page_size = pages[rng() % 4];
    d.n_pages = log_int(2147483647);
    d.dtype = rng() % 2 ? VQ_F16 : VQ_BF16;
    d.scale = 0.1f;
    vq_attn_batch b = {};
    b.n_seqs = log_int(65535);
    const bool one_each = rng() % 2;
    b.n_tokens = one_each ? b.n_seqs : log_int(1 << 24);
    b.table_width = log_int((1 << 29) / d.page_size);
    b.max_len = rng() % 4 ? log_int(b.table_width * d.page_size) : b.table_width * d.page_size;
    b.kv_len = (const int32_t*)at(1);
    b.page_table = (const int32_t*)at(2);
    b.q_start = one_each ? nullptr : (const int32_t*)at(3);
    size_t n = 0;
    if ((long long)b.n_tokens * d.heads / 128 + (long long)b.n_seqs * d.heads > 1 << 20) {
      REQUIRE(vq_attn_workspace_bytes(&d, &b, &n) == VQ_ERR_BAD_ARG);
      continue;
    }
    REQUIRE(vq_attn_workspace_bytes(&d, &b, &n) == VQ_OK && n >= 16);
    vq::g_workspace = n;
    const vq_strides wide = {(int64_t)d.heads * d.head_dim, d.head_dim, 1};
    const int64_t ld = ((int64_t)b.n_tokens + 7) / 8 * 8;
    const vq_strides features = {1, d.head_dim * ld, ld};
    const vq_strides* s = rng() % 3 == 0 ? nullptr : rng() % 2 ? &wide : &features;
    const long long before = vq::g_launches;
    REQUIRE(vq_attn_prompt(&d, &b, at(4), s, at(5), at(6), at(7), s, rng() % 2 ? (float*)at(8) : nullptr, at(9), n, nullptr) == VQ_OK);
    if (one_each) REQUIRE(vq_attn_decode(&d, &b, at(4), s, at(5), at(6), at(7), s, nullptr, at(9), n, nullptr) == VQ_OK);
    const bool short_prompt = vq_attn_prompt(&d, &b, at(4), s, at(5), at(6), at(7), s, nullptr, at(9), n - 1, nullptr) == VQ_ERR_BAD_ARG;
    const bool short_decode = b.n_tokens == b.n_seqs && vq_attn_decode(&d, &b, at(4), s, at(5), at(6), at(7), s, nullptr, at(9), n - 1, nullptr) == VQ_ERR_BAD_ARG;
    REQUIRE(short_prompt || short_decode);   // no more than one of them needs
    REQUIRE(vq_cache_append(&d, &b, at(4), nullptr, at(5), nullptr, at(6), at(7), nullptr) == VQ_OK);
    REQUIRE(vq::g_launches > before);
  }
}

static void strides() {
  vq::g_workspace = 1 << 30;
  vq_attn_desc d = {8, 2, 128, 16, 100, VQ_F16, 0.1f, 0};
  vq_attn_batch b = {4, 4, 10, 160, nullptr, (const int32_t*)at(1), (const int32_t*)at(2)};
  struct { vq_strides s; bool output; } good[] = {
      {{0, 128, 1}, false}, {{1024, 0, 1}, false}, {{1024, 64, 1}, false}, {{1000, 128, 1}, false}, {{1, 128 * 3, 3}, false}, {{0, 0, 1}, false},
      {{1024, 128, 1}, true}, {{1, 1024, 8}, true}, {{1, 128 * 5, 5}, true}, {{130, 130 * 4, 1}, true}, {{2, 2048, 16}, true}, {{1 << 20, 128, 1}, true}};
  for (const auto& g : good) {
    REQUIRE(vq_attn_decode(&d, &b, at(4), &g.s, at(5), at(6), at(7), nullptr, nullptr, at(9), 1 << 30, nullptr) == VQ_OK);
    REQUIRE(vq_attn_prompt(&d, &b, at(4), nullptr, at(5), at(6), at(7), &g.s, nullptr, at(9), 1 << 30, nullptr) == (g.output ? VQ_OK : VQ_ERR_BAD_ARG));
  }
  b.n_seqs = b.n_tokens = 1;   // one token: its stride is not looked at
  const vq_strides any = {-5, 128, 1};
  REQUIRE(vq_attn_decode(&d, &b, at(4), &any, at(5), at(6), at(7), &any, nullptr, at(9), 1 << 30, nullptr) == VQ_OK);
}

int main() {
  std::mt19937 rng(1);
  copies(rng);
  calls(rng);
  strides();
  std::printf("host check ok\n");
  return 0;
}
