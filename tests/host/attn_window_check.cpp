// The plans of attention with a window and over pages in 8 bits (tests/test_attn_window_host.py): stand-ins for the kernel launchers check that
// every token that a row sees is in a part, and that each launch stays inside a workspace that was asked for without a window, for this batch or a
// larger one.  Copies of pages in 8 bits are carried out on host memory, a launch's pairs in reverse order, and compared with one pair after another.
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
size_t g_workspace = 0;
vq_attn_desc g_desc;
vq_attn_window g_window;   // window 0: none
std::mt19937 rng(5);
long long g_launches = 0;

const char* scales(const void* pages) {
  return (const char*)pages + (int64_t)g_desc.n_pages * g_desc.kv_heads * g_desc.page_size * g_desc.head_dim;
}

hipError_t launch_append(const AppendArgs& a, int, hipStream_t) {
  ++g_launches;
  const bool e = g_desc.cache_dtype == VQ_E4M3;
  REQUIRE((const char*)a.k_scales == (e ? scales(a.k_pages) : nullptr) && (const char*)a.v_scales == (e ? scales(a.v_pages) : nullptr));
  REQUIRE(a.bf16 == (g_desc.dtype == VQ_BF16));
  // threads of the widest grid: a workgroup of 256 for 32 positions of a head
  REQUIRE((a.c.n_tokens / 32 + 2ll * a.c.n_seqs) * a.c.kv_heads * 256 <= 4294967295ll);
  return hipSuccess;
}

hipError_t launch_copy(CopyArgs& a, hipStream_t) {
  ++g_launches;
  REQUIRE(a.n_pairs >= 1 && a.n_pairs <= kCopyPairs && a.n_buffers >= 1 && a.n_buffers <= kCopyBuffers && a.page_bytes % 16 == 0);
  for (int b = 0; b < a.n_buffers; ++b)
    for (int i = a.n_pairs - 1; i >= 0; --i) {
      char* base = (char*)a.buffer[b];
      std::memcpy(base + a.from_to[i][1] * a.page_bytes, base + a.from_to[i][0] * a.page_bytes, a.page_bytes);
      char* s = base + a.scales_at;
      std::memcpy(s + (size_t)a.from_to[i][1] * a.scale_words * 4, s + (size_t)a.from_to[i][0] * a.scale_words * 4, (size_t)a.scale_words * 4);
    }
  return hipSuccess;
}

void check(const AttnArgs& a) {
  ++g_launches;
  const bool e = g_desc.cache_dtype == VQ_E4M3;
  REQUIRE((const char*)a.k_scales == (e ? scales(a.k_pages) : nullptr) && (const char*)a.v_scales == (e ? scales(a.v_pages) : nullptr));
  if (g_window.window) REQUIRE(a.window == g_window.window && a.sinks == g_window.sinks);
  else REQUIRE(a.sinks == 0 && a.window == (e ? kEveryToken : 0) && kEveryToken > a.c.max_len);
}

int some_length(int most) { return most == 0 ? 0 : rng() % 2 ? most : (int)(rng() % (unsigned)most) + 1; }

hipError_t launch_attn_decode(const DecodeArgs& d, int head_dim, bool, hipStream_t) {
  const AttnArgs& a = d.a;
  const DecodePlan& p = d.plan;
  check(a);
  const bool e = a.k_scales != nullptr;
  const int step = e ? 64 : 32;      // of a wave
  REQUIRE(p.chunk >= 4 * step && p.chunk % (4 * step) == 0 && p.parts >= 1 && p.parts <= kMostParts);
  REQUIRE(p.waves == 4 || (p.waves == 8 && !e && p.parts == 1 && head_dim <= kTogetherDim && p.together == 1));
  REQUIRE(p.together >= 1 && p.together <= (head_dim > kTogetherDim ? 1 : e && head_dim > kThreeDim8 ? 2 : 3));
  for (int i = 0; i < 8; ++i) {      // what the kernel goes through of a sequence
    const int len = i == 0 ? a.c.max_len : some_length(a.c.max_len);
    int skip = 0;
    if (a.window) {
      const int first = len > a.window ? len - a.window : 0, low = ((a.sinks < len ? a.sinks : len) + step - 1) / step * step;
      skip = first / step * step - low > 0 ? first / step * step - low : 0;
    }
    REQUIRE(len - skip >= 0 && (int64_t)p.chunk * p.parts >= len - skip);
    REQUIRE((int64_t)len + p.chunk + 16 * step < 2147483647);
  }
  if (p.parts > 1) {
    const long long units = (long long)a.c.n_seqs * a.c.kv_heads * p.tiles;
    REQUIRE(units <= kJoinCounters);
    REQUIRE((size_t)((char*)d.part - (char*)d.counter) + (size_t)units * p.parts * part_floats(p, head_dim) * 4 <= g_workspace);
  }
  return hipSuccess;
}

hipError_t launch_attn_prompt(const PromptArgs& d, int head_dim, bool, hipStream_t) {
  const AttnArgs& a = d.a;
  const PromptPlan& p = d.plan;
  check(a);
  REQUIRE(p.steps >= 1 && p.parts >= 1 && p.parts <= 65535 && (p.teams == 1 || (p.teams == 2 && head_dim <= 128)));
  REQUIRE(p.slots == a.c.n_tokens / p.tokens + a.c.n_seqs && p.tokens <= kPromptRows);
  for (int i = 0; i < 16; ++i) {     // what it goes through of a tile whose first and last rows have these positions
    const int last = some_length(a.c.max_len) - 1;
    if (last < 0) continue;
    const int first_row = last - (int)(rng() % (unsigned)p.tokens);
    int all = last / kPromptTokens + 1;
    if (a.window) {
      const int first = first_row - a.window + 1 > 0 ? first_row - a.window + 1 : 0;
      const int over = first / kPromptTokens - (a.sinks + kPromptTokens - 1) / kPromptTokens;   // in whole steps
      if (over > 0) all -= over;
      const int fine = first / 16 - (a.sinks + 31) / 32 * 2;                                     // in sixteens, pages in 16 bits
      if (!a.k_scales && fine > 0 && (last / 16 - fine) / 4 + 1 < all) all = (last / 16 - fine) / 4 + 1;
    }
    REQUIRE(all >= 1 && (int64_t)p.steps * p.parts >= all);
  }
  if (p.parts > 1) {
    const size_t units = (size_t)p.slots * (a.heads / p.heads);
    REQUIRE(units <= kJoinCounters);
    REQUIRE((size_t)((char*)d.part - (char*)d.counter) + units * p.parts * prompt_part_floats(head_dim) * 4 <= g_workspace);
  }
  return hipSuccess;
}
}  // namespace vq

static void* at(uintptr_t i) { return reinterpret_cast<void*>(i << 45); }   // never read

static void copies() {
  vq_attn_desc d = {1, 1, 64, 32, 1, VQ_F16, 0.f, {VQ_E4M3}};
  for (int round = 0; round < 40; ++round) {
    d.n_pages = 2 + vq::rng() % (round < 30 ? 30 : 2000);
    d.kv_heads = d.heads = 1 + vq::rng() % 3;
    const size_t codes = (size_t)d.kv_heads * 64 * 32, scales = (size_t)d.kv_heads * 8, size = d.n_pages * (codes + scales);
    size_t said = 0;
    REQUIRE(vq_cache_bytes(&d, &said) == VQ_OK && said == size);
    const int n_buffers = 1 + vq::rng() % 3, n_pairs = 1 + vq::rng() % (round < 30 ? 60 : 3000);
    std::vector<std::vector<char>> want(n_buffers, std::vector<char>(size));
    std::vector<void*> raw;
    for (auto& b : want) {
      for (auto& c : b) c = (char)vq::rng();
      raw.push_back(std::aligned_alloc(16, (size + 15) / 16 * 16));
      std::memcpy(raw.back(), b.data(), size);
    }
    std::vector<int32_t> pairs;
    for (int i = 0; i < n_pairs; ++i) {
      const size_t from = vq::rng() % d.n_pages, to = vq::rng() % d.n_pages;
      pairs.push_back((int32_t)from);
      pairs.push_back((int32_t)to);
      for (auto& b : want) {
        std::memmove(&b[to * codes], &b[from * codes], codes);
        std::memmove(&b[d.n_pages * codes + to * scales], &b[d.n_pages * codes + from * scales], scales);
      }
    }
    REQUIRE(vq_cache_copy(&d, n_buffers, raw.data(), n_pairs, pairs.data(), nullptr) == VQ_OK);
    for (int b = 0; b < n_buffers; ++b) {
      REQUIRE(std::memcmp(raw[b], want[b].data(), size) == 0);
      std::free(raw[b]);
    }
  }
}

int main() {
  const int dims[] = {64, 96, 128, 256}, pages[] = {16, 32, 64, 128};
  auto log_int = [&](long long most) { return 1 + (int)((long long)(vq::rng() % (1u << (1 + vq::rng() % 31))) % most); };
  copies();
  long long served = 0;
  for (int i = 0; i < 20000; ++i) {
    vq_attn_desc d = {};
    d.kv_heads = vq::rng() % 2 ? log_int(64) : log_int(8);
    d.heads = d.kv_heads * log_int(1024 / d.kv_heads < 100 ? 1024 / d.kv_heads : 100);
    d.head_dim = dims[vq::rng() % 4];
    d.page_size = pages[vq::rng() % 4];
    d.n_pages = log_int(2147483647);
    d.dtype = vq::rng() % 2 ? VQ_F16 : VQ_BF16;
    d.cache_dtype = vq::rng() % 2 ? VQ_E4M3 : 0;
    d.scale = 0.1f;
    vq::g_desc = d;
    vq_attn_batch large = {};
    large.n_seqs = log_int(vq::rng() % 2 ? 65535 : 300);
    large.n_tokens = vq::rng() % 3 ? log_int(1 << 20) : large.n_seqs;
    large.table_width = (1 << 29) / d.page_size;
    large.max_len = log_int(vq::rng() % 2 ? 1 << 29 : 20000);
    large.kv_len = (const int32_t*)at(1);
    large.page_table = (const int32_t*)at(2);
    large.q_start = (const int32_t*)at(3);
    size_t n = 0;
    if (vq_attn_workspace_bytes(&d, &large, &n) != VQ_OK) continue;
    vq::g_workspace = n;
    for (int j = 0; j < 20; ++j) {
      vq_attn_batch b = large;
      if (vq::rng() % 3) b.n_seqs = 1 + vq::rng() % large.n_seqs;
      if (vq::rng() % 3) b.n_tokens = vq::rng() % 2 ? log_int(large.n_tokens) : 1 + vq::rng() % large.n_tokens;
      if (vq::rng() % 3) b.max_len = vq::rng() % 2 ? log_int(large.max_len) : vq::rng() % (large.max_len + 1u);
      vq::g_window = {vq::rng() % 4 ? log_int(1 << 29) : 0, vq::rng() % 2 ? 0 : vq::rng() % 4 ? (int)(vq::rng() % 200) : log_int(1 << 29)};
      const vq_attn_window* w = vq::g_window.window ? &vq::g_window : nullptr;
      const int st = w ? vq_attn_prompt_window(&d, &b, w, at(4), nullptr, at(5), at(6), at(7), nullptr, nullptr, at(9), n, nullptr)
                       : vq_attn_prompt(&d, &b, at(4), nullptr, at(5), at(6), at(7), nullptr, nullptr, at(9), n, nullptr);
      REQUIRE(st == VQ_OK);
      REQUIRE(vq_cache_append(&d, &b, at(4), nullptr, at(5), nullptr, at(6), at(7), nullptr) == VQ_OK);
      b.n_seqs = b.n_tokens = b.n_seqs < b.n_tokens ? b.n_seqs : b.n_tokens;
      const int one = w ? vq_attn_decode_window(&d, &b, w, at(4), nullptr, at(5), at(6), at(7), nullptr, nullptr, at(9), n, nullptr)
                        : vq_attn_decode(&d, &b, at(4), nullptr, at(5), at(6), at(7), nullptr, nullptr, at(9), n, nullptr);
      REQUIRE(one == VQ_OK);
      served += 2;
    }
  }
  REQUIRE(served > 100000 && vq::g_launches > served);
  std::printf("host check ok\n");
  return 0;
}
