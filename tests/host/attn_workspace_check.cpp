// The workspace of attention over the paged cache (tests/test_attn_workspace.py): one that was sized for a batch serves every batch of
// no more sequences, new tokens and tokens in a sequence.  Stand-ins for the kernel launchers check that each launch stays inside.
#include <cstdio>
#include <cstdlib>
#include <random>

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
hipError_t launch_append(const AppendArgs&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_copy(CopyArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_attn_decode(const DecodeArgs& d, int head_dim, bool, hipStream_t) {
  const DecodePlan& p = d.plan;
  const size_t units = (size_t)d.a.c.n_seqs * d.a.c.kv_heads * p.tiles;
  if (p.parts > 1) REQUIRE((size_t)((char*)d.part - (char*)d.counter) + units * p.parts * part_floats(p, head_dim) * 4 <= g_workspace);
  return hipSuccess;
}
hipError_t launch_attn_prompt(const PromptArgs& d, int head_dim, bool, hipStream_t) {
  const PromptPlan& p = d.plan;
  const size_t units = (size_t)p.slots * (d.a.heads / p.heads);
  if (p.parts > 1) REQUIRE((size_t)((char*)d.part - (char*)d.counter) + units * p.parts * prompt_part_floats(head_dim) * 4 <= g_workspace);
  return hipSuccess;
}
}  // namespace vq

static void* at(uintptr_t i) { return reinterpret_cast<void*>(i << 20); }   // never read

int main() {
  std::mt19937 rng(3);
  const int dims[] = {64, 96, 128, 256}, pages[] = {16, 32, 64, 128};
  auto log_int = [&](long long most) { return 1 + (int)((long long)(rng() % (1u << (1 + rng() % 31))) % most); };
  long long served = 0;
  for (int i = 0; i < 30000; ++i) {
    vq_attn_desc d = {};
    d.kv_heads = rng() % 2 ? log_int(64) : log_int(8);
    d.heads = d.kv_heads * log_int(1024 / d.kv_heads < 100 ? 1024 / d.kv_heads : 100);
    d.head_dim = dims[rng() % 4];
    d.page_size = pages[rng() % 4];
    d.n_pages = 1000;
    d.dtype = VQ_F16;
    d.scale = 0.1f;
    vq_attn_batch large = {};
    large.n_seqs = log_int(rng() % 2 ? 65535 : 300);
    large.n_tokens = rng() % 3 ? log_int(1 << 20) : large.n_seqs;
    large.table_width = (1 << 29) / d.page_size;
    large.max_len = log_int(rng() % 2 ? 1 << 29 : 20000);
    large.kv_len = (const int32_t*)at(1);
    large.page_table = (const int32_t*)at(2);
    large.q_start = (const int32_t*)at(3);
    size_t n = 0;
    if (vq_attn_workspace_bytes(&d, &large, &n) != VQ_OK) continue;
    vq::g_workspace = n;
    for (int j = 0; j < 40; ++j) {
      vq_attn_batch b = large;
      if (rng() % 3) b.n_seqs = rng() % 2 ? log_int(large.n_seqs) : 1 + rng() % large.n_seqs;
      if (rng() % 3) b.n_tokens = rng() % 2 ? log_int(large.n_tokens) : 1 + rng() % large.n_tokens;
      if (rng() % 3) b.max_len = rng() % 2 ? log_int(large.max_len) : 1 + rng() % large.max_len;
      if (rng() % 3 == 0 && b.n_tokens < b.n_seqs) b.n_seqs = b.n_tokens;
      if (rng() % 3 == 0 && b.n_seqs < b.n_tokens) b.n_tokens = b.n_seqs;
      size_t less = 0;
      REQUIRE(vq_attn_workspace_bytes(&d, &b, &less) == VQ_OK && less <= n);
      REQUIRE(vq_attn_prompt(&d, &b, at(4), nullptr, at(5), at(6), at(7), nullptr, nullptr, at(9), n, nullptr) == VQ_OK);
      if (b.n_tokens == b.n_seqs) REQUIRE(vq_attn_decode(&d, &b, at(4), nullptr, at(5), at(6), at(7), nullptr, nullptr, at(9), n, nullptr) == VQ_OK);
      ++served;
    }
  }
  REQUIRE(served > 500000);
  std::printf("workspace check ok\n");
  return 0;
}
