// Prints the plan of a call of vq_attn_prompt (tests/test_attn_long_plans.py): heads, kv_heads, head_dim, sequences, new tokens, max_len.
#include <cstdio>
#include <cstdlib>

#include "../../paper_2402_15319_amd/csrc/vq_attn.h"

namespace vq {
hipError_t launch_append(const AppendArgs&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_copy(CopyArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_attn_decode(const DecodeArgs&, int, bool, hipStream_t) { return hipSuccess; }
hipError_t launch_attn_prompt(const PromptArgs& d, int, bool, hipStream_t) {
  std::printf("%d %d %d %d %d\n", d.plan.heads, d.plan.tokens, d.plan.teams, d.plan.steps, d.plan.parts);
  return hipSuccess;
}
}  // namespace vq

int main(int argc, char** argv) {
  if (argc != 7) return 2;
  int v[6];
  for (int i = 0; i < 6; ++i) v[i] = std::atoi(argv[1 + i]);
  const auto at = [](uintptr_t i) { return reinterpret_cast<void*>(i << 20); };   // never read
  const vq_attn_desc d = {v[0], v[1], v[2], 16, 100, VQ_F16, 0.1f, 0};
  const vq_attn_batch b = {v[3], v[4], 1 << 24, v[5], (const int32_t*)at(1), (const int32_t*)at(2), (const int32_t*)at(3)};
  return vq_attn_prompt(&d, &b, at(4), nullptr, at(5), at(6), at(7), nullptr, nullptr, at(9), (size_t)1 << 40, nullptr) == VQ_OK ? 0 : 1;
}
