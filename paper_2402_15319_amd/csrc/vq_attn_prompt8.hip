// Causal attention of prompts: pages in 8 bits, heads of 64, 96 and 128.
#include "vq_attn_prompt_impl.h"

namespace vq {
namespace {

// 4,096 tokens x 32 heads of 128: 160 to 168 us by the card, 845 TFLOP/s at 163, 42 % of the matrix units' time, and 4 to 7 % behind 16 bits, whose K and V go to LDS past the registers:
// codes stored before a step's products 180 us, behind them 179, and from places that are kept and without bank conflicts 163 to 168.
template <bool BF16, int D, int TEAMS>
__global__ __launch_bounds__(64 * kWaves * TEAMS, D == 256 ? 1 : 2) void prompt8_kernel(const PromptArgs A) {
  prompt_body<BF16, D, TEAMS, true, true>(A);
}

struct Kernels {
  template <bool BF16, int D, int TEAMS>
  static constexpr auto kernel = prompt8_kernel<BF16, D, TEAMS>;
};

}  // namespace

hipError_t launch_attn_prompt8(const PromptArgs& a, int head_dim, bool bf16, hipStream_t s) {
  if (head_dim == 256) return launch_attn_prompt8_256(a, bf16, s);
  return bf16 ? launch_prompt_small<Kernels, true>(a, head_dim, s) : launch_prompt_small<Kernels, false>(a, head_dim, s);
}

}  // namespace vq
