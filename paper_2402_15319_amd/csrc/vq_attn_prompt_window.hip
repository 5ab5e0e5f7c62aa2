// Causal attention of prompts: pages in 16 bits, a window and sinks, heads of 64, 96 and 128.
#include "vq_attn_prompt_impl.h"

namespace vq {
namespace {

// 5,000 tokens, window 1,024, 32 heads on 8 of 128: 103 us at the rate of long prompts (40 % of the matrix units' time), with 17 steps to a tile where 16 are seen.
// Nine prompts of up to 2,500, window 333, 32 heads of 96: 79 us; seven or eight steps to a tile, half of them with a mask, and a beginning and an end that take
// as long as four.  Three steps in LDS took 5 % longer, two teams 25 %.
template <bool BF16, int D, int TEAMS>
__global__ __launch_bounds__(64 * kWaves * TEAMS, D == 256 ? 1 : 2) void prompt_window_kernel(const PromptArgs A) {
  prompt_body<BF16, D, TEAMS, false, true>(A);
}

struct Kernels {
  template <bool BF16, int D, int TEAMS>
  static constexpr auto kernel = prompt_window_kernel<BF16, D, TEAMS>;
};

}  // namespace

hipError_t launch_attn_prompt_window(const PromptArgs& a, int head_dim, bool bf16, hipStream_t s) {
  if (head_dim == 256) return launch_attn_prompt_window_256(a, bf16, s);
  return bf16 ? launch_prompt_small<Kernels, true>(a, head_dim, s) : launch_prompt_small<Kernels, false>(a, head_dim, s);
}

}  // namespace vq
