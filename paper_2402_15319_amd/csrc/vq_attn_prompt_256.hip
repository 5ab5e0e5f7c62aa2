// Causal attention of prompts: pages in 16 bits, every earlier token, heads of 256.  Their accumulators and the rest take more than the 256 vector registers an
// instruction can name, so this source is compiled with the accumulators in the others.
#include "vq_attn_prompt_impl.h"

namespace vq {
namespace {

template <bool BF16, int D, int TEAMS>
__global__ __launch_bounds__(64 * kWaves * TEAMS, D == 256 ? 1 : 2) void prompt_kernel(const PromptArgs A) {
  prompt_body<BF16, D, TEAMS, false, false>(A);
}

struct Kernels {
  template <bool BF16, int D, int TEAMS>
  static constexpr auto kernel = prompt_kernel<BF16, D, TEAMS>;
};

}  // namespace

hipError_t launch_attn_prompt_256(const PromptArgs& a, bool bf16, hipStream_t s) {
  return bf16 ? launch_prompt<Kernels, true, 256>(a, s) : launch_prompt<Kernels, false, 256>(a, s);
}

}  // namespace vq
