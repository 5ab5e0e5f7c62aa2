// Causal attention of prompts: heads of 64, 96 and 128.
#include "vq_attn_prompt_impl.h"

namespace vq {
namespace {

template <bool BF16>
hipError_t launch_type(const PromptArgs& a, int head_dim, hipStream_t s) {
  if (head_dim == 64) return launch_prompt<BF16, 64>(a, s);
  if (head_dim == 96) return launch_prompt<BF16, 96>(a, s);
  return launch_prompt<BF16, 128>(a, s);
}

}  // namespace

hipError_t launch_attn_prompt(const PromptArgs& a, int head_dim, bool bf16, hipStream_t s) {
  if (head_dim == 256) return launch_attn_prompt_256(a, bf16, s);
  return bf16 ? launch_type<true>(a, head_dim, s) : launch_type<false>(a, head_dim, s);
}

}  // namespace vq
