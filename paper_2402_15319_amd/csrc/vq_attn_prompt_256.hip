// Causal attention of prompts: heads of 256.  Their accumulators and the rest take more than the 256 vector registers an
// instruction can name, so this source is compiled with the accumulators in the others.
#include "vq_attn_prompt_impl.h"

namespace vq {

hipError_t launch_attn_prompt_256(const PromptArgs& a, bool bf16, hipStream_t s) {
  return bf16 ? launch_prompt<true, 256>(a, s) : launch_prompt<false, 256>(a, s);
}

}  // namespace vq
