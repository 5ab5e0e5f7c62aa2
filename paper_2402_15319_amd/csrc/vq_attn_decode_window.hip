// Attention of one new token of every sequence over the paged cache: pages in 16 bits, a window and sinks.
#include "vq_attn_decode_impl.h"

namespace vq {
namespace {

// Bound by memory: 48 sequences of 6,400 to 12,000 tokens x 8 key/value heads of 128, window 2,048, pages of 64: 80 us for the 56 of 403 MB, in two
// parts to a sequence.  Two runs of 32 tokens in a step, so that pages of 64 are whole lines too: 84 us.
template <bool BF16, int D, bool WHOLE_LINES, int kWaves, int TILES>
__global__ __launch_bounds__(64 * kWaves, D == 256 ? 1 : 2) void decode_window_kernel(const DecodeArgs A) {
  decode_body<BF16, D, WHOLE_LINES, kWaves, TILES, false, true>(A);
}

struct Kernels {
  static constexpr int kWholeLines = 5, kThreeDim = kTogetherDim;
  static constexpr bool kEightWaves = true;
  template <bool BF16, int D, bool WHOLE_LINES, int kWaves, int TILES>
  static constexpr auto kernel = decode_window_kernel<BF16, D, WHOLE_LINES, kWaves, TILES>;
};

}  // namespace

hipError_t launch_attn_decode_window(const DecodeArgs& a, int head_dim, bool bf16, hipStream_t s) {
  return launch_any<Kernels>(a, head_dim, bf16, s);
}

}  // namespace vq
