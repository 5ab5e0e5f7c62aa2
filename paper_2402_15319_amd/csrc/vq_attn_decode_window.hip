// Attention of one new token of every sequence over the paged cache: pages in 16 bits, a window and sinks.
#include "vq_attn_decode_impl.h"

namespace vq {
namespace {

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
