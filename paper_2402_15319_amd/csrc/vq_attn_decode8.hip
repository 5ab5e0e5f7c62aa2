// Attention of one new token of every sequence over the paged cache: pages in 8 bits.
#include "vq_attn_decode_impl.h"

namespace vq {
namespace {

template <bool BF16, int D, bool WHOLE_LINES, int kWaves, int TILES>
__global__ __launch_bounds__(64 * kWaves, D == 256 ? 1 : 2) void decode8_kernel(const DecodeArgs A) {
  decode_body<BF16, D, WHOLE_LINES, kWaves, TILES, true, true>(A);
}

struct Kernels {
  static constexpr int kWholeLines = 6, kThreeDim = kThreeDim8;
  static constexpr bool kEightWaves = false;
  template <bool BF16, int D, bool WHOLE_LINES, int kWaves, int TILES>
  static constexpr auto kernel = decode8_kernel<BF16, D, WHOLE_LINES, kWaves, TILES>;
};

}  // namespace

hipError_t launch_attn_decode8(const DecodeArgs& a, int head_dim, bool bf16, hipStream_t s) {
  return launch_any<Kernels>(a, head_dim, bf16, s);
}

}  // namespace vq
