// Attention of one new token of every sequence over the paged cache: pages in 16 bits, every token.
#include "vq_attn_decode_impl.h"

namespace vq {
namespace {

template <bool BF16, int D, bool WHOLE_LINES, int kWaves, int TILES>
__global__ __launch_bounds__(64 * kWaves, D == 256 ? 1 : 2) void decode_kernel(const DecodeArgs A) {
  decode_body<BF16, D, WHOLE_LINES, kWaves, TILES, false, false>(A);
}

struct Kernels {
  static constexpr int kWholeLines = 5, kThreeDim = kTogetherDim;
  static constexpr bool kEightWaves = true;
  template <bool BF16, int D, bool WHOLE_LINES, int kWaves, int TILES>
  static constexpr auto kernel = decode_kernel<BF16, D, WHOLE_LINES, kWaves, TILES>;
};

}  // namespace

hipError_t launch_attn_decode(const DecodeArgs& a, int head_dim, bool bf16, hipStream_t s) {
  if (a.a.k_scales) return launch_attn_decode8(a, head_dim, bf16, s);
  if (a.a.window > 0) return launch_attn_decode_window(a, head_dim, bf16, s);
  return launch_any<Kernels>(a, head_dim, bf16, s);
}

}  // namespace vq
