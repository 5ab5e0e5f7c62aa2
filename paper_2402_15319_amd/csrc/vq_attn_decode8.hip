// Attention of one new token of every sequence over the paged cache: pages in 8 bits.
#include "vq_attn_decode_impl.h"

namespace vq {
namespace {

// Bound by memory where sequences are many or long, at the rate of 16 bits with half the bytes: 40 sequences of 2,000 to 4,096 tokens x 32 heads of 128 164 us,
// 5.9 TB/s; 130,001 tokens x 8 48 us, 5.6.  One of 401 x 32 is latency, 6.6 us.  Two waves to a SIMD: for three (168 registers) 12 bytes would be spilled, 184
// us for 164.  K past the caches 173, V through them 179, both asked for at a step's end 167.
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
