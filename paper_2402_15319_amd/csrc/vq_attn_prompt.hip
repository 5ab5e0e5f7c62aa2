// Attention over the paged cache, plainly: one wave per (new token, query head).
#include "vq_attn_device.h"

namespace vq {
namespace {

// 64 tokens at a time, one a lane, for the logits; then the lanes take dimensions and go through the 64 tokens' values.
// The running maximum and sum are those of a softmax in one pass: both, and the sums over the values, are scaled down
// whenever the maximum grows.
template <bool BF16>
__global__ __launch_bounds__(64) void attn_plain_kernel(const AttnArgs a, int head_dim) {
  const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
  const int s = sequence_of(a.c, t);
  int first, last;
  rows_of(a.c, s, &first, &last);
  if (t < first || t >= last) return;
  const int n = cached_tokens(a.c, s) - last + t + 1;   // tokens that this row attends
  const int size = 1 << a.c.page_shift;
  const uint16_t* q = a.q + t * a.qs.token + h * a.qs.head;
  float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = 0; j0 < n; j0 += 64) {
    const int j = j0 + lane;
    const int page = page_inside(a.c, a.c.table[(int64_t)s * a.c.table_width + ((j < n ? j : n - 1) >> a.c.page_shift)]);
    const int64_t base = ((int64_t)page * a.c.kv_heads + h / a.group) * size * head_dim;
    float x = -INFINITY;
    if (j < n) {
      const uint16_t* k = a.k_pages + base + (j & (size - 1)) * head_dim;
      x = 0.f;
      for (int d = 0; d < head_dim; ++d) x = fmaf(to_f32<BF16>(q[d * a.qs.dim]), to_f32<BF16>(k[d]), x);
      x *= a.scale_log2;
    }
    float top = x;
    for (int b = 1; b < 64; b <<= 1) top = fmaxf(top, __shfl_xor(top, b));
    const float m_new = fmaxf(m, top);
    const float zero = m_new == -INFINITY ? 0.f : m_new;
    const float p = exp2f(x - zero), shrink = exp2f(m - zero);
    float sum = p;
    for (int b = 1; b < 64; b <<= 1) sum += __shfl_xor(sum, b);
    l = l * shrink + sum;
    m = m_new;
    for (int i = 0; i < 4; ++i) o[i] *= shrink;
    const int most = n - j0 < 64 ? n - j0 : 64;
    for (int r = 0; r < most; ++r) {
      const float pr = __shfl(p, r);
      const int64_t from = __shfl(base, r) + ((j0 + r) & (size - 1));
      for (int i = 0; i < 4; ++i) {
        const int d = lane + 64 * i;
        if (d < head_dim) o[i] = fmaf(pr, to_f32<BF16>(a.v_pages[from + (int64_t)d * size]), o[i]);
      }
    }
  }
  uint16_t* out = a.out + t * a.os.token + h * a.os.head;
  for (int i = 0; i < 4; ++i) {
    const int d = lane + 64 * i;
    if (d < head_dim) out[d * a.os.dim] = from_f32<BF16>(n > 0 ? o[i] / l : 0.f);
  }
  if (a.lse && lane == 0) a.lse[(int64_t)t * a.heads + h] = n > 0 ? (m + log2f(l)) * 0.693147180559945f : -INFINITY;
}

}  // namespace

hipError_t launch_attn_prompt(const AttnArgs& a, int head_dim, bool bf16, hipStream_t s) {
  const dim3 grid(a.c.n_tokens, a.heads);
  if (bf16) attn_plain_kernel<true><<<grid, 64, 0, s>>>(a, head_dim);
  else attn_plain_kernel<false><<<grid, 64, 0, s>>>(a, head_dim);
  return hipGetLastError();
}

}  // namespace vq
