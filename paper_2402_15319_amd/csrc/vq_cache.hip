// The pages of the key-value cache: new tokens into them, and copies of them.
#include "vq_attn_device.h"

namespace vq {
namespace {

// One workgroup per (token, key/value head).
__global__ __launch_bounds__(64) void append_kernel(const AppendArgs a, int head_dim) {
  const int t = blockIdx.x, h = blockIdx.y;
  const int s = sequence_of(a.c, t);
  int first, last;
  rows_of(a.c, s, &first, &last);
  const int pos = cached_tokens(a.c, s) - last + t;
  if (t < first || t >= last || pos < 0) return;
  const int page = a.c.table[(int64_t)s * a.c.table_width + (pos >> a.c.page_shift)];
  if ((uint32_t)page >= (uint32_t)a.c.n_pages) return;
  const int size = 1 << a.c.page_shift, slot = pos & (size - 1);
  const int64_t base = ((int64_t)page * a.c.kv_heads + h) * size * head_dim;
  for (int d = threadIdx.x; d < head_dim; d += 64) {
    a.k_pages[base + slot * head_dim + d] = a.k[t * a.ks.token + h * a.ks.head + d * a.ks.dim];
    a.v_pages[base + d * size + slot] = a.v[t * a.vs.token + h * a.vs.head + d * a.vs.dim];
  }
}

// One workgroup per (pair, buffer).
__global__ __launch_bounds__(256) void copy_kernel(const CopyArgs a) {
  char* base = (char*)a.buffer[blockIdx.y];
  const uint4* from = (const uint4*)(base + (uint64_t)a.from_to[blockIdx.x][0] * a.page_bytes);
  uint4* to = (uint4*)(base + (uint64_t)a.from_to[blockIdx.x][1] * a.page_bytes);
  for (uint64_t i = threadIdx.x; i < a.page_bytes / 16; i += 256) to[i] = from[i];
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, int head_dim, hipStream_t s) {
  append_kernel<<<dim3(a.c.n_tokens, a.c.kv_heads), 64, 0, s>>>(a, head_dim);
  return hipGetLastError();
}

hipError_t launch_copy(const CopyArgs& a, hipStream_t s) {
  copy_kernel<<<dim3(a.n_pairs, a.n_buffers), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace vq
