// The pages of the key-value cache: new tokens into them, and copies of them.
#include <stddef.h>
#include <string.h>

#include "vq_attn_device.h"

namespace vq {
namespace {

typedef u32x4 __attribute__((aligned(2))) u32x4_any;   // eight values wherever they lie: the memory takes any even address

// Eight by eight values, turned: in[i] holds (i, 0..7), out[j] (0..7, j).
__device__ __forceinline__ void turn8(const u32x4 (&in)[8], u32x4 (&out)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      out[j][i] = __builtin_amdgcn_perm(in[2 * i + 1][j / 2], in[2 * i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
}

// Where a token goes: the head's values in its page, or -1.
__device__ __forceinline__ int64_t head_of(const CacheArgs& c, int s, int pos, int h, int head_dim) {
  const int page = c.table[(int64_t)s * c.table_width + (pos >> c.page_shift)];
  if ((uint32_t)page >= (uint32_t)c.n_pages) return -1;
  return (((int64_t)page * c.kv_heads + h) << c.page_shift) * head_dim;
}

// A token at a time: a thread takes eight dimensions of a head's key and value.
__global__ __launch_bounds__(256) void append_one_kernel(const AppendArgs a, int head_dim) {
  const int t = blockIdx.x, pieces = head_dim / 8, i = blockIdx.y * 256 + threadIdx.x, h = i / pieces, d = 8 * (i - h * pieces);
  const Tile tile = a.c.q_start ? tile_of(a.c, t, 1, 0, kFarBeyond) : Tile{t, 0, t, t + 1, cached_tokens(a.c, t, kFarBeyond)};
  const int s = tile.sequence, pos = tile.cached - tile.last + t;
  if (h >= a.c.kv_heads || t < tile.first || t >= tile.last || pos < 0 || pos >= a.c.max_len) return;
  const int size = 1 << a.c.page_shift, slot = pos & (size - 1);
  const uint16_t* k = a.k + t * a.ks.token + h * a.ks.head + d * a.ks.dim;
  const uint16_t* v = a.v + t * a.vs.token + h * a.vs.head + d * a.vs.dim;
  const u32x4 kx = gather8(k, a.ks.dim), vx = gather8(v, a.vs.dim);
  const int64_t base = head_of(a.c, s, pos, h, head_dim);
  if (base < 0) return;
  *reinterpret_cast<u32x4*>(a.k_pages + base + slot * head_dim + d) = kx;
#pragma unroll
  for (int j = 0; j < 8; ++j) a.v_pages[base + (int64_t)(d + j) * size + slot] = (uint16_t)(vx[j / 2] >> (j % 2 * 16));
}

// Any number of new tokens: a workgroup takes 64 positions of a sequence and a head, half of its waves the keys and half the
// values, a lane eight positions by eight dimensions in registers.  Loads and stores are 16 bytes along whatever is contiguous, 128
// in a row of lanes; where the source runs along the other index than the page, the lane turns its block.
constexpr int kTile = 64;
template <int D>
__global__ __launch_bounds__(128 * ((D + 63) / 64)) void append_kernel(const AppendArgs a) {
  constexpr int kHalves = (D + 63) / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool values = wave >= kHalves;
  const int h = blockIdx.x % a.c.kv_heads;
  const Tile tile = tile_of(a.c, blockIdx.x / a.c.kv_heads, kTile, 2, kFarBeyond);
  const int s = tile.sequence, first = tile.first, last = tile.last;
  const int behind = tile.cached - last, from = behind + first > 0 ? behind + first : 0;   // token t has position behind + t
  // lanes: positions first where the source runs along them, dimensions first where it runs along those
  const Strides st = values ? a.vs : a.ks;
  const bool along_tokens = st.token == 1 && st.dim != 1;
  const int x = along_tokens ? lane & 7 : lane >> 3, y = along_tokens ? lane >> 3 : lane & 7;
  const int pos = (from / kTile + tile.number) * kTile + 8 * x;
  // Its dimensions: 8 y .. + 7, or, where nothing is turned, every eighth from y, so that the lanes of an instruction have successive ones.
  const bool spread = D % 64 == 0 && values && along_tokens;
  const int d = 64 * (wave % kHalves) + (spread ? y : 8 * y), d_step = spread ? 8 : 1;
  const int64_t dim = st.dim * d_step;
  const int stop = tile.cached < a.c.max_len ? tile.cached : a.c.max_len;
  const int lo = from - pos > 0 ? from - pos : 0, hi = stop - pos < 8 ? stop - pos : 8;   // its positions lo .. hi - 1 are new and have a place
  if (lo >= hi || d >= D) return;
  const int64_t base = head_of(a.c, s, pos, h, D);
  if (base < 0) return;
  const uint16_t* src = (values ? a.v : a.k) + (int64_t)(pos - behind) * st.token + h * st.head + d * st.dim;
  const bool whole = lo == 0 && hi == 8;
  u32x4 in[8], turned[8];
  bool by_token = true;   // in[i] is position i's dimensions; otherwise dimension i's positions
  if (st.dim == 1) {
#pragma unroll
    for (int i = 0; i < 8; ++i) in[i] = *reinterpret_cast<const u32x4_any*>(src + (i < lo ? lo : i < hi ? i : hi - 1) * st.token);
  } else if (st.token == 1 && whole) {
    by_token = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) in[i] = *reinterpret_cast<const u32x4_any*>(src + i * dim);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint16_t* row = src + (i < lo ? lo : i < hi ? i : hi - 1) * st.token;
      in[i] = gather8(row, dim);
    }
  }
  if (by_token == values) {
    turn8(in, turned);
#pragma unroll
    for (int i = 0; i < 8; ++i) in[i] = turned[i];
  }
  const int size = 1 << a.c.page_shift, slot = pos & (size - 1);
  if (!values) {
    uint16_t* to = a.k_pages + base + slot * D + d;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i >= lo && i < hi) *reinterpret_cast<u32x4*>(to + i * D) = in[i];
  } else {
    uint16_t* to = a.v_pages + base + (int64_t)d * size + slot;
    if (whole) {
#pragma unroll
      for (int i = 0; i < 8; ++i) *reinterpret_cast<u32x4*>(to + i * d_step * size) = in[i];
    } else {   // other tokens' slots stay as they are
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j >= lo && j < hi) to[i * d_step * size + j] = (uint16_t)(in[i][j / 2] >> (j % 2 * 16));
    }
  }
}

// One workgroup per 16 KB of a page, pair and buffer: four loads of 16 bytes a thread, then four stores.
constexpr int kPiece = 16384;
template <int PAIRS>
__global__ __launch_bounds__(256) void copy_kernel(const CopyArgsOf<PAIRS> a) {
  const int pair = blockIdx.x / a.pieces, piece = blockIdx.x - pair * a.pieces;
  char* base = (char*)a.buffer[blockIdx.y];
  const uint64_t at = (uint64_t)piece * kPiece + threadIdx.x * 16;
  const char* from = base + a.from_to[pair][0] * a.page_bytes;
  char* to = base + a.from_to[pair][1] * a.page_bytes;
  u32x4 v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (at + 4096 * i < a.page_bytes) v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from + at + 4096 * i));
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (at + 4096 * i < a.page_bytes) __builtin_nontemporal_store(v[i], reinterpret_cast<u32x4*>(to + at + 4096 * i));
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, int head_dim, hipStream_t s) {
  // Few new tokens for each sequence: most of a block of eight positions would be empty (64 sequences x 32 heads of 128, in the order of the
  // batched product: one new token each 7.6 us, 15.7 in blocks; two 11.9 and 16.2; four 19.5 and 17.5).  Few altogether: a block's
  // turn takes longer than they do (16 tokens of 8 sequences x 8 heads 5.0 and 8.5 us; 32 of one x 32 heads 5.8 and 6.0).
  if (!a.c.q_start || a.c.n_tokens <= 2 * (int64_t)a.c.n_seqs || (int64_t)a.c.n_tokens * a.c.kv_heads <= 1024) {
    append_one_kernel<<<dim3(a.c.n_tokens, (a.c.kv_heads * head_dim / 8 + 255) / 256), 256, 0, s>>>(a, head_dim);
    return hipGetLastError();
  }
  const unsigned tiles = (unsigned)((a.c.n_tokens / kTile + 2 * (int64_t)a.c.n_seqs) * a.c.kv_heads);
  if (head_dim == 64) append_kernel<64><<<tiles, 128, 0, s>>>(a);
  else if (head_dim == 96) append_kernel<96><<<tiles, 256, 0, s>>>(a);
  else if (head_dim == 128) append_kernel<128><<<tiles, 256, 0, s>>>(a);
  else append_kernel<256><<<tiles, 512, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_copy(CopyArgs& a, hipStream_t s) {
  a.pieces = (int32_t)((a.page_bytes + kPiece - 1) / kPiece);
  if (a.n_pairs <= kCopyFew) {   // few pairs: fewer bytes of arguments for each launch
    CopyArgsOf<kCopyFew> few;
    memcpy(&few, &a, offsetof(CopyArgs, from_to) + a.n_pairs * sizeof(a.from_to[0]));
    copy_kernel<kCopyFew><<<dim3(a.n_pairs * a.pieces, a.n_buffers), 256, 0, s>>>(few);
  } else {
    copy_kernel<kCopyPairs><<<dim3(a.n_pairs * a.pieces, a.n_buffers), 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace vq
