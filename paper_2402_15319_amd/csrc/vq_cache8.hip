// New tokens' keys and values into pages in 8 bits.
#include "vq_attn_device.h"

namespace vq {
namespace {

typedef u32x4 __attribute__((aligned(2))) u32x4_any;   // eight values wherever they lie
typedef short s16x2 __attribute__((ext_vector_type(2)));

// Two values over a power of two, rounded to codes (nearest, ties to even) in the lower or upper half of a dword; what is no finite number becomes NaN.
template <bool BF16, bool HIGH> __device__ __forceinline__ uint32_t codes2(uint32_t old, uint32_t pair, float scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  const s16x2 o = __builtin_bit_cast(s16x2, old);
  if constexpr (BF16) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(o, __builtin_bit_cast(bf16x2, pair), scale, HIGH));
  else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(o, __builtin_bit_cast(f16x2, pair), scale, HIGH));
}
template <bool BF16> __device__ __forceinline__ u32x2 codes8(u32x4 v, float scale) {
  return {codes2<BF16, true>(codes2<BF16, false>(0, v[0], scale), v[1], scale), codes2<BF16, true>(codes2<BF16, false>(0, v[2], scale), v[3], scale)};
}

// Magnitudes as 16-bit integers, which order as the numbers do.  1.875 * 2^15, or 2^127, is the largest whose nearest code at the largest scale is still
// one of the type; 448 is 1.75 * 2^8.
template <bool BF16> constexpr uint32_t kMost = BF16 ? 0x7f70 : 0x7b80;
template <bool BF16> constexpr uint32_t kInfinite = BF16 ? 0x7f80 : 0x7c00;

// The largest magnitude of the lane's values, as they count for a scale; those beyond the type's codes are brought into their range.
template <bool BF16, int N> __device__ __forceinline__ uint32_t largest(u32x4 (&x)[N]) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) most = larger2(most, x[i][j] & 0x7fff7fffu);
  most = (most & 0xffff) > most >> 16 ? most & 0xffff : most >> 16;
  if (most <= kMost<BF16>) return most;
  most = 0;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t at = j % 2 * 16, u = x[i][j / 2] >> at & 0x7fff, to = u >= kInfinite<BF16> ? 0x7fffu : u > kMost<BF16> ? kMost<BF16> : u;
      x[i][j / 2] ^= (u ^ to) << at;
      most = to < 0x7fff && to > most ? to : most;
    }
  return most;
}

// The smallest power of two, not below the type's least, that brings a magnitude to 448 or less.
template <bool BF16> __device__ __forceinline__ float scale_for(uint32_t most) {
  constexpr int kBits = BF16 ? 7 : 10, kBias = BF16 ? 127 : 15, kLeast = BF16 ? -117 : -15;
  const int e = (int)((most + ((1 << kBits) - 1 - (3 << (kBits - 2)))) >> kBits) - kBias - 8;   // one more where the fraction is over .75
  return __builtin_bit_cast(float, ((e > kLeast ? e : kLeast) + 127) << 23);
}

// Codes at a scale, rounded to a larger one.
template <bool BF16> __device__ __forceinline__ u32x2 coarser(u32x2 codes, float from, float to) {
  return codes8<BF16>(values8<BF16>(codes[0], codes[1], from), to);
}

// Eight by eight values, turned: in[i] holds (i, 0..7), out[j] (0..7, j).
__device__ __forceinline__ void turn8(const u32x4 (&in)[8], u32x4 (&out)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) out[j][i] = __builtin_amdgcn_perm(in[2 * i + 1][j / 2], in[2 * i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
}

// Where a token's head is, in heads of pages, or -1.
__device__ __forceinline__ int64_t head_of(const CacheArgs& c, int s, int pos, int h) {
  const int page = c.table[(int64_t)s * c.table_width + (pos >> c.page_shift)];
  return (uint32_t)page < (uint32_t)c.n_pages ? (int64_t)page * c.kv_heads + h : -1;
}

constexpr int octets(int d) { return d == 64 ? 8 : d == 256 ? 32 : 16; }   // lanes for a head's dimensions, 8 each (of 16, those of 96 leave 4 idle)

// Few new tokens for each sequence: the threads of a token take eight dimensions of a head's key and value each.  What bounds it is the way through
// the sequences' lengths, the table and the scale to the first store (one token of 8 sequences x 8 heads: 3.8 us, of 64
// 4.0), and for hundreds of tokens the values' single bytes, 16 or more apart (512 sequences x 8 heads: 8.6 us, 3 MB).  The threads look at the block's other
// new tokens, if there are any, for its scale; those of the first one also see to the earlier tokens' codes, where the scale grows, and to the scale.  (Another token's
// threads may find the new scale in place of the old one: theirs is the same from either.)
template <bool BF16, int D>
__global__ __launch_bounds__(256) void append8_few_kernel(const AppendArgs a) {
  constexpr int kLanes = octets(D);
  const int t = blockIdx.x, i = blockIdx.y * 256 + threadIdx.x, h = i / kLanes, d = 8 * (i % kLanes);
  const Tile tile = a.c.q_start ? tile_of(a.c, t, 1, 0, kFarBeyond) : Tile{t, 0, t, t + 1, cached_tokens(a.c, t, kFarBeyond)};
  const int s = tile.sequence, pos = tile.cached - tile.last + t;
  if (t < tile.first || t >= tile.last || pos < 0 || pos >= a.c.max_len) return;
  const int size = 1 << a.c.page_shift, slot = pos & (size - 1), in = pos & (kBlock - 1);
  // the block's new tokens, and how many earlier ones lie before them
  const int first = t - in > tile.first ? t - in : tile.first, last = t - in + kBlock < tile.last ? t - in + kBlock : tile.last;
  const int beyond = t + (a.c.max_len - pos), stop = last < beyond ? last : beyond, kept = in - (t - first);
  const bool there = h < a.c.kv_heads && d < D;
  u32x4 x[2][1] = {{{0, 0, 0, 0}}, {{0, 0, 0, 0}}};
  uint32_t most[2] = {0, 0};
  const uint16_t* k_from = a.k + h * a.ks.head + d * a.ks.dim;
  const uint16_t* v_from = a.v + h * a.vs.head + d * a.vs.dim;
  auto look = [&](int j) {
    if (there) {
      x[0][0] = gather8(k_from + j * a.ks.token, a.ks.dim);
      x[1][0] = gather8(v_from + j * a.vs.token, a.vs.dim);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t now = largest<BF16>(x[e]);
      most[e] = now > most[e] ? now : most[e];
    }
  };
#pragma unroll 1
  for (int j = first; j < stop; ++j)
    if (j != t) look(j);
  look(t);   // the last one: its values stay
  const int64_t head = there ? head_of(a.c, s, pos, h) : -1;
  const int64_t block = (head << (a.c.page_shift - 4)) + (slot >> 4);
  float old[2] = {0.f, 0.f};
  if (kept > 0 && head >= 0) {
    old[0] = a.k_scales[block];
    old[1] = a.v_scales[block];
  }
#pragma unroll
  for (int w = 1; w < kLanes; w *= 2)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t other = __shfl_xor(most[e], w);
      most[e] = other > most[e] ? other : most[e];
    }
  if (head < 0) return;
  const float scale[2] = {fmaxf(scale_for<BF16>(most[0]), old[0]), fmaxf(scale_for<BF16>(most[1]), old[1])};
  uint8_t* k = reinterpret_cast<uint8_t*>(a.k_pages) + (head << a.c.page_shift) * D + slot * D + d;
  uint8_t* v = reinterpret_cast<uint8_t*>(a.v_pages) + (head << a.c.page_shift) * D + ((int64_t)d << a.c.page_shift) + slot;
  *reinterpret_cast<u32x2*>(k) = codes8<BF16>(x[0][0], scale[0]);
  const u32x2 codes = codes8<BF16>(x[1][0], scale[1]);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e * size] = (uint8_t)(codes[e / 4] >> (e % 4 * 8));
  if (t != first) return;
  if (kept > 0 && scale[0] > old[0])
#pragma unroll 1
    for (int j = 1; j <= kept; ++j) {
      u32x2* at = reinterpret_cast<u32x2*>(k - j * D);
      *at = coarser<BF16>(*at, old[0], scale[0]);
    }
  if (kept > 0 && scale[1] > old[1])
#pragma unroll 1
    for (int e = 0; e < 8; ++e) {   // a dimension's slots of the block are read at once; other tokens may be writing theirs
      uint8_t* at = v + e * size - kept;
      const u32x4 was = *reinterpret_cast<const u32x4*>(at);
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const u32x2 now = coarser<BF16>(u32x2{was[2 * w], was[2 * w + 1]}, old[1], scale[1]);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (8 * w + j < kept) at[8 * w + j] = (uint8_t)(now[j / 4] >> (j % 4 * 8));
      }
    }
  if (d == 0) {
    a.k_scales[block] = scale[0];
    a.v_scales[block] = scale[1];
  }
}

// Any number of new tokens: a workgroup takes 64 positions of a sequence and a head, half of its waves the keys and half the values, a lane eight positions by
// eight dimensions in registers.  Where the source runs along positions a wave takes all of them and 64 dimensions, otherwise all dimensions of as many positions
// as it has lanes for.  The lanes, and in the first case the waves, that have a block exchange their largest magnitudes.  Loads are 16 bytes along whatever is
// contiguous in the source, 128 or more in a row of lanes; the lane turns its block where the page runs along the other; values' codes of whole blocks
// go through LDS to the lane that stores a dimension's 16 at once, successive dimensions in successive lanes.  Memory bounds it where rows are whole (11,700 tokens x 32
// heads of 128, pages of 16, 287 MB: 61 us, 4.7 TB/s, and 67 with values stored 8 bytes by 8 from where they are; a conversion of as many bytes in order 51).  In
// the order of the batched product the loads do, 77 us with no more traffic (201 MB read, 98 written) and 62 where sequences begin at multiples of 64 in the source and in
// the page: otherwise lines are read in two halves, and odd numbers cost 16-byte loads their alignment.  8 waves to a SIMD, loads past the caches (85 us) or stores past them do no better.  16 positions in place of 64 (a
// block to a lane) reads half lines: 44 us for 32 tokens of one sequence, 6 with 64.
constexpr int kTile8 = 64;
template <bool BF16, int D>
__global__ __launch_bounds__(128 * ((D + 63) / 64)) void append8_kernel(const AppendArgs a) {
  constexpr int kParts = (D + 63) / 64;   // waves for the dimensions
  constexpr int kLanes = octets(D);        // that share a position, where the source runs along dimensions
  __shared__ u32x4 codes_of[kParts][256];  // of values
  __shared__ uint32_t of_blocks[2 * kParts][kTile8 / kBlock];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool values = wave >= kParts;
  const int h = blockIdx.x % a.c.kv_heads;
  const Tile tile = tile_of(a.c, blockIdx.x / a.c.kv_heads, kTile8, 2, kFarBeyond);
  const int s = tile.sequence, first = tile.first, last = tile.last;
  const int behind = tile.cached - last, from = behind + first > 0 ? behind + first : 0;   // token t has position behind + t
  const int stop = tile.cached < a.c.max_len ? tile.cached : a.c.max_len;
  const int tile0 = (from / kTile8 + tile.number) * kTile8;
  if (last <= first || from >= stop || tile0 >= stop) return;        // no new token: for the whole workgroup
  // lanes: positions first where the source runs along them, dimensions first where it runs along those
  const auto along = [](const Strides& st) { return st.token == 1 && st.dim != 1; };
  const Strides st = values ? a.vs : a.ks;
  const bool along_tokens = along(st);
  const int x = along_tokens ? lane & 7 : wave % kParts * (64 / kLanes) + lane / kLanes, y = along_tokens ? lane >> 3 : lane % kLanes;
  const int pos = tile0 + 8 * x, block0 = pos & -kBlock;
  // Its dimensions: 8 y .. + 7, or, where nothing is turned, every eighth from y, so that the lanes of an instruction have successive ones.
  const bool spread = D % 64 == 0 && values && along_tokens;
  const int d = (along_tokens ? 64 * (wave % kParts) : 0) + (spread ? y : 8 * y), d_step = spread ? 8 : 1;
  const int64_t dim = st.dim * d_step;
  // Of its positions lo .. hi - 1 are new and have a place, and those before `kept` hold earlier tokens of the block.
  const bool mine = d < D && block0 < stop && block0 + kBlock > from;
  const int lo = from - pos > 0 ? from - pos : 0, hi = mine ? (stop - pos < 8 ? stop - pos : 8) : 0;
  const int kept = mine ? (lo < 8 ? lo : 8) : 0;
  const bool whole = lo == 0 && hi == 8;
  u32x4 in[8], turned[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) in[i] = {0, 0, 0, 0};
  bool by_token = true;   // in[i] is position i's dimensions; otherwise dimension i's positions
  if (lo < hi) {
    const uint16_t* src = (values ? a.v : a.k) + (int64_t)(pos - behind) * st.token + h * st.head + d * st.dim;
    if (st.dim == 1 && whole) {
#pragma unroll
      for (int i = 0; i < 8; ++i) in[i] = *reinterpret_cast<const u32x4_any*>(src + i * st.token);
    } else if (st.dim == 1) {
#pragma unroll
      for (int i = 0; i < 8; ++i) in[i] = *reinterpret_cast<const u32x4_any*>(src + (i < lo ? lo : i < hi ? i : hi - 1) * st.token);
    } else if (st.token == 1 && whole) {
      by_token = false;
#pragma unroll
      for (int i = 0; i < 8; ++i) in[i] = *reinterpret_cast<const u32x4_any*>(src + i * dim);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) in[i] = gather8(src + (i < lo ? lo : i < hi ? i : hi - 1) * st.token, dim);
    }
  }
  // (the source does not wait for the table)
  const int64_t head = mine ? head_of(a.c, s, pos, h) : -1;
  const int size = 1 << a.c.page_shift, slot = pos & (size - 1);
  float* scales = (values ? a.v_scales : a.k_scales) + (head << (a.c.page_shift - 4)) + (slot >> 4);
  const float old = head >= 0 && from > block0 ? *scales : 0.f;
  uint32_t most = largest<BF16>(in);   // (positions that are not new repeat one that is)
  auto exchange = [&](int w) {
    const uint32_t other = __shfl_xor(most, w);
    most = other > most ? other : most;
  };
  // the lanes with the block's other positions and the wave's other dimensions, then the waves with other dimensions
  if (along_tokens) {
    exchange(1);
    exchange(8);
    exchange(16);
    exchange(32);
  } else {
#pragma unroll
    for (int w = 1; w <= kLanes; w *= 2) exchange(w);
  }
  if (kParts > 1 && (along(a.ks) || along(a.vs))) {   // the same for all of the workgroup's waves, which meet here
    if (y == 0) of_blocks[wave][x >> 1] = most;   // (two lanes, the same number)
    __syncthreads();
    if (along_tokens)
#pragma unroll
      for (int i = 0; i < kParts; ++i) {
        const uint32_t other = of_blocks[(values ? kParts : 0) + i][x >> 1];
        most = other > most ? other : most;
      }
  }
  if (head < 0) return;
  const float scale = fmaxf(scale_for<BF16>(most), old);
  const bool grows = kept > 0 && scale > old;
  if (by_token == values) {
    turn8(in, turned);
#pragma unroll
    for (int i = 0; i < 8; ++i) in[i] = turned[i];
  }
  if (!values) {
    uint8_t* to = reinterpret_cast<uint8_t*>(a.k_pages) + (head << a.c.page_shift) * D + slot * D + d;
    if (whole) {
#pragma unroll
      for (int i = 0; i < 8; ++i) *reinterpret_cast<u32x2*>(to + i * D) = codes8<BF16>(in[i], scale);
    } else if (lo < hi || grows) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        u32x2* at = reinterpret_cast<u32x2*>(to + i * D);
        if (i >= lo && i < hi) *at = codes8<BF16>(in[i], scale);
        else if (grows && i < kept) *at = coarser<BF16>(*at, old, scale);
      }
    }
  } else {
    uint8_t* to = reinterpret_cast<uint8_t*>(a.v_pages) + (head << a.c.page_shift) * D + ((int64_t)d << a.c.page_shift) + slot;
    const int step = d_step * size;
    if (!along_tokens && D % 64 == 0 && __ballot(block0 >= from && block0 + kBlock <= stop) == ~0ull) {   // (lanes that have left count as 0)
      u32x4* room = &codes_of[wave - kParts][0];   // [block of the wave][dimension], an octet of dimensions turned by its number, which spreads them over the banks
#pragma unroll
      for (int i = 0; i < 8; ++i)
        *reinterpret_cast<u32x2*>(reinterpret_cast<char*>(room + lane / (2 * kLanes) * D + d + ((i + y) & 7)) + (x & 1) * 8) = codes8<BF16>(in[i], scale);
      asm volatile("" ::: "memory");   // (a wave's own LDS operations are in order)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int at = 64 * j + lane, b = at / D, e = at % D, dim = (e & -8) + ((e - (e >> 3)) & 7);
        const int64_t base = __shfl((int64_t)(head << a.c.page_shift) * D + (slot & -kBlock), b * 2 * kLanes);
        *reinterpret_cast<u32x4*>(reinterpret_cast<uint8_t*>(a.v_pages) + base + ((int64_t)dim << a.c.page_shift)) = room[at];
      }
    } else if (whole) {
#pragma unroll
      for (int i = 0; i < 8; ++i) *reinterpret_cast<u32x2*>(to + i * step) = codes8<BF16>(in[i], scale);
    } else if (lo < hi || grows) {   // other tokens' slots stay as they are
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        u32x2* at = reinterpret_cast<u32x2*>(to + i * step);
        const u32x2 was = *at, fresh = codes8<BF16>(in[i], scale), moved = grows ? coarser<BF16>(was, old, scale) : was;
        u32x2 now;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          uint32_t keep = 0, put = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            keep |= 4 * w + j < kept ? 0xffu << (8 * j) : 0u;
            put |= 4 * w + j >= lo && 4 * w + j < hi ? 0xffu << (8 * j) : 0u;
          }
          now[w] = (moved[w] & keep) | (fresh[w] & put) | (was[w] & ~keep & ~put);
        }
        *at = now;
      }
    }
  }
  if (d == 0 && pos == block0) *scales = scale;
}

template <bool BF16, int D>
hipError_t launch_dim(const AppendArgs& a, hipStream_t s) {
  // Few new tokens for each sequence: most of a tile would be empty, but each of them goes through the block's others.  (64 sequences x 32 heads of 128, rows
  // whole: one new token each 5.7 us, 13.0 in tiles; four 16.3 and 14.0.  In the order of the batched product: one 8.4 and 18.8; two 14.6 and 19.8; three 27.5
  // and 21.7.  512 sequences x 8 heads, rows whole: four 28.5 and 35.8; in the order of the product two 23.7 and 49.5, four 69.7 and 52.6.)  The host knows their mean
  // alone, so these lines are for sequences with about as many each: a chunk among single tokens goes token by token too (64 behind 63 of them, 8 heads, rows whole: 13.7 us,
  // 6.9 in tiles, in the order of the product 20.2 and 9.3; 32 heads 22.2 and 12.5, 47.1 and 17.9; 512 behind 511, 8 heads: 27.1 and 36.3, 75.2 and 55.7).  Where that
  // counts, the chunk is better appended by a call of its own.
  const int few = a.ks.dim == 1 && a.vs.dim == 1 ? 3 : 2;
  if (!a.c.q_start || a.c.n_tokens <= few * (int64_t)a.c.n_seqs)
    append8_few_kernel<BF16, D><<<dim3(a.c.n_tokens, (a.c.kv_heads * octets(D) + 255) / 256), 256, 0, s>>>(a);
  else
    append8_kernel<BF16, D><<<(unsigned)((a.c.n_tokens / kTile8 + 2 * (int64_t)a.c.n_seqs) * a.c.kv_heads), 128 * ((D + 63) / 64), 0, s>>>(a);
  return hipGetLastError();
}

template <bool BF16>
hipError_t launch_type(const AppendArgs& a, int head_dim, hipStream_t s) {
  if (head_dim == 64) return launch_dim<BF16, 64>(a, s);
  if (head_dim == 96) return launch_dim<BF16, 96>(a, s);
  if (head_dim == 128) return launch_dim<BF16, 128>(a, s);
  return launch_dim<BF16, 256>(a, s);
}

}  // namespace

hipError_t launch_append8(const AppendArgs& a, int head_dim, hipStream_t s) {
  return a.bf16 ? launch_type<true>(a, head_dim, s) : launch_type<false>(a, head_dim, s);
}

}  // namespace vq
