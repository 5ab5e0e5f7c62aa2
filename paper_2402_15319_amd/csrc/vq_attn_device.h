// Device-side helpers of attention over the paged cache.
#pragma once
#include "vq_attn.h"

namespace vq {

// A value of the cache's type, and back with one rounding to nearest even.
template <bool BF16> __device__ __forceinline__ float to_f32(uint16_t u) {
  if constexpr (BF16) return __builtin_bit_cast(float, (uint32_t)u << 16);
  else return (float)__builtin_bit_cast(_Float16, u);
}
template <bool BF16> __device__ __forceinline__ uint16_t from_f32(float f) {
  if constexpr (BF16) return __builtin_bit_cast(uint16_t, (__bf16)f);
  else return __builtin_bit_cast(uint16_t, (_Float16)f);
}

// Tokens in the cache of sequence s: `most` at most.
__device__ __forceinline__ int cached_tokens(const CacheArgs& c, int s, int most) {
  const int n = c.kv_len[s];
  return n < 0 ? 0 : n < most ? n : most;
}
// Attention takes a longer sequence as one of max_len tokens.  New tokens keep their positions, and those from max_len on have no place; with
// 2^30 for more than that, none of them has one (max_len is at most 2^29, there are little more than 2^27 new tokens at most) and no
// index overflows.
constexpr int kFarBeyond = 1 << 30;

// Work is handed out in tiles of `unit` new tokens of a sequence, at most floor(tokens / unit) + extra of them.  Those of
// sequence i start at slot floor(first token / unit) + extra * i, which leaves room for the last ones of the sequences before;
// this is the sequence of a slot, the slot's number among its own, the sequence's rows (new tokens) first .. last - 1 and the tokens
// in its cache (`most` at most), all inside the arrays whatever they hold.  A wave looks at 64 sequences at a time, with one wait for all of it.
struct Tile { int sequence, number, first, last, cached; };
__device__ __forceinline__ Tile tile_of(const CacheArgs& c, int slot, int unit, int extra, int most) {
  const int lane = threadIdx.x & 63;
  Tile t = {0, slot, 0, 0, 0};   // an empty sequence, where q_start does not begin with 0
  for (int base = 0; base < c.n_seqs; base += 64) {
    const int i = base + lane, in = i < c.n_seqs ? i : c.n_seqs - 1;
    int first = c.q_start ? c.q_start[in] : in, last = c.q_start ? c.q_start[in + 1] : in + 1;
    const int cached = cached_tokens(c, in, most);
    first = first < 0 ? 0 : first < c.n_tokens ? first : c.n_tokens;
    last = last < first ? first : last < c.n_tokens ? last : c.n_tokens;
    const int at = first / unit + extra * i;
    const int before = __popcll(__ballot(i < c.n_seqs && at <= slot));
    if (before == 0) break;
    t.sequence = base + before - 1;
    t.number = slot - __builtin_amdgcn_readlane(at, before - 1);
    t.first = __builtin_amdgcn_readlane(first, before - 1);
    t.last = __builtin_amdgcn_readlane(last, before - 1);
    t.cached = __builtin_amdgcn_readlane(cached, before - 1);
    if (before < 64) break;
  }
  return t;
}

// A page number from a table, moved into the cache where it lies outside.
__device__ __forceinline__ int page_inside(const CacheArgs& c, int page) {
  return (int)((uint32_t)page < (uint32_t)c.n_pages ? (uint32_t)page : (uint32_t)c.n_pages - 1);
}

// Eight values of the cache's type, the share of a lane in an operand of a matrix instruction.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

// Eight values `step` apart.
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ u32x4 gather8(const uint16_t* from, int64_t step) {
  u16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = from[i * step];
  return __builtin_bit_cast(u32x4, v);
}

// 16 x 16 += 16 x 32 . 32 x 16.  Lane L holds row (a) or column (b) L % 16 at k = 8 (L / 16) .. + 7, and of the result
// column L % 16 at rows 4 (L / 16) .. + 3.
template <bool BF16> __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// 32 x 32 += 32 x 16 . 16 x 32.  Lane L holds row (a) or column (b) L % 32 at k = 8 (L / 32) .. + 7, and of the result column
// L % 32 at rows 8 (i / 4) + 4 (L / 32) + i % 4, i < 16.
typedef float f32x16 __attribute__((ext_vector_type(16)));
template <bool BF16> __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Eight weights rounded to the cache's type: a matrix instruction takes both operands in one 16-bit type, and a weight in two halves
// would double the second product (long prompts are bound by their products).  Each weight is off by 2^-11 (fp16) or 2^-8 (bf16)
// of itself at most, the sum of the weights not: out has about that error again beside its own last rounding.
template <bool BF16> __device__ __forceinline__ u32x4 pack8(f32x8 p) {
  if constexpr (BF16) return __builtin_bit_cast(u32x4, __builtin_convertvector(p, bf16x8));
  else return __builtin_bit_cast(u32x4, __builtin_convertvector(p, f16x8));
}

// What one workgroup hands to another of the same launch goes past the caches that only some of the XCDs see: accesses of agent
// scope, two values at a time, and before the word that says so the stores' completion.  (Fences of agent scope would do the
// same for ordinary accesses, but write back and drop the XCD's whole L2: 24 sequences of 2,000 to 4,096 tokens in two parts, 1,536
// workgroups, took 802 us with them and 240 us in one part.)
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void shared_store(float* p, float a, float b) {
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), __builtin_bit_cast(uint64_t, f32x2{a, b}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 shared_load(const float* p) {
  return __builtin_bit_cast(f32x2, __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
__device__ __forceinline__ void shared_stores_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// 64 lanes x 16 bytes (base + voff, voff per lane) into 1 KB of LDS from byte address lds on.  No register takes the data; the
// wave's vmcnt counts it, the compiler does not.
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(voff), "s"(base) : "memory", "m0");
}

// The wave's loads into LDS have arrived and its reads from LDS have been answered, then the workgroup's other waves'.
__device__ __forceinline__ void lds_turn() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }   // v_exp_f32: 1 ulp

// What brings sums from one maximum to a larger one: never 0, which an infinite sum must not meet.  (The smallest number of all, so that
// outputs of bf16 close to their smallest do not feel it.)
__device__ __forceinline__ float rescale(float from, float to) { return fmaxf(exp2_fast(from - to), 0x1p-149f); }

// Stands for a sum that is no number while the values that are none are looked for; where there are none, the sum went beyond
// the range of its 32 bits, and is no number in the end.
constexpr float kUnknown = 0x1.5a5a5ap-120f;

// The halves of a dword that are no finite numbers: all ones.
template <bool BF16> __device__ __forceinline__ uint32_t odd_halves(uint32_t v) {
  constexpr uint32_t kExp = BF16 ? 0x7f807f80u : 0x7c007c00u, kOne = BF16 ? 0x00800080u : 0x04000400u;
  return (((v & kExp) + kOne) >> 15 & 0x00010001u) * 0xffffu;
}

// Weights are exp2(x - m) with m a maximum less kLift: in fp16 weights below 2^-14 lose bits, so the largest start from 2^kLift
// there.  It cancels in out and in lse.  m is left as it is until a logit is more than kSlack above the maximum it was taken from.
template <bool BF16> constexpr float kLift = BF16 ? 0.f : 6.f;
constexpr float kSlack = 8.f;

}  // namespace vq
