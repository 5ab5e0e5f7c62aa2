// Attention of one new token of every sequence over the paged cache: the kernels' body.
#pragma once
#include <type_traits>

#include "vq_attn_device.h"

namespace vq {
namespace {

// One workgroup: `chunk` tokens of a sequence, the query heads of TILES tiles of up to 16.  Its waves take 32 tokens at a time in turn, 64 of
// pages in 8 bits: a lane's tokens are kOwn = 8 or 16, the bytes of one load.
//   S^T = K Q^T: an instruction's rows are 16 tokens, its columns the query heads.  The rows' tokens are chosen so that lane
//   L ends up with the logits of tokens kOwn (L / 16) .. + kOwn - 1 of head L % 16, which is just the operand (or two) that
//   O^T += V^T P^T takes: neither product moves anything between lanes, and a page's V is laid out so that V^T is read as it lies.
// m and the sums are those of a softmax in one pass; a lane adds up its own weights until the end.
// WHOLE_LINES: pages of at most 32 tokens (64 in 8 bits), whose V a load reads in whole lines of memory that nobody reads again: they pass the
// caches by (24 sequences of 2,000 to 4,096 tokens x 32 heads, pages of 16: 195 us, 217 without).  In larger pages a step's 64 bytes of a row of
// V^T are half a line, and the wave with the other half wants it kept (130,001 tokens, pages of 64: 95 us, 107 if not); the
// same holds for K, whose rows four instructions read in turn.
// TILES: more than 16 query heads share what is read of their key/value head (64 sequences of 4,096 to 8,192, 48 heads to one of 128: 59 us,
// 118 a tile to a workgroup).
// E4M3: pages in 8 bits.  A lane's tokens are one block, so that it has one scale for its keys and one for its values in a step; codes become
// values of the type, exactly, in one instruction for two (scale included), and everything behind that is as in 16 bits.
// WINDOW: a.window and a.sinks.  What no row sees between the sinks and the window, in whole steps, is passed over: `t` below counts the
// tokens that are gone through, real(t) is the place of one in its sequence.
template <bool BF16, int D, bool WHOLE_LINES, int kWaves, int TILES, bool E4M3, bool WINDOW>
__device__ __forceinline__ void decode_body(const DecodeArgs& A) {
  constexpr int KS = D / 32, DT = D / 16;
  constexpr int kOwn = E4M3 ? 16 : 8, kStep = 4 * kOwn;             // tokens of a lane, and of a wave, in a step
  constexpr int NS = kOwn / 4, NV = kOwn / 8;                       // instructions for a step's logits, and for its values, for each fragment
  constexpr int KF = E4M3 ? (D + 63) / 64 : KS;                     // loads of a lane for a token's keys: 16 bytes each, 8 the last one of 96 codes
  const AttnArgs& a = A.a;
  const int part = blockIdx.z, s = blockIdx.y;
  const int beside = (A.plan.tiles + TILES - 1) / TILES, kvh = blockIdx.x / beside, tile0 = (blockIdx.x - kvh * beside) * TILES;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int len = cached_tokens(a.c, s, a.c.max_len);
  // The window's first token; tokens low_end .. low_end + skip - 1 are passed over.
  int first_seen = 0, low_end = 0, skip = 0;
  if constexpr (WINDOW) {
    first_seen = len > a.window ? len - a.window : 0;
    low_end = ((a.sinks < len ? a.sinks : len) + kStep - 1) & -kStep;
    skip = (first_seen & -kStep) - low_end;
    skip = skip > 0 ? skip : 0;
  }
  auto real = [&](int t) { return WINDOW && t >= low_end ? t + skip : t; };
  const int all = len - skip, begin = part * A.plan.chunk;
  if (begin >= all && part > 0) return;
  const int end = all - begin < A.plan.chunk ? all : begin + A.plan.chunk;
  const int h0 = kvh * a.group + tile0 * kTileHeads;                // first query head
  const int heads = a.group - tile0 * kTileHeads;                   // how many there are from it
  const int shift = a.c.page_shift, mask = (1 << shift) - 1;

  // The pages of the first step, asked for before q (16 sequences of up to 600 tokens over 8-bit pages: 8.1 us, 8.3 behind it; with three tiles of heads
  // it would be 20 bytes of scratch more).
  constexpr int kStride = kStep * kWaves;
  const int last_page = len > 0 ? (len - 1) >> shift : 0, k_run = (col >> 2) * kOwn;
  const int32_t* table = a.c.table + (int64_t)s * a.c.table_width;
  auto page_at = [&](int t) { return table[t >> shift < last_page ? t >> shift : last_page]; };
  int k_page = 0, v_page = 0, t0 = begin + kStep * wave;
  auto first_pages = [&]() {
    if (t0 >= end) return;
    k_page = page_at(real(t0) + k_run);
    v_page = page_at(real(t0) + kOwn * g);
  };
  if constexpr (TILES < 3) first_pages();
  // The lane's dimensions of fragment k: 8 of 32, or, where a load brings 16 codes, those of two fragments side by side.
  auto q_dim = [&](int k) { return E4M3 && k < D / 64 * 2 ? 64 * (k / 2) + 16 * g + 8 * (k % 2) : 32 * k + 8 * g; };
  u32x4 q[TILES][KS];
  const bool whole_rows = a.qs.dim == 1 && ((a.qs.token | a.qs.head) & 7) == 0;
  // Any other order: each value is fetched once for the workgroup and goes through LDS (61 sequences, 8 heads to a key/value head, the
  // tokens next to one another: 66 us, 79 with every wave fetching all).
  constexpr int kRow = D + 8;   // of q in LDS: 16 rows' pieces in different banks
  __shared__ __attribute__((aligned(16))) uint16_t q_rows[TILES * kTileHeads * kRow];
  if (!whole_rows) {
    const int rows = heads < TILES * kTileHeads ? heads : TILES * kTileHeads;
    const uint16_t* at = a.q + s * a.qs.token + h0 * a.qs.head;
    for (int i = tid; i < rows * D; i += 64 * kWaves) q_rows[i / D * kRow + i % D] = at[i / D * a.qs.head + i % D * a.qs.dim];
    __syncthreads();
  }
  auto load_q = [&]() {
#pragma unroll
    for (int n = 0; n < TILES; ++n) {
#pragma unroll
      for (int k = 0; k < KS; ++k) q[n][k] = {0, 0, 0, 0};
      if (16 * n + col >= heads) continue;
      if (whole_rows) {
        const uint16_t* row = a.q + s * a.qs.token + (h0 + 16 * n + col) * a.qs.head;
#pragma unroll
        for (int k = 0; k < KS; ++k) q[n][k] = *reinterpret_cast<const u32x4*>(row + q_dim(k));
      } else {
#pragma unroll
        for (int k = 0; k < KS; ++k) q[n][k] = *reinterpret_cast<const u32x4*>(&q_rows[(16 * n + col) * kRow + q_dim(k)]);
      }
    }
  };
  load_q();
  if constexpr (TILES >= 3) first_pages();

  const int64_t head_page = (int64_t)D << shift;                    // values of a head in a page
  // Where the lane's rows of K (kOwn tokens of a page: row L % 16 is token kOwn (L % 16 / 4) + L % 4, and 4 more in each further
  // instruction) and its kOwn tokens of V^T start, for the tokens at t0.
  const int k_in = col & 3;
  u32x4 kf[NS][KF], vf[DT];
  float k_scale = 1.f, v_scale = 1.f;                               // E4M3: of the lane's keys and of its values
  auto scale_at = [&](int page, int t) { return (((int64_t)page_inside(a.c, page) * a.c.kv_heads + kvh) << (shift - 4)) + ((t & mask) >> 4); };
  // (Behind the last step there is nothing to load: all lanes then read the same 16 bytes of the buffer's first page, so that the loop
  // is one stretch of code in which every wait knows what is under way.)
  auto load_k = [&](int t, int page, bool there) {
    const int64_t at = ((int64_t)page_inside(a.c, page) * a.c.kv_heads + kvh) * head_page + (((t + k_run) & mask) + k_in) * D;
    if constexpr (E4M3) {
      const uint8_t* pages = reinterpret_cast<const uint8_t*>(a.k_pages);
      const uint8_t* base = there ? pages + at + 16 * g : pages;
      k_scale = a.k_scales[there ? scale_at(page, t + k_run) : 0];
#pragma unroll
      for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int k = 0; k < KF; ++k) {
          const uint8_t* from = base + 4 * i * D + 64 * k;
          if (k < D / 64) {
            kf[i][k] = *reinterpret_cast<const u32x4*>(from);
          } else {   // the last 32 dimensions: 8 a lane
            const u32x2 u = *reinterpret_cast<const u32x2*>(there ? from - 8 * g : from);
            kf[i][k] = {u[0], u[1], 0, 0};
          }
        }
    } else {
      const uint16_t* base = a.k_pages + at + 8 * g;
      base = there ? base : a.k_pages;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        kf[0][k] = *reinterpret_cast<const u32x4*>(base + 32 * k);
        kf[1][k] = *reinterpret_cast<const u32x4*>(base + 4 * D + 32 * k);
      }
    }
  };
  // (What is the lane's own within a page goes into 32 bits: as part of an address of 64 it took two registers of three tiles' through scratch, which every step waited
  // for: 64 sequences of 4,096 to 8,192, 48 heads of 128 to one, 73 us for 68.)
  auto load_v = [&](int t, int page, bool there) {
    const int64_t at = ((int64_t)page_inside(a.c, page) * a.c.kv_heads + kvh) * head_page + (uint32_t)(col << shift | ((t + kOwn * g) & mask));
    typedef typename std::conditional<E4M3, uint8_t, uint16_t>::type Code;
    const Code* pages = reinterpret_cast<const Code*>(a.v_pages);
    const Code* base = pages + at;
    base = there ? base : pages;
    if constexpr (E4M3) v_scale = a.v_scales[there ? scale_at(page, t + kOwn * g) : 0];
#pragma unroll
    for (int i = 0; i < DT; ++i) {
      const u32x4* from = reinterpret_cast<const u32x4*>(base + ((int64_t)(16 * i) << shift));
      if constexpr (WHOLE_LINES) vf[i] = __builtin_nontemporal_load(from);
      else vf[i] = *from;
    }
  };
  // Fragment k of instruction i's keys, and the values of fragment h (8 of the lane's tokens) of dimensions 16 i ..
  auto k_fragment = [&](int i, int k) {
    if constexpr (E4M3) return values8<BF16>(kf[i][k / 2][k % 2 * 2], kf[i][k / 2][k % 2 * 2 + 1], k_scale);
    else return kf[i][k];
  };
  auto v_fragment = [&](int i, int h) {
    if constexpr (E4M3) return values8<BF16>(vf[i][2 * h], vf[i][2 * h + 1], v_scale);
    else return vf[i];
  };
  // Of the lane's tokens at t0 those from `last` on are unseen, and those from `low` to `first`; whether there are any among the wave's.
  struct Unseen {
    int last, low, first;
    __device__ __forceinline__ bool seen(int i) const { return i < last && (!WINDOW || i >= first || i < low); }
  };
  auto unseen_at = [&](int t0) {
    const int t = t0 + kOwn * g;
    return Unseen{len - t, WINDOW ? a.sinks - t : 0, WINDOW ? first_seen - t : 0};
  };
  auto masked = [&](int t0) { return t0 + kStep > len || (WINDOW && t0 < first_seen && t0 + kStep > a.sinks); };
  // What is no number in another token's place must not meet even a weight of 0: cleared.
  auto clear_unseen = [&](const Unseen& u) {
    if constexpr (E4M3) {
      u32x4 keep = {0, 0, 0, 0};
      bool any = false;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        keep[i / 4] |= u.seen(i) ? 0xffu << (i % 4 * 8) : 0u;
        any |= u.seen(i);
      }
#pragma unroll
      for (int i = 0; i < DT; ++i) vf[i] &= keep;
      v_scale = any ? v_scale : 1.f;   // a block without a token has a scale of any kind
    } else {
      u32x4 keep;
#pragma unroll
      for (int j = 0; j < 4; ++j) keep[j] = (u.seen(2 * j) ? 0xffffu : 0u) | (u.seen(2 * j + 1) ? 0xffff0000u : 0u);
#pragma unroll
      for (int i = 0; i < DT; ++i) vf[i] &= keep;
    }
  };

  // m: what the weights' exponents are taken from, the same in the four lanes of a head.  It follows the running maximum only
  // where a logit is more than kSlack above it (weights are then up to 2^(kLift + kSlack)): most steps scale nothing.
  float m[TILES], from[TILES], l[TILES];   // from: m, or 0 while m is -infinity
  f32x4 o[TILES][DT];
#pragma unroll
  for (int n = 0; n < TILES; ++n) {
    m[n] = -INFINITY;
    from[n] = l[n] = 0.f;
#pragma unroll
    for (int i = 0; i < DT; ++i) o[n][i] = {0.f, 0.f, 0.f, 0.f};
  }
  // k_page, v_page: of the step after the one whose loads are under way: no load waits for the table
  if (t0 < end) {
    const int r0 = real(t0), r1 = real(t0 + kStride);
    load_k(r0, k_page, true);
    load_v(r0, v_page, true);
    k_page = page_at(r1 + k_run);
    v_page = page_at(r1 + kOwn * g);
  }
  for (; t0 < end; t0 += kStride) {
    const bool more = t0 + kStride < end;
    const int now = real(t0), next = real(t0 + kStride), after = real(t0 + 2 * kStride);
    f32x4 sx[NS][TILES];
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int n = 0; n < TILES; ++n) sx[i][n] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      u32x4 f[NS];
#pragma unroll
      for (int i = 0; i < NS; ++i) f[i] = k_fragment(i, k);
#pragma unroll
      for (int n = 0; n < TILES; ++n)
#pragma unroll
        for (int i = 0; i < NS; ++i) sx[i][n] = mfma16<BF16>(f[i], q[n][k], sx[i][n]);
    }
    __builtin_amdgcn_sched_barrier(0);   // into the registers that the products have just read, not into others before them
    load_k(next, k_page, more);
    k_page = page_at(after + k_run);
    typename std::conditional<E4M3, float[kOwn], f32x8>::type x[TILES];
#pragma unroll
    for (int n = 0; n < TILES; ++n)
#pragma unroll
      for (int i = 0; i < kOwn; ++i) x[n][i % NS * 4 + i / NS] = sx[i % NS][n][i / NS] * a.scale_log2;
    if (masked(now)) {   // an unseen token: no weight, and what is no number must not meet it
      const Unseen u = unseen_at(now);
#pragma unroll
      for (int n = 0; n < TILES; ++n)
#pragma unroll
        for (int i = 0; i < kOwn; ++i) x[n][i] = u.seen(i) ? x[n][i] : -INFINITY;
      clear_unseen(u);
    }
    u32x4 pf[NV][TILES];
#pragma unroll
    for (int n = 0; n < TILES; ++n) {
      float top = -INFINITY;
#pragma unroll
      for (int h = 0; h < NV; ++h)
        top = fmaxf(top, fmaxf(fmaxf(fmaxf(x[n][8 * h], x[n][8 * h + 1]), fmaxf(x[n][8 * h + 2], x[n][8 * h + 3])),
                               fmaxf(fmaxf(x[n][8 * h + 4], x[n][8 * h + 5]), fmaxf(x[n][8 * h + 6], x[n][8 * h + 7]))));
      if (__any(top > m[n] + (kLift<BF16> + kSlack))) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float old = m[n];
        m[n] = fmaxf(m[n], top - kLift<BF16>);
        from[n] = m[n] == -INFINITY ? 0.f : m[n];
        const float shrink = exp2_fast(old - from[n]);
        l[n] *= shrink;
#pragma unroll
        for (int i = 0; i < DT; ++i) o[n][i] *= shrink;
      }
#pragma unroll
      for (int h = 0; h < NV; ++h) {
        f32x8 p;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[i] = exp2_fast(x[n][8 * h + i] - from[n]);
          l[n] += p[i];
        }
        pf[h][n] = pack8<BF16>(p);
      }
      if constexpr (!E4M3) {
#pragma unroll
        for (int i = 0; i < DT; ++i) o[n][i] = mfma16<BF16>(vf[i], pf[0][n], o[n][i]);
      }
    }
    if constexpr (E4M3) {   // a fragment is made once for all tiles
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int h = 0; h < NV; ++h) {
          const u32x4 f = v_fragment(i, h);
#pragma unroll
          for (int n = 0; n < TILES; ++n) o[n][i] = mfma16<BF16>(f, pf[h][n], o[n][i]);
        }
    }
    __builtin_amdgcn_sched_barrier(0);
    load_v(next, v_page, more);
    v_page = page_at(after + kOwn * g);
  }

  // A weight that rounds to 0 makes NaN of an infinite value, where the weight itself leaves infinity.  Where a sum is no number, though the
  // sum of the weights is one, its values that are no numbers decide alone: they are added once more, with the weight 1, or 0 where
  // the logit is -infinity.  (Values in 8 bits are finite or NaN, and any weight leaves NaN.)
  if constexpr (!E4M3) {
  bool lost = false;
#pragma unroll
  for (int n = 0; n < TILES; ++n) {
    float largest = o[n][0][0];
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) largest = __builtin_elementwise_maximum(largest, o[n][i][j]);   // NaN where one of them is
    lost |= __builtin_isunordered(largest, largest) && !__builtin_isunordered(l[n], l[n]);
  }
  if (__builtin_expect(__any(lost), 0)) {
#pragma unroll
    for (int n = 0; n < TILES; ++n)
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[n][i][j] = __builtin_isunordered(o[n][i][j], o[n][i][j]) ? kUnknown : o[n][i][j];
    if constexpr (TILES * D >= 3 * 128) {   // q once more, or the loop above spills more of it for its sake (64 sequences, 48 heads to one: 75 us for 70)
      asm volatile("" ::: "memory");
      load_q();
    }
    for (int v = begin + 32 * wave; v < end; v += kStride) {
      const int t = real(v);
      load_k(t, page_at(t + k_run), true);
      u32x4 there[TILES];
#pragma unroll
      for (int n = 0; n < TILES; ++n) {
        f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          s0 = mfma16<BF16>(kf[0][k], q[n][k], s0);
          s1 = mfma16<BF16>(kf[1][k], q[n][k], s1);
        }
        f32x8 p;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[i] = s0[i] * a.scale_log2 == -INFINITY ? 0.f : 1.f;
          p[4 + i] = s1[i] * a.scale_log2 == -INFINITY ? 0.f : 1.f;
        }
        there[n] = pack8<BF16>(p);
      }
      __builtin_amdgcn_sched_barrier(0);   // the values into the keys' registers
      load_v(t, page_at(t + 8 * g), true);
      clear_unseen(unseen_at(t));
#pragma unroll
      for (int i = 0; i < DT; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) vf[i][j] &= odd_halves<BF16>(vf[i][j]);
#pragma unroll
        for (int n = 0; n < TILES; ++n) o[n][i] = mfma16<BF16>(vf[i], there[n], o[n][i]);
      }
    }
#pragma unroll
    for (int n = 0; n < TILES; ++n)
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[n][i][j] = o[n][i][j] == kUnknown ? __builtin_nanf("") : o[n][i][j];
  }
  }

  // The waves' sums, brought to one maximum: four values of a head a thread.
  constexpr int kThreads = 64 * kWaves;
  __shared__ float wave_m[kWaves][kTileHeads], wave_l[kWaves][kTileHeads];
  __shared__ __attribute__((aligned(16))) float wave_o[kWaves][kTileHeads * D];
  __shared__ uint32_t arrived;
  const int parts = (all + A.plan.chunk - 1) / A.plan.chunk;
  const int64_t unit = ((int64_t)s * a.c.kv_heads + kvh) * A.plan.tiles + tile0;
  const size_t part_size = part_floats(A.plan, D);
  // [tile][part]: 16 maxima and sums of weights, cols x D sums over values
  auto parts_of = [&](int n) { return A.part + (size_t)(unit + n) * A.plan.parts * part_size; };
  auto cols_of = [&](int n) { return heads - 16 * n < kTileHeads ? heads - 16 * n : kTileHeads; };   // 0 and less: no such tile
  // out and lse of four values of head c of a tile; an empty row has no weights
  auto finish = [&](int n, int i, f32x4 sum, float top, float weight) {
    const int c = i / (D / 4), d = 4 * (i % (D / 4)), h = h0 + 16 * n + c;
    uint16_t* to = a.out + s * a.os.token + h * a.os.head + d * a.os.dim;
#pragma unroll
    for (int j = 0; j < 4; ++j) to[j * a.os.dim] = from_f32<BF16>(len > 0 ? sum[j] / weight : 0.f);
    if (a.lse && d == 0) a.lse[(int64_t)s * a.heads + h] = len > 0 ? (top + __log2f(weight)) * 0.693147180559945f : -INFINITY;
  };
#pragma unroll
  for (int n = 0; n < TILES; ++n) {
    float sum_l = l[n] + __shfl_xor(l[n], 16);
    sum_l += __shfl_xor(sum_l, 32);
    if (n > 0) __syncthreads();   // the tile before is read
    if (g == 0) {
      wave_m[wave][col] = m[n];
      wave_l[wave][col] = sum_l;
    }
    if (col < cols_of(n)) {
#pragma unroll
      for (int i = 0; i < DT; ++i) *reinterpret_cast<f32x4*>(&wave_o[wave][col * D + 16 * i + 4 * g]) = o[n][i];
    }
    __syncthreads();
    for (int i = tid; i < cols_of(n) * (D / 4); i += kThreads) {
      const int c = i / (D / 4);
      float top = wave_m[0][c];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) top = fmaxf(top, wave_m[w][c]);
      const float base = top == -INFINITY ? 0.f : top;
      f32x4 sum = {0.f, 0.f, 0.f, 0.f};
      float weight = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = rescale(wave_m[w][c], base);
        sum += f * *reinterpret_cast<const f32x4*>(&wave_o[w][4 * i]);
        weight += f * wave_l[w][c];
      }
      if (parts <= 1) {
        finish(n, i, sum, top, weight);
      } else {
        float* mine = parts_of(n) + part * part_size;
        shared_store(mine + 2 * kTileHeads + 4 * i, sum[0], sum[1]);
        shared_store(mine + 2 * kTileHeads + 4 * i + 2, sum[2], sum[3]);
        if (i % (D / 4) == 0) shared_store(mine + 2 * c, top, weight);
      }
    }
  }
  if (parts <= 1) return;

  // Several parts: whoever finishes last joins them, in the parts' order.
  shared_stores_done();
  __syncthreads();
  if (tid == 0) arrived = __hip_atomic_fetch_add(&A.counter[unit], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (arrived != (uint32_t)parts - 1) return;
  if (tid == 0) __hip_atomic_store(&A.counter[unit], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  constexpr int kFew = 8;
  __shared__ float some[kThreads / kTileHeads][kTileHeads];
  for (int n = 0; n < TILES && cols_of(n) > 0; ++n) {
    const int cols = cols_of(n), quads = cols * (D / 4);
    const float* whole = parts_of(n);
    if (parts <= kFew) {   // few: a thread asks for all it needs at once
      for (int i = tid; i < quads; i += kThreads) {
        f32x2 ml[kFew], v[kFew][2];
#pragma unroll
        for (int p = 0; p < kFew; ++p) {
          const float* from = whole + (p < parts ? p : 0) * part_size;
          ml[p] = shared_load(from + 2 * (i / (D / 4)));
          v[p][0] = shared_load(from + 2 * kTileHeads + 4 * i);
          v[p][1] = shared_load(from + 2 * kTileHeads + 4 * i + 2);
        }
        float top = ml[0][0];
#pragma unroll
        for (int p = 1; p < kFew; ++p) top = fmaxf(top, ml[p][0]);
        const float base = top == -INFINITY ? 0.f : top;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        float weight = 0.f;
#pragma unroll
        for (int p = 0; p < kFew; ++p) {
          if (p >= parts) break;
          const float f = rescale(ml[p][0], base);
          sum += f * f32x4{v[p][0][0], v[p][0][1], v[p][1][0], v[p][1][1]};
          weight += f * ml[p][1];
        }
        finish(n, i, sum, top, weight);
      }
      continue;
    }
    // The parts' factors: thread (head tid % 16, every 16th part).
    constexpr int kEach = (kMostParts + kThreads / kTileHeads - 1) / (kThreads / kTileHeads);
    static_assert(kMostParts * kTileHeads <= kWaves * kTileHeads * D, "the factors fit where the waves' sums were");
    float* factor = wave_o[0];                                        // [part][16]
    const int c0 = tid % kTileHeads, r0 = tid / kTileHeads;
    float pm[kEach], pl[kEach];
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int p = r0 + j * (kThreads / kTileHeads);
      const bool there = p < parts && c0 < cols;
      const f32x2 v = there ? shared_load(whole + p * part_size + 2 * c0) : f32x2{-INFINITY, 0.f};
      pm[j] = v[0];
      pl[j] = v[1];
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j) top = fmaxf(top, pm[j]);
    some[r0][c0] = top;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kThreads / kTileHeads; ++r) top = fmaxf(top, some[r][c0]);
    const float base = top == -INFINITY ? 0.f : top;
    float weight = 0.f;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int p = r0 + j * (kThreads / kTileHeads);
      const float f = rescale(pm[j], base);
      weight += f * pl[j];
      if (p < parts) factor[p * kTileHeads + c0] = f;
    }
    __syncthreads();
    some[r0][c0] = weight;
    if (r0 == 0) wave_m[0][c0] = top;
    __syncthreads();
    if (r0 == 0) {
      weight = 0.f;
#pragma unroll
      for (int r = 0; r < kThreads / kTileHeads; ++r) weight += some[r][c0];
      wave_l[0][c0] = weight;
    }
    __syncthreads();
    // The sums: where there are fewer groups of four values than threads, several threads share one, each with every
    // `share`th part.
    const int share = quads < kThreads ? kThreads / quads : 1, mine = share > 1 ? tid / quads : 0;
    f32x4* shared_sum = reinterpret_cast<f32x4*>(wave_o[0]);
    for (int i0 = 0; i0 < quads; i0 += kThreads) {
      const int i = share > 1 ? tid % quads : i0 + tid, c = i / (D / 4);
      const bool busy = i < quads && mine < share;
      f32x4 sum = {0.f, 0.f, 0.f, 0.f};
      if (busy) {
        const float* from_part = whole + 2 * kTileHeads + 4 * i;
        int p = mine;
        for (; p + 7 * share < parts; p += 8 * share) {
          f32x2 v[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) v[j] = shared_load(from_part + (p + j / 2 * share) * part_size + j % 2 * 2);
#pragma unroll
          for (int j = 0; j < 8; ++j) sum += factor[(p + j * share) * kTileHeads + c] * f32x4{v[2 * j][0], v[2 * j][1], v[2 * j + 1][0], v[2 * j + 1][1]};
        }
        for (; p < parts; p += share) {
          const f32x2 u = shared_load(from_part + p * part_size), v = shared_load(from_part + p * part_size + 2);
          sum += factor[p * kTileHeads + c] * f32x4{u[0], u[1], v[0], v[1]};
        }
      }
      if (share > 1) {   // quads < kThreads: one turn of the loop
        __syncthreads();
        if (busy) shared_sum[tid] = sum;
        __syncthreads();
        for (int r = 1; r < share && mine == 0; ++r) sum += shared_sum[r * quads + i];
      }
      if (busy && mine == 0) finish(n, i, sum, wave_m[0][c], wave_l[0][c]);
    }
    __syncthreads();   // the next tile's numbers go where these were
  }
}

// Instances by the plan: Kernels names the kernel of each, up to which page_shift a load of V reads whole lines, and up to which head_dim three
// tiles share a workgroup.
template <typename Kernels, bool BF16, int D, bool WHOLE_LINES>
void launch_pages(const DecodeArgs& a, dim3 grid, hipStream_t s) {
  if constexpr (D <= Kernels::kThreeDim)
    if (a.plan.together == 3) return Kernels::template kernel<BF16, D, WHOLE_LINES, 4, 3><<<grid, 256, 0, s>>>(a);
  if constexpr (D <= kTogetherDim) {
    if (a.plan.together == 2) return Kernels::template kernel<BF16, D, WHOLE_LINES, 4, 2><<<grid, 256, 0, s>>>(a);
    if constexpr (Kernels::kEightWaves)
      if (a.plan.waves == 8) return Kernels::template kernel<BF16, D, WHOLE_LINES, 8, 1><<<grid, 512, 0, s>>>(a);   // the plan has none for larger heads
  }
  Kernels::template kernel<BF16, D, WHOLE_LINES, 4, 1><<<grid, 256, 0, s>>>(a);
}

template <typename Kernels, bool BF16, int D>
void launch_dim(const DecodeArgs& a, hipStream_t s) {
  // Workgroups go to the 8 XCDs in turn: with the heads first every XCD has as much of every sequence, whatever its length (parts
  // first, and 8 of them: the XCD of the last parts had nothing where sequences were short; 61 ragged ones 165 us, 77 so).
  const dim3 grid(a.a.c.kv_heads * ((a.plan.tiles + a.plan.together - 1) / a.plan.together), a.a.c.n_seqs, a.plan.parts);
  if (a.a.c.page_shift <= Kernels::kWholeLines) launch_pages<Kernels, BF16, D, true>(a, grid, s);
  else launch_pages<Kernels, BF16, D, false>(a, grid, s);
}

template <typename Kernels, bool BF16>
void launch_type(const DecodeArgs& a, int head_dim, hipStream_t s) {
  if (head_dim == 64) launch_dim<Kernels, BF16, 64>(a, s);
  else if (head_dim == 96) launch_dim<Kernels, BF16, 96>(a, s);
  else if (head_dim == 128) launch_dim<Kernels, BF16, 128>(a, s);
  else launch_dim<Kernels, BF16, 256>(a, s);
}

template <typename Kernels>
hipError_t launch_any(const DecodeArgs& a, int head_dim, bool bf16, hipStream_t s) {
  if (bf16) launch_type<Kernels, true>(a, head_dim, s);
  else launch_type<Kernels, false>(a, head_dim, s);
  return hipGetLastError();
}

}  // namespace
}  // namespace vq
