// Attention of one new token of every sequence over the paged cache.
#include "vq_attn_device.h"

namespace vq {
namespace {

// One workgroup: `chunk` tokens of a sequence, the query heads of TILES tiles of up to 16.  Its waves take 32 tokens at a time in turn.
//   S^T = K Q^T: two instructions' rows are 16 tokens each, their columns the query heads.  The rows' tokens are chosen so that lane
//   L ends up with the logits of tokens 8 (L / 16) .. + 7 of head L % 16, which is just the operand that
//   O^T += V^T P^T takes: neither product moves anything between lanes, and a page's V is laid out so that V^T is read as it lies.
// m and the sums are those of a softmax in one pass; a lane adds up its own weights until the end.
// WHOLE_LINES: pages of at most 32 tokens, whose V a load reads in whole lines of memory that nobody reads again: they pass the
// caches by (24 sequences of 2,000 to 4,096 tokens x 32 heads, pages of 16: 195 us, 217 without).  In larger pages a step's 64 bytes of a row of
// V^T are half a line, and the wave with the other half wants it kept (130,001 tokens, pages of 64: 95 us, 107 if not); the
// same holds for K, whose rows four instructions read in turn.
// TILES: more than 16 query heads share what is read of their key/value head (64 sequences of 4,096 to 8,192, 48 heads to one of 128: 59 us,
// 118 a tile to a workgroup).
template <bool BF16, int D, bool WHOLE_LINES, int kWaves, int TILES>
__global__ __launch_bounds__(64 * kWaves, D == 256 ? 1 : 2) void decode_kernel(const DecodeArgs A) {
  constexpr int KS = D / 32, DT = D / 16;
  const AttnArgs& a = A.a;
  const int part = blockIdx.z, s = blockIdx.y;
  const int beside = (A.plan.tiles + TILES - 1) / TILES, kvh = blockIdx.x / beside, tile0 = (blockIdx.x - kvh * beside) * TILES;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int len = cached_tokens(a.c, s, a.c.max_len);
  const int begin = part * A.plan.chunk;
  if (begin >= len && part > 0) return;
  const int end = len - begin < A.plan.chunk ? len : begin + A.plan.chunk;
  const int h0 = kvh * a.group + tile0 * kTileHeads;                // first query head
  const int heads = a.group - tile0 * kTileHeads;                   // how many there are from it
  const int shift = a.c.page_shift, mask = (1 << shift) - 1;

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
        for (int k = 0; k < KS; ++k) q[n][k] = *reinterpret_cast<const u32x4*>(row + 32 * k + 8 * g);
      } else {
#pragma unroll
        for (int k = 0; k < KS; ++k) q[n][k] = *reinterpret_cast<const u32x4*>(&q_rows[(16 * n + col) * kRow + 32 * k + 8 * g]);
      }
    }
  };
  load_q();

  const int64_t head_page = (int64_t)D << shift;                    // values of a head in a page
  const int last_page = len > 0 ? (len - 1) >> shift : 0;
  // Where the lane's rows of K (8 tokens of a page: row L % 16 is token 8 (L % 16 / 4) + L % 4, and 4 more in the second
  // instruction) and its 8 tokens of V^T start, for the 32 tokens at t0.
  const int k_run = (col >> 2) * 8, k_in = col & 3;
  u32x4 kf[2][KS], vf[DT];
  const int32_t* table = a.c.table + (int64_t)s * a.c.table_width;
  auto page_at = [&](int t) { return table[t >> shift < last_page ? t >> shift : last_page]; };
  // (Behind the last step there is nothing to load: all lanes then read the same 16 bytes of the buffer's first page, so that the loop
  // is one stretch of code in which every wait knows what is under way.)
  auto load_k = [&](int t0, int page, bool there) {
    const uint16_t* base = a.k_pages + ((int64_t)page_inside(a.c, page) * a.c.kv_heads + kvh) * head_page + (((t0 + k_run) & mask) + k_in) * D + 8 * g;
    base = there ? base : a.k_pages;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      kf[0][k] = *reinterpret_cast<const u32x4*>(base + 32 * k);
      kf[1][k] = *reinterpret_cast<const u32x4*>(base + 4 * D + 32 * k);
    }
  };
  auto load_v = [&](int t0, int page, bool there) {
    const uint16_t* base = a.v_pages + ((int64_t)page_inside(a.c, page) * a.c.kv_heads + kvh) * head_page + ((int64_t)col << shift) + ((t0 + 8 * g) & mask);
    base = there ? base : a.v_pages;
#pragma unroll
    for (int i = 0; i < DT; ++i) {
      const u32x4* from = reinterpret_cast<const u32x4*>(base + ((int64_t)(16 * i) << shift));
      if constexpr (WHOLE_LINES) vf[i] = __builtin_nontemporal_load(from);
      else vf[i] = *from;
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
  constexpr int kStride = 32 * kWaves;
  int k_page = 0, v_page = 0;   // of the step after the one whose loads are under way: no load waits for the table
  int t0 = begin + 32 * wave;
  if (t0 < end) {
    k_page = page_at(t0 + k_run);
    v_page = page_at(t0 + 8 * g);
    load_k(t0, k_page, true);
    load_v(t0, v_page, true);
    k_page = page_at(t0 + kStride + k_run);
    v_page = page_at(t0 + kStride + 8 * g);
  }
  for (; t0 < end; t0 += kStride) {
    const bool more = t0 + kStride < end;
    f32x4 s0[TILES], s1[TILES];
#pragma unroll
    for (int n = 0; n < TILES; ++n) s0[n] = s1[n] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int n = 0; n < TILES; ++n) {
        s0[n] = mfma16<BF16>(kf[0][k], q[n][k], s0[n]);
        s1[n] = mfma16<BF16>(kf[1][k], q[n][k], s1[n]);
      }
    __builtin_amdgcn_sched_barrier(0);   // into the registers that the products have just read, not into others before them
    load_k(t0 + kStride, k_page, more);
    k_page = page_at(t0 + 2 * kStride + k_run);
    f32x8 x[TILES];
#pragma unroll
    for (int n = 0; n < TILES; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[n][i] = s0[n][i] * a.scale_log2;
        x[n][4 + i] = s1[n][i] * a.scale_log2;
      }
    if (t0 + 32 > len) {   // beyond the last token: no weight, and what is no number must not meet it
      const int rest = len - t0 - 8 * g;
#pragma unroll
      for (int n = 0; n < TILES; ++n)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[n][i] = i < rest ? x[n][i] : -INFINITY;
      u32x4 keep;
#pragma unroll
      for (int j = 0; j < 4; ++j) keep[j] = (2 * j < rest ? 0xffffu : 0u) | (2 * j + 1 < rest ? 0xffff0000u : 0u);
#pragma unroll
      for (int i = 0; i < DT; ++i) vf[i] &= keep;
    }
#pragma unroll
    for (int n = 0; n < TILES; ++n) {
      float top = fmaxf(fmaxf(fmaxf(x[n][0], x[n][1]), fmaxf(x[n][2], x[n][3])), fmaxf(fmaxf(x[n][4], x[n][5]), fmaxf(x[n][6], x[n][7])));
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
      f32x8 p;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = exp2_fast(x[n][i] - from[n]);
        l[n] += p[i];
      }
      const u32x4 pf = pack8<BF16>(p);
#pragma unroll
      for (int i = 0; i < DT; ++i) o[n][i] = mfma16<BF16>(vf[i], pf, o[n][i]);
    }
    __builtin_amdgcn_sched_barrier(0);
    load_v(t0 + kStride, v_page, more);
    v_page = page_at(t0 + 2 * kStride + 8 * g);
  }

  // A weight that rounds to 0 makes NaN of an infinite value, where the weight itself leaves infinity.  Where a sum is no number, though the
  // sum of the weights is one, its values that are no numbers decide alone: they are added once more, with the weight 1, or 0 where
  // the logit is -infinity.
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
    for (int t = begin + 32 * wave; t < end; t += kStride) {
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
      const int rest = len - t - 8 * g;
#pragma unroll
      for (int i = 0; i < DT; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          vf[i][j] &= odd_halves<BF16>(vf[i][j]) & ((2 * j < rest ? 0xffffu : 0u) | (2 * j + 1 < rest ? 0xffff0000u : 0u));
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

  // The waves' sums, brought to one maximum: four values of a head a thread.
  constexpr int kThreads = 64 * kWaves;
  __shared__ float wave_m[kWaves][kTileHeads], wave_l[kWaves][kTileHeads];
  __shared__ __attribute__((aligned(16))) float wave_o[kWaves][kTileHeads * D];
  __shared__ uint32_t arrived;
  const int parts = (len + A.plan.chunk - 1) / A.plan.chunk;
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
    const float* all = parts_of(n);
    if (parts <= kFew) {   // few: a thread asks for all it needs at once
      for (int i = tid; i < quads; i += kThreads) {
        f32x2 ml[kFew], v[kFew][2];
#pragma unroll
        for (int p = 0; p < kFew; ++p) {
          const float* from = all + (p < parts ? p : 0) * part_size;
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
      const f32x2 v = there ? shared_load(all + p * part_size + 2 * c0) : f32x2{-INFINITY, 0.f};
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
        const float* from_part = all + 2 * kTileHeads + 4 * i;
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

template <bool BF16, int D, bool WHOLE_LINES>
void launch_pages(const DecodeArgs& a, dim3 grid, hipStream_t s) {
  if constexpr (D <= kTogetherDim) {
    if (a.plan.together == 3) return decode_kernel<BF16, D, WHOLE_LINES, 4, 3><<<grid, 256, 0, s>>>(a);
    if (a.plan.together == 2) return decode_kernel<BF16, D, WHOLE_LINES, 4, 2><<<grid, 256, 0, s>>>(a);
    if (a.plan.waves == 8) return decode_kernel<BF16, D, WHOLE_LINES, 8, 1><<<grid, 512, 0, s>>>(a);   // the plan has none for larger heads
  }
  decode_kernel<BF16, D, WHOLE_LINES, 4, 1><<<grid, 256, 0, s>>>(a);
}

template <bool BF16, int D>
void launch_dim(const DecodeArgs& a, hipStream_t s) {
  // Workgroups go to the 8 XCDs in turn: with the heads first every XCD has as much of every sequence, whatever its length (parts
  // first, and 8 of them: the XCD of the last parts had nothing where sequences were short; 61 ragged ones 165 us, 77 so).
  const dim3 grid(a.a.c.kv_heads * ((a.plan.tiles + a.plan.together - 1) / a.plan.together), a.a.c.n_seqs, a.plan.parts);
  if (a.a.c.page_shift <= 5) launch_pages<BF16, D, true>(a, grid, s);
  else launch_pages<BF16, D, false>(a, grid, s);
}

template <bool BF16>
void launch_type(const DecodeArgs& a, int head_dim, hipStream_t s) {
  if (head_dim == 64) launch_dim<BF16, 64>(a, s);
  else if (head_dim == 96) launch_dim<BF16, 96>(a, s);
  else if (head_dim == 128) launch_dim<BF16, 128>(a, s);
  else launch_dim<BF16, 256>(a, s);
}

}  // namespace

hipError_t launch_attn_decode(const DecodeArgs& a, int head_dim, bool bf16, hipStream_t s) {
  if (bf16) launch_type<true>(a, head_dim, s);
  else launch_type<false>(a, head_dim, s);
  return hipGetLastError();
}

}  // namespace vq
