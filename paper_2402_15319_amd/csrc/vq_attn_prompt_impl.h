// Causal attention of any number of new tokens of every sequence over the paged cache: the kernels' body.
#pragma once
#include <type_traits>

#include "vq_attn_device.h"

namespace vq {
namespace {

constexpr int kWaves = 4 /* of a team */, kRows = kPromptRows, kTokens = kPromptTokens;   // rows of a workgroup's tile; tokens of a step
static_assert(kRows == 32 * kWaves, "32 rows a wave");

// 16-byte pieces of a row of K in LDS change places so that 16 rows' pieces of one number lie in different banks: piece p of row r
// lies where piece p ^ k_turn(r) would.
template <int D> __device__ __forceinline__ int k_turn(int r) {
  return D % 128 == 0 ? r & 15 : D == 64 ? (r >> 1) & 7 : (r >> 2) & 3;
}

// One workgroup: up to 128 rows of one sequence and one key/value head, a row being a (new token, query head of the group) pair, 32
// a wave, and all tokens that they attend (or a part of them), 64 at a time.
//   S^T = K Q^T, O^T += V^T P^T, 32 x 32 x 16: a lane has one row's logits (half of a step's), weights and sums, so that a row's
//   maximum and sum need the other half-wave only, and P goes from the first product's registers into the second's as
//   it is: row m of the first operand is token m with bits 2 and 3 exchanged, which leaves a lane with eight successive tokens.
// K and V^T of a step come into LDS past the registers, each wave 16 tokens of both (one page), while the step before is
// worked on.  With two teams of such waves (see the plan) each takes every second step, and the second's sums go to the first in the end.
// E4M3: pages in 8 bits.  A wave's 16 tokens are one block; their codes come into registers while the step before the one before is worked on, and go
// to LDS as values of the type (exactly), each once for the workgroup, so that the products are those of 16 bits.  Tokens that no row sees and
// values that are no numbers stay behind on the way, so that no step looks for them again.
// WINDOW: a.window and a.sinks.  What no row of the tile sees between the sinks and the window is passed over: in 16 bits in whole sixteens of tokens, each
// one wave's loads of a step, where that takes a step less than in whole steps (grains, below).  Grains are counted as they are gone through; place(number
// of one) is where it begins in the sequence.  Sinks are then an even number of sixteens, so that the 32 tokens of half a step are neighbours.  (In whole steps, 4 sinks take
// a step of their own: 5,000 tokens, 32 heads on 8, window 1,024 106.7 us, 102.7 so; 4,000 tokens, window 64 34.6 and 28.5, 256 44.2 and 38.3.  Nine prompts without sinks,
// window 333, pay 1.4 of 78 us for it.  In 8 bits the steps stay whole: it would be in the way of the registers, 4,096 tokens 161 and 165.)
template <bool BF16, int D, int TEAMS, bool E4M3, bool WINDOW>
__device__ __forceinline__ void prompt_body(const PromptArgs& A) {
  const AttnArgs& a = A.a;
  constexpr int KS = D / 16, DT = D / 32, kLoads = D / 32;     // loads of a wave for its 16 tokens' K, and for their V
  constexpr int kHalf = kTokens * D * 2, kStep = 2 * kHalf;    // bytes of K, or V, of a step
  __shared__ __attribute__((aligned(1024))) char lds[TEAMS * 2 * kStep];
  __shared__ uint32_t odd_values[WINDOW ? kWaves * TEAMS : 1];   // values that are no numbers and were taken out, by the waves that did
  const int tid = threadIdx.x, number = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, half = lane >> 5, col = lane & 31;
  const int wave = number % kWaves, team = number / kWaves;
  // The heads are neighbours, and so are on the 8 XCDs in turn: those of an XCD keep to their keys and values.  Of the tiles the last come
  // first: they attend most.
  const int group = a.group, heads_in = A.plan.heads, wide = a.heads / heads_in;   // query heads of a tile; tiles beside one another
  const int slot = (int)A.plan.slots - 1 - blockIdx.x / wide, beside = blockIdx.x % wide, head0 = beside * heads_in, kvh = head0 / group;
  const int tokens = A.plan.tokens;
  const Tile tile = tile_of(a.c, slot, tokens, 1, a.c.max_len);
  const int s = tile.sequence, first = tile.first, n = tile.last - first, len = tile.cached, behind = len - n;   // new token i: position behind + i
  const int token0 = tile.number * tokens;
  if (token0 >= n) return;
  // Row r is token r % tokens of head r / tokens.  The wave's are tokens low .. high (none if low >= n), the lane's one is valid or
  // works on some other.
  const int row = 32 * wave, end = heads_in * tokens - 1, row1 = row + 31 < end ? row + 31 : end;
  const bool one_head = row <= end && row / tokens == row1 / tokens;
  const int low = row > end ? n : token0 + (one_head ? row % tokens : 0), last = token0 + (one_head ? row1 % tokens : tokens - 1);
  const int high = last < n ? last : n - 1;
  const int mine = row + col <= end ? row + col : end, token_in = token0 + mine % tokens, token = token_in < n ? token_in : n - 1;
  const int head = head0 + mine / tokens;
  const bool valid = row + col <= end && token_in < n;
  const int most = behind + (token0 + tokens < n ? token0 + tokens : n) - 1;   // highest position of the tile
  const int pos = behind + token, wave_first = behind + low, wave_last = low < n ? behind + high : -1;
  // The first token in a window of the tile; grains sinks_end .. sinks_end + skip - 1 are passed over.
  constexpr int kGrain = E4M3 ? kTokens : 16, kOfStep = kTokens / kGrain;
  int first_seen = 0, sinks_end = 0, skip = 0, all = most < 0 ? 0 : (uint32_t)most / kTokens + 1;   // steps of the tile
  if constexpr (WINDOW) {
    first_seen = behind + token0 - a.window + 1 > 0 ? behind + token0 - a.window + 1 : 0;
    auto pass_over = [&](uint32_t unit, uint32_t sinks_unit) {   // where that takes fewer steps
      const int sinks = ((uint32_t)a.sinks + sinks_unit - 1) / sinks_unit * (sinks_unit / kGrain), over = (uint32_t)first_seen / unit * (unit / kGrain) - sinks;
      if (over <= 0 || most < 0) return;
      const int rest = ((uint32_t)most / kGrain - over) / kOfStep + 1;
      if (rest >= all) return;
      sinks_end = sinks;
      skip = over;
      all = rest;
    };
    pass_over(kTokens, kTokens);
    if constexpr (!E4M3) pass_over(16, 32);
  }
  // Where a grain begins, the wave's own tokens of a step, and half of a step's.
  auto place = [&](int grain) { return kGrain * (WINDOW && grain >= sinks_end ? grain + skip : grain); };
  auto own_place = [&](int step) { return E4M3 ? place(step) + 16 * wave : place(kOfStep * step + wave); };
  auto half_place = [&](int step, int t) { return E4M3 ? place(step) + 32 * t : place(kOfStep * step + 2 * t); };
  const int begin = blockIdx.y * A.plan.steps, steps = all - begin < A.plan.steps ? all : begin + A.plan.steps;
  if (begin >= all && begin > 0) return;

  // Loads: the wave's tokens are 16 wave .. + 15 of the step.  K: rows of D values, their pieces turned; V^T: for each dimension two
  // pieces of eight tokens, exchanged where bit 3 of the dimension is set.
  const int shift = a.c.page_shift, mask = (1 << shift) - 1, last_page = len > 0 ? (len - 1) >> shift : 0;
  uint32_t k_off[kLoads];
  if constexpr (!E4M3) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int at = 64 * j + lane, r = at / (D / 8), p = at % (D / 8);
      k_off[j] = (r * D + (p ^ k_turn<D>(r)) * 8) * 2;
    }
  }
  const uint32_t v_off = (((lane >> 1) << shift) + 8 * ((lane & 1) ^ ((lane >> 4) & 1))) * 2;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds) + team * (2 * kStep);
  const int32_t* table = a.c.table + (int64_t)s * a.c.table_width;
  // Lane i: the wave's page in the i-th (mod 64) of the steps that are being loaded; asked for before q, which the loads need not wait for.
  auto pages_from = [&](int step) {
    const int j = own_place(step + TEAMS * lane) >> shift;
    return table[j < last_page ? j : last_page];
  };
  int pages = pages_from(begin + team);
  u32x4 q[KS];
  {
    const uint16_t* from = a.q + (int64_t)(first + token) * a.qs.token + head * a.qs.head;
    if (a.qs.dim == 1 && ((a.qs.token | a.qs.head) & 7) == 0) {
#pragma unroll
      for (int k = 0; k < KS; ++k) q[k] = *reinterpret_cast<const u32x4*>(from + 16 * k + 8 * half);
    } else {
#pragma unroll
      for (int k = 0; k < KS; ++k) q[k] = gather8(from + (16 * k + 8 * half) * a.qs.dim, a.qs.dim);
    }
  }

  auto page_of = [&](int step) {   // of the wave's tokens; steps one after another
    const int at = ((step - begin) / TEAMS) & 63;
    if (at == 0 && step >= begin + TEAMS) pages = pages_from(step);
    return page_inside(a.c, __builtin_amdgcn_readlane(pages, at));
  };
  auto load = [&](int step) {
    const int page = page_of(step);
    const int in = own_place(step) & mask;
    const int64_t page_head = ((int64_t)page * a.c.kv_heads + kvh) * ((int64_t)D << shift);
    const uint16_t* k = a.k_pages + page_head + in * D;
    const uint16_t* v = a.v_pages + page_head + in;
    const uint32_t to = lds0 + ((step / TEAMS) & 1) * kStep + wave * (kHalf / kWaves);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) load_to_lds(k, k_off[j], to + 1024 * j);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) load_to_lds(v + ((int64_t)(32 * j) << shift), v_off, to + kHalf + 1024 * j);
  };
  // The same in 8 bits, in two halves.  16 codes of a token's dimensions, or of a dimension's tokens, to a load; of heads of 96 the last 32 dimensions
  // are 8 to a load.
  const int this_lane = lane;
  // Where a lane's first pieces go: 16 codes of K are pieces 2 lane and 2 lane + 1 of the wave's tokens, one token after another (further ones 16 / (D / 64) tokens
  // later, whose turn differs from the first token's in bits that those of the first tokens leave out), 16 of V the two of dimension lane.
  const int swapped = lane >> 2 & 1, k_at0 = 2 * lane + swapped;
  const int k_place = (k_at0 / (D / 8) * (D / 8) + ((k_at0 % (D / 8)) ^ k_turn<D>(k_at0 / (D / 8)))) * 16, v_place = (2 * lane + (swapped ^ (lane >> 3 & 1))) * 16;
  constexpr int kCodes = D / 64, kFrags = (D + 63) / 64;
  u32x4 k_codes[E4M3 ? kFrags : 1], v_codes[E4M3 ? kFrags : 1];
  float k_scale = 1.f, v_scale = 1.f;
  auto apart = [](int x) {   // the same number, but nothing is made of it beforehand or for another place: that would take registers of the products
    asm volatile("" : "+v"(x));
    return x;
  };
  auto fetch = [&](int step) {
    const int lane = apart(this_lane);
    const int page = page_of(step);
    const int in = own_place(step) & mask;
    const int64_t head = (int64_t)page * a.c.kv_heads + kvh;
    const uint8_t* k = reinterpret_cast<const uint8_t*>(a.k_pages) + (head * D << shift) + in * D;
    const uint8_t* v = reinterpret_cast<const uint8_t*>(a.v_pages) + (head * D << shift) + in;
    const int64_t block = (head << (shift - 4)) + (in >> 4);
    k_scale = a.k_scales[block];
    v_scale = a.v_scales[block];
#pragma unroll
    for (int j = 0; j < kCodes; ++j) {
      k_codes[j] = *reinterpret_cast<const u32x4*>(k + 1024 * j + 16 * lane);
      v_codes[j] = *reinterpret_cast<const u32x4*>(v + ((64 * j + lane) << shift));
    }
    if constexpr (E4M3 && kFrags > kCodes) {
      const u32x2 x = *reinterpret_cast<const u32x2*>(k + 1024 * kCodes + 8 * lane);
      const u32x2 y = *reinterpret_cast<const u32x2*>(v + ((64 * kCodes + (lane >> 1)) << shift) + 8 * (lane & 1));
      k_codes[kCodes] = {x[0], x[1], 0, 0};
      v_codes[kCodes] = {y[0], y[1], 0, 0};
    }
  };
  auto store = [&](int step) {
    const int lane = apart(this_lane);
    const int step_at = place(kOfStep * step);
    if (step_at + kTokens > len || (step_at < first_seen && step_at + kTokens > a.sinks)) {
      const int at = apart(step_at + 16 * wave);
      auto seen = [&](int t) { return t < len && (t < a.sinks || t >= first_seen); };
      u32x4 keep = {0, 0, 0, 0};
      bool any = false;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        keep[i / 4] |= seen(at + i) ? 0xffu << (i % 4 * 8) : 0u;
        any |= seen(at + i);
      }
#pragma unroll
      for (int j = 0; j < kCodes; ++j) v_codes[j] &= keep;
      if constexpr (E4M3 && kFrags > kCodes) {
        v_codes[kCodes][0] &= lane & 1 ? keep[2] : keep[0];
        v_codes[kCodes][1] &= lane & 1 ? keep[3] : keep[1];
      }
      v_scale = any ? v_scale : 1.f;   // a block without a token has a scale of any kind
    }
    auto odd = [](uint32_t c) { return ((c & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; };
    uint32_t some = 0;
#pragma unroll
    for (int j = 0; j < (E4M3 ? kFrags : 1); ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) some |= odd(v_codes[j][e]);
    if (__builtin_expect(__any(some), 0)) {
#pragma unroll
      for (int j = 0; j < (E4M3 ? kFrags : 1); ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) v_codes[j][e] &= ~((odd(v_codes[j][e]) >> 7) * 0xffu);
      odd_values[number] = 1;
    }
    char* to = lds + (2 * team + ((step / TEAMS) & 1)) * kStep + wave * (kHalf / kWaves);
#pragma unroll
    for (int j = 0; j < kCodes; ++j) {
      // Of a lane's two pieces every second four lanes write the other one first: 8 lanes then write 128 bytes of different banks.
      const u32x4 k = swapped ? u32x4{k_codes[j][2], k_codes[j][3], k_codes[j][0], k_codes[j][1]} : k_codes[j];
      const u32x4 v = swapped ? u32x4{v_codes[j][2], v_codes[j][3], v_codes[j][0], v_codes[j][1]} : v_codes[j];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        *reinterpret_cast<u32x4*>(to + ((k_place ^ 16 * h ^ 16 * (j * 1024 / D & 15)) + 2048 * j)) = values8<BF16>(k[2 * h], k[2 * h + 1], k_scale);
        *reinterpret_cast<u32x4*>(to + kHalf + ((v_place ^ 16 * h) + 2048 * j)) = values8<BF16>(v[2 * h], v[2 * h + 1], v_scale);
      }
    }
    if constexpr (E4M3 && kFrags > kCodes) {
      const int at = 128 * kCodes + lane, r = at / (D / 8), d = 64 * kCodes + (lane >> 1);
      *reinterpret_cast<u32x4*>(to + (r * (D / 8) + ((at % (D / 8)) ^ k_turn<D>(r))) * 16) = values8<BF16>(k_codes[kCodes][0], k_codes[kCodes][1], k_scale);
      *reinterpret_cast<u32x4*>(to + kHalf + (2 * d + ((lane & 1) ^ ((d >> 3) & 1))) * 16) = values8<BF16>(v_codes[kCodes][0], v_codes[kCodes][1], v_scale);
    }
  };

  int step = begin + team;
  if constexpr (WINDOW) odd_values[number] = 0;
  if constexpr (E4M3) {
    if (step < steps) {
      fetch(step);
      store(step);
      if (step + TEAMS < steps) fetch(step + TEAMS);
    }
  } else {
    if (step < steps) load(step);
  }
#pragma unroll
  for (int k = 0; k < KS; ++k) asm volatile("" : "+v"(q[k]));   // here, or the compiler waits for them in the loop, and with them for its loads

  float m = -INFINITY, from = 0.f, l = 0.f;   // as in the kernel of one new token
  f32x16 o[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
  const int k_row = (col & 0x13) | (col & 4) << 1 | (col & 8) >> 1;
  uint32_t left_out = 0;   // values that are no numbers, in steps with a mask
  auto up_to_last = [&](int at) {   // what is left of the lane's tokens at + 8 half .. + 7: those up to the sequence's last one that some row may see
    const int rest = len - at - 8 * half, lo = WINDOW ? a.sinks - at - 8 * half : 0, hi = WINDOW ? first_seen - at - 8 * half : 0;
    auto there = [&](int i) { return i < rest && (!WINDOW || i < lo || i >= hi); };
    u32x4 keep;
#pragma unroll
    for (int j = 0; j < 4; ++j) keep[j] = (there(2 * j) ? 0xffffu : 0u) | (there(2 * j + 1) ? 0xffff0000u : 0u);
    return keep;
  };

  // 16 bits, WINDOW: takes out of the step's values in LDS what is no number.  Another wave that is at the same does the same; one whose rows all see the
  // step may read it before or after, and finds the word of it behind its last step: a wave's own LDS operations are carried out in order, and the two
  // asm statements with "words" keep the compiler to it, here (the word before any value) and there (the words behind all values).
  auto values_in_lds = [&](int step) {
    return reinterpret_cast<u32x4*>(lds + (2 * team + ((step / TEAMS) & 1)) * kStep + kHalf) + apart(this_lane);
  };
  auto clear_odd = [&](int step) {
    u32x4* vt = values_in_lds(step);
    odd_values[number] = 1;
    asm volatile("; words: written" ::: "memory");
#pragma unroll 1
    for (int n = 0; n < kHalf / 16; n += 64) {
      u32x4 v = vt[n];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] &= ~odd_halves<BF16>(v[i]);
      vt[n] = v;
    }
  };
  // The same of the wave's own tokens that no row sees, whatever they are, before anybody reads them.
  auto clear_unseen = [&](int step) {
    const int lane = apart(this_lane), at0 = own_place(step);
    u32x4* vt = values_in_lds(step) + wave * (kHalf / kWaves / 16);
#pragma unroll
    for (int n = 0; n < kHalf / kWaves / 16; n += 64) {
      const int d = (n + lane) / 2, at = at0 + 8 * ((lane & 1) ^ (d >> 3 & 1));
      u32x4 keep = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 8; ++i) keep[i / 2] |= at + i < len && (at + i < a.sinks || at + i >= first_seen) ? 0xffffu << (i % 2 * 16) : 0u;
      vt[n] &= keep;
    }
  };
  auto next_step = [&](int step) {   // E4M3: while the last products of a step are still under way
    if (step + TEAMS < steps) store(step + TEAMS);
    if (step + 2 * TEAMS < steps) fetch(step + 2 * TEAMS);
  };
  // masked: some row of the wave leaves out some token of the step.  Where it is known only here (WINDOW), both kinds of steps are one stretch of code.
  auto work = [&](int step, auto masked) {
    constexpr bool known = !std::is_same<decltype(masked), bool>::value;
    const char* kt = lds + (2 * team + ((step / TEAMS) & 1)) * kStep;
    const char* vt = kt + kHalf;
    f32x16 x[2];
    // The products of the logits go before another wave's weights (nine packed prompts 94 to 95 us, 98 without).
    __builtin_amdgcn_s_setprio(1);
    // An operand's fragments, up to 16 asked for before the first is used.  (KS = 2 DT: both products have 4 DT.)
    constexpr int kBatch = 4 * DT < 16 ? 4 * DT : 16;
    u32x4 f[kBatch];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < 16; ++j) x[t][j] = 0.f;
#pragma unroll
    for (int k0 = 0; k0 < KS; k0 += kBatch / 2) {
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int r = 32 * (k & 1) + k_row;
        f[k] = *reinterpret_cast<const u32x4*>(kt + (r * (D / 8) + ((2 * (k0 + k / 2) + half) ^ k_turn<D>(r))) * 16);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < kBatch; ++k) x[k & 1] = mfma32<BF16>(f[k], q[k0 + k / 2], x[k & 1]);
      __builtin_amdgcn_sched_barrier(0);
    }
    const char* v_at = vt + col * 32 + (half ^ ((col >> 3) & 1)) * 16;
    auto v_batch = [&](int at) {   // fragments at .. of V^T: 32 dimensions of the first 16 tokens, the next 32, ..
#pragma unroll
      for (int j = 0; j < kBatch; ++j) f[j] = *reinterpret_cast<const u32x4*>(v_at + ((at + j) / DT * D + (at + j) % DT * 32) * 32);
      __builtin_amdgcn_sched_barrier(0);
    };
    if (!known || !masked) v_batch(0);   // under way while the weights are made
    __builtin_amdgcn_s_setprio(0);
    if (masked) {
      if constexpr (WINDOW) {
        // Bit i of a word: the lane sees its token i; a logit's bit, spread over a word, keeps it or not (with compares and selects, some 60
        // instructions more, nine prompts of up to 2,500, heads of 96, window 333 took 80.7 us, 77.4 so; 61 tokens 7.1 and 6.9).
        const int first = half_place(step, 0) + (apart(this_lane) >> 5 << 3), rel = apart(pos) - first;
        const int sinks = a.sinks - first, in = sinks < rel + 1 ? sinks : rel + 1;
        auto below = [](int n) { return n > 31 ? ~0u : (1u << (n > 0 ? n : 0)) - 1; };
        // (The wait is what has to lie between a matrix instruction and a read of its result: the compiler does not look into the two instructions below.)
        asm volatile("s_nop 15\n\ts_nop 7" : "+v"(x[0]), "+v"(x[1]));
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int on = t * (half_place(step, 1) - half_place(step, 0));
          const uint32_t seen = (below(rel + 1 - on) & ~below(rel + 1 - a.window - on)) | below(in - on);
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            uint32_t keep;
            asm("v_bfe_i32 %1, %2, %3, 1\n\tv_bfi_b32 %0, %1, %0, %4" : "+v"(x[t][j]), "=&v"(keep) : "v"(seen), "n"(16 * (j >> 3) + (j & 7)), "s"(0xff800000u));
          }
        }
      } else {
        const int rel = pos - step * kTokens - 8 * half;   // tokens of the lane up to here are attended
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int j = 0; j < 16; ++j) x[t][j] = 32 * t + 16 * (j >> 3) + (j & 7) <= rel ? x[t][j] : -INFINITY;
      }
    }
    float top = x[0][0];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < 16; ++j) top = fmaxf(top, x[t][j]);
    if (__any(top * a.scale_log2 > m + (kLift<BF16> + kSlack))) {
      top = fmaxf(top, __shfl_xor(top, 32)) * a.scale_log2;
      const float old = m;
      m = fmaxf(m, top - kLift<BF16>);
      from = m == -INFINITY ? 0.f : m;
      const float shrink = exp2_fast(old - from);
      l *= shrink;
#pragma unroll
      for (int i = 0; i < DT; ++i) o[i] *= shrink;
    }
    u32x4 p[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      f32x8 w;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        w[j] = exp2_fast(fmaf(x[c >> 1][8 * (c & 1) + j], a.scale_log2, -from));
        l += w[j];
      }
      p[c] = pack8<BF16>(w);
    }
    if (known && masked) {
      // A row's weight of 0 must not meet a value that is no number: tokens behind the last one are cleared, and what else there is
      // of them is left out of the product; it is added after the last step.
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          u32x4 f = *reinterpret_cast<const u32x4*>(v_at + (c * D + 32 * i) * 32) & up_to_last(step * kTokens + 16 * c);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t odd = odd_halves<BF16>(f[j]);
            left_out |= odd;
            f[j] &= ~odd;
          }
          o[i] = mfma32<BF16>(f, p[c], o[i]);
        }
    } else {
#pragma unroll
      for (int at = 0; at < 4 * DT; at += kBatch) {
        if (at > 0) v_batch(at);
        if (!E4M3 && !known && masked) {
          // To the same end a product with zeros (of any order: each value meets one) says whether there is a value at all that is no number, in place of
          // hundreds of instructions that look at each; then it is cleared in LDS.
          f32x4 none = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < kBatch; ++j) none = mfma16<BF16>(f[j], u32x4{0, 0, 0, 0}, none);
          const float any = (none[0] + none[1]) + (none[2] + none[3]);
          if (__builtin_expect(__any(__builtin_isunordered(any, any)), 0)) {
            clear_odd(step);
            v_batch(at);
          }
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) o[(at + j) % DT] = mfma32<BF16>(f[j], p[(at + j) / DT], o[(at + j) % DT]);
      }
    }
  };

  auto turn = [&](int step) {
    if constexpr (E4M3) {
      lds_written();
    } else {
      if constexpr (WINDOW) {
        const int at = own_place(step);
        if (step < steps && (at + 16 > len || (at < first_seen && at + 16 > a.sinks))) {
          lds_arrived();
          clear_unseen(step);
        }
      }
      lds_turn();
      if (step + TEAMS < steps) load(step + TEAMS);
    }
  };
  if constexpr (WINDOW) {
    // Steps whose tokens all of the wave's rows attend, and others with a token that one of them does.
    for (; step - team < steps; step += TEAMS) {
      turn(step);
      const int at = half_place(step, 0), end = half_place(step, 1) + 31;   // (the step with the last sinks and the window's first tokens is one with a mask)
      if ((TEAMS == 1 || step < steps) && at <= wave_last && (end > wave_first - a.window || at < a.sinks))
        work(step, !(end - at < kTokens && end <= wave_first && (at > wave_last - a.window || end < a.sinks)));
      if constexpr (E4M3) next_step(step);
    }
  } else {
  // First the steps whose tokens all of the wave's rows attend.
  const int whole = low < n && wave_first >= 0 ? (wave_first + 1) / kTokens : 0;
  for (; step < whole && step < steps; step += TEAMS) {
    turn(step);
    work(step, std::false_type());
  }
  for (; step - team < steps; step += TEAMS) {
    turn(step);
    if ((TEAMS == 1 || step < steps) && step * kTokens <= wave_last) work(step, std::true_type());
  }
  }

  // A weight that rounds to 0 makes NaN of an infinite value, where the weight itself leaves infinity.  Where a sum is no number, though the
  // sum of the weights is one, its values that are no numbers decide alone: all of them are added in one more turn through the
  // wave's steps, with the weight 1, or 0 where the logit is -infinity.
  float largest = o[0][0];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) largest = __builtin_elementwise_maximum(largest, o[i][j]);   // NaN where one of them is
  if constexpr (WINDOW) {
    asm volatile("; words: read" ::: "memory");
    if (begin < steps) {   // (no step, no barrier behind the words' first values)
#pragma unroll
      for (int i = 0; i < kWaves; ++i) left_out |= odd_values[kWaves * team + i];
    }
  }
  if (__builtin_expect(__any(left_out != 0 || (__builtin_isunordered(largest, largest) && !__builtin_isunordered(l, l))), 0)) {
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] = __builtin_isunordered(o[i][j], o[i][j]) ? kUnknown : o[i][j];
    // 32 tokens at a time: what each row attends of them, with a weight (there) or without (none), times 1 for infinity, 64 for -infinity and
    // 4,096 for NaN: no more than 16 of each in a sum.  (4,096 tokens x 32 heads of 128 whose values are all NaN: 1.7 ms, 0.17 with none.)
    constexpr uint32_t kExp = BF16 ? 0x7f80 : 0x7c00, kOne = BF16 ? 0x3f80 : 0x3c00, k64 = BF16 ? 0x4280 : 0x5400, k4096 = BF16 ? 0x4580 : 0x6c00;
    for (int gone = (begin + team) * kTokens; gone < steps * kTokens; gone += gone % kTokens ? 32 + (TEAMS - 1) * kTokens : 32) {
      const int at = place(gone / kGrain) + gone % kGrain;
      if (at > wave_last) break;
      int64_t head[2], block[2];   // of the 16 tokens' page; their scales
      u32x4 keep[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int t = at + 16 * h, page = table[t >> shift < last_page ? t >> shift : last_page];
        head[h] = ((int64_t)page_inside(a.c, page) * a.c.kv_heads + kvh) * ((int64_t)D << shift);
        block[h] = (((int64_t)page_inside(a.c, page) * a.c.kv_heads + kvh) << (shift - 4)) + ((t & mask) >> 4);
        keep[h] = up_to_last(t);
      }
      auto values = [&](int h, int i) {
        const int64_t from = head[h] + ((int64_t)(32 * i + col) << shift) + ((at + 16 * h) & mask) + 8 * half;
        if constexpr (E4M3) {
          const u32x2 u = *reinterpret_cast<const u32x2*>(reinterpret_cast<const uint8_t*>(a.v_pages) + from);
          return values8<BF16>(u[0], u[1], a.v_scales[block[h]]) & keep[h];
        } else {
          return *reinterpret_cast<const u32x4*>(a.v_pages + from) & keep[h];
        }
      };
      uint32_t odd = 0;
#pragma unroll 1
      for (int i = 0; i < 2 * DT; ++i) {
        const u32x4 f = values(i & 1, i >> 1);
        odd |= odd_halves<BF16>(f[0]) | odd_halves<BF16>(f[1]) | odd_halves<BF16>(f[2]) | odd_halves<BF16>(f[3]);
      }
      if (!__any(odd)) continue;
      f32x16 x;
#pragma unroll
      for (int j = 0; j < 16; ++j) x[j] = 0.f;
      const int64_t k_from = (k_row < 16 ? head[0] : head[1]) + (((at + k_row) & mask) * D) + 8 * half;
#pragma unroll
      for (int c = 0; c < KS; ++c) {
        u32x4 f;
        if constexpr (E4M3) {
          const u32x2 u = *reinterpret_cast<const u32x2*>(reinterpret_cast<const uint8_t*>(a.k_pages) + k_from + 16 * c);
          f = values8<BF16>(u[0], u[1], a.k_scales[k_row < 16 ? block[0] : block[1]]);
        } else {
          f = *reinterpret_cast<const u32x4*>(a.k_pages + k_from + 16 * c);
        }
        x = mfma32<BF16>(f, q[c], x);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 there = {0, 0, 0, 0}, none = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int t = at + 16 * h + 8 * half + j;
          const bool mine = t <= pos && (!WINDOW || t > pos - a.window || t < a.sinks), zero = x[8 * h + j] * a.scale_log2 == -INFINITY;
          there[j / 2] |= mine && !zero ? kOne << (j % 2 * 16) : 0u;
          none[j / 2] |= mine && zero ? kOne << (j % 2 * 16) : 0u;
        }
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          const u32x4 f = values(h, i);
          u32x4 code = {0, 0, 0, 0}, all_nan = {0, 0, 0, 0};
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint32_t u = f[j / 2] >> (j % 2 * 16) & 0xffff, size = u & 0x7fff;
            code[j / 2] |= (size < kExp ? 0u : size > kExp ? k4096 : u > kExp ? k64 : kOne) << (j % 2 * 16);
            all_nan[j / 2] |= (size < kExp ? 0u : k4096) << (j % 2 * 16);
          }
          f32x16 y;
#pragma unroll
          for (int j = 0; j < 16; ++j) y[j] = 0.f;
          y = mfma32<BF16>(code, there, y);
          y = mfma32<BF16>(all_nan, none, y);
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const uint32_t count = (uint32_t)y[j];
            o[i][j] += (count & 63 ? INFINITY : 0.f) - (count >> 6 & 63 ? INFINITY : 0.f);
            o[i][j] = count >> 12 ? __builtin_nanf("") : o[i][j];
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] = o[i][j] == kUnknown ? __builtin_nanf("") : o[i][j];
  }

  l += __shfl_xor(l, 32);
  if constexpr (TEAMS == 2) {
    // What the second team has goes through LDS, [maximum and sum of the weights, then four sums over values at a time][lane].
    constexpr int kPieces = 1 + 4 * DT;
    static_assert(kWaves * kPieces * 1024 <= (int)sizeof(lds));
    f32x4* at = reinterpret_cast<f32x4*>(lds) + wave * (kPieces * 64) + lane;
    __syncthreads();
    if (team == 1) {
      at[0] = f32x4{m, l, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4 * DT; ++i)
        at[(1 + i) * 64] = f32x4{o[i >> 2][4 * (i & 3)], o[i >> 2][4 * (i & 3) + 1], o[i >> 2][4 * (i & 3) + 2], o[i >> 2][4 * (i & 3) + 3]};
    }
    __syncthreads();
    if (team == 1) return;
    const f32x4 ml = at[0];
    const float old = m;
    m = fmaxf(m, ml[0]);
    const float base = m == -INFINITY ? 0.f : m, f0 = rescale(old, base), f1 = rescale(ml[0], base);
    // Here and below one of two products is fused with the sum, as written: a build that chooses changes the last bits.  (Which one it is calls have had since
    // there are teams and parts.)
    l = fmaf(f0, l, f1 * ml[1]);
#pragma unroll
    for (int i = 0; i < 4 * DT; ++i) {
      const f32x4 v = at[(1 + i) * 64];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float first = o[i >> 2][4 * (i & 3) + j];
        o[i >> 2][4 * (i & 3) + j] = !WINDOW || i < 6 ? fmaf(f1, v[j], f0 * first) : fmaf(f0, first, f1 * v[j]);
      }
    }
  }
  const int parts = (all + A.plan.steps - 1) / A.plan.steps;
  if (parts > 1) {
    // Whoever finishes last joins the parts, in their order; a part's loads are under way together (a wait for each took 25 us of 63, 256
    // dimensions).  A lane's numbers lie where the same lane finds them: [part][maximum and sum
    // of the weights, then two sums over values at a time][lane].
    __shared__ uint32_t arrived;
    constexpr int kPairs = 1 + 8 * DT;
    const int64_t unit = (int64_t)slot * wide + beside;
    float* mine = A.part + ((unit * A.plan.parts * kWaves + wave) * kPairs * 64 + lane) * 2;   // of part 0
    constexpr int64_t kPart = (int64_t)kWaves * kPairs * 128;
    if (low < n) {
      float* to = mine + blockIdx.y * kPart;
      shared_store(to, m, l);
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) shared_store(to + (1 + 8 * i + j) * 128, o[i][2 * j], o[i][2 * j + 1]);
    }
    shared_stores_done();
    __syncthreads();
    if (tid == 0) arrived = __hip_atomic_fetch_add(&A.counter[unit], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (arrived != (uint32_t)parts - 1) return;
    if (tid == 0) __hip_atomic_store(&A.counter[unit], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (low >= n) return;
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    for (int p = 0; p < parts; ++p) {
      const float* of = mine + p * kPart;
      constexpr int kAhead = D == 256 ? 16 : 8 * DT;   // loads under way together
      const f32x2 ml = shared_load(of);
      f32x2 v[kAhead];
      float old = 0.f, now = 0.f;
#pragma unroll
      for (int at = 0; at < 8 * DT; at += kAhead) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) v[j] = shared_load(of + (1 + at + j) * 128);
        __builtin_amdgcn_sched_barrier(0);
        if (at == 0) {
          const float top = fmaxf(m, ml[0]), base = top == -INFINITY ? 0.f : top;
          old = rescale(m, base);
          now = rescale(ml[0], base);
          m = top;
          l = fmaf(old, l, now * ml[1]);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int d = 2 * (at + j) + e;
            o[d >> 4][d & 15] = !WINDOW && (D == 64 || D == 256) ? fmaf(now, v[j][e], old * o[d >> 4][d & 15]) : fmaf(old, o[d >> 4][d & 15], now * v[j][e]);
          }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  const bool any = pos >= 0;
  const float scale = any ? 1.f / l : 0.f;
  uint16_t* to = a.out + (int64_t)(first + token) * a.os.token + head * a.os.head;
  if (a.os.dim == 1 && ((a.os.token | a.os.head) & 7) == 0) {
    // The half-waves exchange fours of dimensions, which leaves a lane with eight in a row.
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        f32x8 v;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = any ? o[i][8 * b + j] * scale : 0.f;
        u32x4 w = pack8<BF16>(v);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const auto r = __builtin_amdgcn_permlane32_swap(w[j], w[2 + j], false, false);
          w[j] = r[0];
          w[2 + j] = r[1];
        }
        if (valid) *reinterpret_cast<u32x4*>(to + 32 * i + 16 * b + 8 * half) = w;
      }
  } else if (valid) {
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int64_t d = 32 * i + 8 * (j >> 2) + 4 * half + (j & 3);
        to[d * a.os.dim] = from_f32<BF16>(any ? o[i][j] * scale : 0.f);
      }
  }
  if (a.lse && half == 0 && valid) a.lse[(int64_t)(first + token) * a.heads + head] = any ? (m + __log2f(l)) * 0.693147180559945f : -INFINITY;
}

// Instances by the plan: Kernels names the kernel of each.
template <typename Kernels, bool BF16, int D>
hipError_t launch_prompt(const PromptArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.a.heads / a.plan.heads * a.plan.slots), a.plan.parts);
  if constexpr (D <= 128)
    if (a.plan.teams == 2) {
      Kernels::template kernel<BF16, D, 2><<<grid, 2 * 64 * kWaves, 0, s>>>(a);
      return hipGetLastError();
    }
  Kernels::template kernel<BF16, D, 1><<<grid, 64 * kWaves, 0, s>>>(a);
  return hipGetLastError();
}

// Heads of 64, 96 and 128.
template <typename Kernels, bool BF16>
hipError_t launch_prompt_small(const PromptArgs& a, int head_dim, hipStream_t s) {
  if (head_dim == 64) return launch_prompt<Kernels, BF16, 64>(a, s);
  if (head_dim == 96) return launch_prompt<Kernels, BF16, 96>(a, s);
  return launch_prompt<Kernels, BF16, 128>(a, s);
}

}  // namespace
}  // namespace vq
