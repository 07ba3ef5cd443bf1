// Block selection: for every query position and kv head the `K` blocks of the
// key axis that its attention reads. The first `sinks` blocks and the last `local`
// ones up to the query's own are always taken; the others compete by
//   score(n) = max over the G query heads of the kv head of <q_g, s_n>,
// s_n the block's summary, ties to the lower index. The result is the one that
// exact arithmetic gives, in ascending order, filled with -1.
//
// Scores: a 16x16x32 bf16 product, 16 rows of queries (A) times 16 summaries (B). A
// position's heads take adjacent rows, padded to a power of two by repeating the last
// head: a lane holds four rows of a block, so the maximum over the heads is taken in
// registers. A workgroup scores `pos` positions against all blocks they may choose
// from and keeps the scores in LDS; each wave then chooses for its own positions.
//
// Choice: fp32 products differ from exact ones by at most E = 2 D 2^-24 max|q| max|s|
// (2-norms; every one of the D additions rounds, or truncates, once; bf16 products are
// exact), so where the last score in and the first one out are more than 2 E apart the
// choice by fp32 scores is the exact one. Elsewhere only the blocks within 2 E of the
// border are scored again in 64 bits (products of bf16 are exact there and their sum
// is to 2^-53), in index order, and the best of them complete the list.
//
// The need-th largest of the scores, every 64th in a lane's registers, is bounded from
// below by the need-th largest of the lanes' largest ones. The few scores above that bound
// less 2 E, which hold every block within 2 E of the border too, then go one to a lane, in
// index order. In both lists each lane finds its rank by comparing its score with all of
// them (a bisection by ballots is a chain of dependent steps: 4096 queries of 256 blocks
// 70 -> 61 us). Where that does not apply (need > 64, or more than 64 such scores) a
// bisection counts all scores; a border of more than 64 (many equal scores) is settled in
// LDS.
//
// What bounds it: 4096 queries of 32/8 heads of 128, 16 of up to 1024 blocks (33 GFLOP),
// 98 us, 53 without the choice and 65 with made-up scores (10 of them the exact scores, which
// about 1% of the positions need): instructions, with two waves on a SIMD; the matrix
// cores are 12% busy. Two positions chosen step by step together need so many registers
// that it takes longer. One token of 16 sequences, 32 of 1024 blocks (25 MB), 11 us: launch,
// the summaries' loads, and one wave's choice, one after the other. 777 queries of 2 x 8/4
// heads of 64, 12 of 157 blocks, 13.1 us: two choices in a row by each wave.
#include "ef_device.hpp"
#include "ef_long.hpp"
#include "wave_ops.hpp"

#include <type_traits>

namespace ef {

namespace {

// LDS pointers by type: through plain ones the compiler loses sight of the address space
// and reads LDS with flat loads, which wait for each other (4096 queries of 1024 blocks
// 150 -> 130 us).
typedef __attribute__((address_space(3))) float lds_float;
typedef __attribute__((address_space(3))) int lds_int;
typedef __attribute__((address_space(3))) u32x4_t lds_chunk;
typedef __attribute__((address_space(3))) floatx4 lds_float4;

// Order-preserving integer of a float (no NaN).
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x);
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}

__device__ __forceinline__ float unordered(uint32_t u) {
  return __uint_as_float(u ^ ((u >> 31) ? 0x80000000u : 0xffffffffu));
}

// ordered(-inf), the score of a block whose products are NaN; a place without a block has 0.
constexpr uint32_t kLowest = 0x007fffffu;

// LDS written by other lanes of this wave becomes visible to it.
__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// f applied to x and the same value of other lanes: those at a DPP move's distance, or
// (OFF = 16, 32) lane l ^ OFF.
template <int CTRL>
__device__ __forceinline__ double dpp_mov64(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const float lo = dpp_mov<CTRL>(__uint_as_float((uint32_t)u));
  const float hi = dpp_mov<CTRL>(__uint_as_float((uint32_t)(u >> 32)));
  return __builtin_bit_cast(double, (uint64_t)__float_as_uint(hi) << 32 | __float_as_uint(lo));
}
template <int OFF>
__device__ __forceinline__ double pair_max64(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  float l0, l1, h0, h1;
  lane_pair<OFF>(__uint_as_float((uint32_t)u), l0, l1);
  lane_pair<OFF>(__uint_as_float((uint32_t)(u >> 32)), h0, h1);
  auto join = [](float lo, float hi) {
    return __builtin_bit_cast(double, (uint64_t)__float_as_uint(hi) << 32 | __float_as_uint(lo));
  };
  const double p = join(l0, h0), q = join(l1, h1);
  return p > q ? p : q;
}

// score(n) in 64 bits, by one wave, the same in every lane; NaN counts as -inf. 16
// lanes take a head, four heads at a time.
template <int D>
__device__ __forceinline__ double exact_score(const uint16_t* q, size_t head_stride, int G,
                                              const uint16_t* s) {
  constexpr int W = D / 32;  // words of two elements per lane
  const int lane = threadIdx.x & 63;
  const int sub = lane & 15;
  uint32_t sw[W];
#pragma unroll
  for (int e = 0; e < W; ++e) sw[e] = reinterpret_cast<const uint32_t*>(s)[sub * W + e];
  double best = -__builtin_inf();
  for (int g = lane >> 4; g - (lane >> 4) < G; g += 4) {
    const uint32_t* qg =
        reinterpret_cast<const uint32_t*>(q + min(g, G - 1) * head_stride) + sub * W;
    double x = 0.0;
#pragma unroll
    for (int e = 0; e < W; ++e) {
      const uint32_t w = qg[e];
      x += (double)bf16lo_to_f32(sw[e]) * (double)bf16lo_to_f32(w);
      x += (double)bf16hi_to_f32(sw[e]) * (double)bf16hi_to_f32(w);
    }
    x += dpp_mov64<kDppQuadXor1>(x);
    x += dpp_mov64<kDppQuadXor2>(x);
    x += dpp_mov64<kDppHalfMirror>(x);
    x += dpp_mov64<kDppRowRor8>(x);
    if (x > best) best = x;  // false for NaN
  }
  return pair_max64<32>(pair_max64<16>(best));
}

// Whether the queries of all G heads of a position are 0.
template <int D>
__device__ __forceinline__ bool all_zero(const uint16_t* q, size_t head_stride, int G) {
  const int lane = threadIdx.x & 63;
  uint32_t x = 0;
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int e = 0; e < D / 64; ++e) x |= q[g * head_stride + lane + 64 * e];
  return __ballot((x & 0x7fffu) != 0) == 0;
}

// The `want` best blocks among those of [c0, c1) whose fp32 score lies within
// [lo, hi], by exact score: their scores become +inf, the others' -inf. The best
// so far are held by the lanes, entry i in slot i / 64 of lane i % 64.
template <int D>
__device__ __forceinline__ void settle_border(lds_float* sc, int c0, int c1, float lo, float hi,
                                              int want, const uint16_t* q, size_t head_stride,
                                              int G, const uint16_t* s) {
  constexpr int SLOTS = kMaxTopk / 64;
  const int lane = threadIdx.x & 63;
  double val[SLOTS];
  int idx[SLOTS];
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) {
    val[i] = __builtin_inf();
    idx[i] = -1;
  }
  int held = 0;
  for (int base = c0; base < c1; base += 64) {
    const int n = base + lane;
    const float x = n < c1 ? sc[n] : kNegInf;
    const bool in = n < c1 && x >= lo && !(x > hi);
    unsigned long long todo = __ballot(in);
    if (in) sc[n] = kNegInf;
    while (todo) {
      const int m = base + __builtin_ctzll(todo);
      todo &= todo - 1;
      const double e = exact_score<D>(q, head_stride, G, s + (size_t)m * D);
      int at = held;  // entry that takes the block, -1: none
      if (held == want) {
        // Worst entry: lowest score, of equal ones the highest index.
        double w = val[0];
        int wi = idx[0], we = lane;
#pragma unroll
        for (int i = 1; i < SLOTS; ++i)
          if (val[i] < w || (val[i] == w && idx[i] > wi)) {
            w = val[i];
            wi = idx[i];
            we = lane + 64 * i;
          }
#pragma unroll
        for (int off = 1; off < 64; off *= 2) {
          const double ow = __shfl_xor(w, off, 64);
          const int oi = __shfl_xor(wi, off, 64), oe = __shfl_xor(we, off, 64);
          if (ow < w || (ow == w && oi > wi)) {
            w = ow;
            wi = oi;
            we = oe;
          }
        }
        at = e > w ? we : -1;
      } else {
        ++held;
      }
#pragma unroll
      for (int i = 0; i < SLOTS; ++i)
        if (at == lane + 64 * i) {
          val[i] = e;
          idx[i] = m;
        }
    }
  }
  wave_lds_sync();
#pragma unroll
  for (int i = 0; i < SLOTS; ++i)
    if (idx[i] >= 0) sc[idx[i]] = -kNegInf;
  wave_lds_sync();
}

// The scores of the blocks [c0, c1) of one position, every 64th in a lane's registers;
// with NV = 0 (more than 64 a lane) they stay in LDS.
template <int NV>
struct Scores {
  const lds_float* sc;
  int c0, c1;
  float v[NV > 0 ? NV : 1];
  __device__ __forceinline__ bool has(int i) const {
    return c0 + 64 * i + (int)(threadIdx.x & 63) < c1;
  }
  __device__ __forceinline__ float fetch(int i) const {  // -inf: no block
    const int n = c0 + 64 * i + (int)(threadIdx.x & 63);
    const float x = sc[min(n, c1 - 1)];
    return n < c1 ? x : kNegInf;
  }
  __device__ __forceinline__ void load() {
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = fetch(i);
  }
  // f(i, score of block c0 + 64 i + lane), ascending in i, all lanes together.
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    if constexpr (NV > 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) f(i, v[i]);
    } else {
      for (int i = 0; c0 + 64 * i < c1; ++i) f(i, fetch(i));
    }
  }
  // The same with the score as an integer, 0 where there is no block.
  template <class F>
  __device__ __forceinline__ void each_key(F f) const {
    each([&](int i, float x) { f(i, has(i) ? ordered(x) : 0u); });
  }
  // Scores from the value of `least` on, compared as floats, which cost no conversion: an
  // integer below kLowest is a NaN, from which on nothing would count, and at kLowest itself
  // places without a block would. Neither is asked for (see bisect).
  __device__ __forceinline__ int count(uint32_t least) const {
    const float t = unordered(least);
    int k = 0;
    each([&](int, float x) { k += (int)__popcll(__ballot(x >= t)); });
    return k;
  }
};

// Lanes of the set below this one, added to n.
__device__ __forceinline__ int rank_in(unsigned long long set, int n = 0) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(set >> 32),
                                        __builtin_amdgcn_mbcnt_lo((uint32_t)set, (uint32_t)n));
}

// A T in [lo, hi] with count(T) = need, or the largest with count(T) >= need, by halves of
// the interval of values, a step per bit of the answer's place among them (halving the
// integers would first look for its exponent), then of the integers between. On entry
// count(lo) = cnt >= need, lo is kLowest or more, and nothing is above hi; only integers
// above lo are counted, none of which is a NaN.
template <class F>
__device__ __forceinline__ uint32_t bisect(uint32_t lo, uint32_t hi, int need, int& cnt, F count) {
  for (int step = 0; cnt != need && lo < hi; ++step) {
    uint32_t mid = ordered(0.5f * unordered(lo) + 0.5f * unordered(hi));
    if (step >= 16 || mid <= lo || mid > hi) mid = hi - (hi - lo) / 2;
    const int n = count(mid);
    if (n >= need) {
      lo = mid;
      cnt = n;
    } else {
      hi = mid - 1;
    }
  }
  return lo;
}

// One position's choice among the blocks [c0, c1), which are more than the `need` wanted
// ones, by one wave. sc: the scores; bound: their largest error.
struct Choice {
  lds_float* sc;
  int c0, c1, need;
  float bound;
  bool summaries;  // whether some summary is not 0
  const uint16_t* q;  // the position's first head
  size_t head_stride;
  int G;
  const uint16_t* s;  // summaries of the kv head
  int* out;           // the position's list from its entry c0 on

  // Scores closer than this may change places (a score of -inf adds nothing to it; an
  // infinite bound stays infinite).
  __device__ __forceinline__ float apart(float x) const {
    return 2.f * bound + (fabsf(x) < -kNegInf ? 4.8e-7f * fabsf(x) : 0.f) + 1e-30f;
  }

  // Among the lanes of the set, each with a block, in ascending order: how many come
  // before this one's by exact score, then index.
  template <int D>
  __device__ __forceinline__ int exact_rank(unsigned long long set, int block) const {
    const int lane = threadIdx.x & 63;
    double exact = 0.0;
    for (unsigned long long m = set; m; m &= m - 1) {
      const int j = __builtin_ctzll(m);
      const int n = __builtin_amdgcn_readlane(block, j);
      const double e = exact_score<D>(q, head_stride, G, s + (size_t)n * D);
      if (lane == j) exact = e;
    }
    int rank = 0;
    for (unsigned long long m = set; m; m &= m - 1) {
      const int j = __builtin_ctzll(m);
      const double e = __shfl(exact, j, 64);
      rank += e > exact || (e == exact && j < lane) ? 1 : 0;
    }
    return rank;
  }
};

// How many of n scores in LDS (whole groups of 16, filled with -inf) are above x: their
// ranks by comparing each with each, two instructions a score, without a chain of
// dependent steps.
__device__ __forceinline__ int above(const lds_float* keys, int n, float x) {
  int rank = 0;
  for (int j = 0; j < n; j += 16) {
    floatx4 k[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) k[e] = reinterpret_cast<const lds_float4*>(keys + j)[e];
#pragma unroll
    for (int e = 0; e < 16; ++e) rank += k[e / 4][e % 4] > x ? 1 : 0;
  }
  return rank;
}

// x of the lowest lane of the set.
__device__ __forceinline__ float lane_of(float x, unsigned long long set) {
  return __builtin_bit_cast(
      float, __builtin_amdgcn_readlane(__float_as_int(x), __builtin_ctzll(set)));
}

// The need-th largest of the lanes' x, from their ranks; equal ones have the same rank.
__device__ __forceinline__ float nth(float x, int rank, int need) {
  unsigned long long m = 0;
  for (int r = need - 1; m == 0; --r) m = __ballot(rank == r);  // rank 0 is always there
  return lane_of(x, m);
}

// The choice by fp32 scores, and by exact ones where few scores come into question; false,
// with nothing written, where exact scores of more than 64 blocks are called for.
// scratch: 128 words of LDS of the wave.
template <int D, int NV>
__device__ __forceinline__ bool choose(const Choice& a, lds_int* scratch) {
  lds_float* const keys = (lds_float*)scratch;
  lds_int* const blocks = scratch + 64;
  const int lane = threadIdx.x & 63;
  const int c0 = a.c0, c1 = a.c1, need = a.need;
  Scores<NV> scores{a.sc, c0, c1, {}};
  scores.load();
  float best = kNegInf;  // this lane's largest
  scores.each([&](int, float x) { best = fmaxf(best, x); });
  const float most_of_all = __builtin_bit_cast(
      float, __builtin_amdgcn_readfirstlane(__float_as_int(wave_max(best))));
  const uint32_t top = ordered(most_of_all);
  // The few scores that can be in or near the border, one to a lane, in index order.
  float few = kNegInf;
  int few_block = c0 + lane, held = c1 - c0;
  uint32_t low = kLowest;  // no more than the need-th largest
  if (held <= 64) {
    if (lane < held) few = scores.fetch(0);
    keys[lane] = few;
  } else if (need <= 64) {
    keys[lane] = best;
    wave_lds_sync();
    const float least = nth(best, above(keys, 64, best), need);
    wave_lds_sync();  // read before they are written again
    low = ordered(least);
    // (Minus an infinite bound this is -inf, or NaN: then they are not few.)
    const float base = least - fmaxf(a.apart(least), a.apart(most_of_all));
    held = 0;
    scores.each([&](int, float x) { held += (int)__popcll(__ballot(x >= base)); });
    if (!(base > kNegInf)) held = 65;
    if (held <= 64) {
      keys[lane] = kNegInf;
      int at = 0;
      scores.each([&](int i, float x) {
        const unsigned long long m = __ballot(x >= base);
        if (x >= base) {
          const int slot = rank_in(m, at);
          keys[slot] = x;
          blocks[slot] = c0 + 64 * i + lane;
        }
        at += (int)__popcll(m);
      });
      wave_lds_sync();
      few = keys[lane];
      few_block = lane < held ? blocks[lane] : 0;
    }
  }
  if (held <= 64) {
    wave_lds_sync();
    const int rank = above(keys, held, few);
    bool take = rank < need;
    const unsigned long long taken = __ballot(take);
    // Last score in, first one out (where that is none of the few, more than e2 below).
    const float least = nth(few, rank, need);
    const unsigned long long out = __ballot(rank == need);
    const float e2 = a.apart(least);
    // More than `need` have rank < need where equal ones are at the border.
    if (__builtin_expect((int)__popcll(taken) != need ||
                             (held > need && !(least - lane_of(few, out) > e2)),
                         0)) {
      const bool here = lane < held;
      const bool finite = e2 < -kNegInf && least > kNegInf;
      const bool sure = here && finite && few > least + e2;
      const bool near = here && !sure && (!finite || few >= least - e2);
      const unsigned long long todo = __ballot(near);
      const int want = need - (int)__popcll(__ballot(sure));
      const int exact = a.template exact_rank<D>(todo, few_block);
      take = sure || (near && exact < want);
    }
    const int slot = rank_in(__ballot(take));
    if (take && slot < need) a.out[slot] = few_block;
    wave_lds_sync();  // read before the wave's next position writes
    return true;
  }

  // Too many for the lanes: the same on all scores, unless exact ones are called for.
  int cnt = low > kLowest ? scores.count(low) : c1 - c0;
  const uint32_t T = bisect(low, top, need, cnt, [&](uint32_t t) { return scores.count(t); });
  uint32_t in = 0xffffffffu, outside = 0;
  scores.each_key([&](int, uint32_t x) {
    in = min(in, x >= T ? x : 0xffffffffu);
    outside = max(outside, x >= T ? 0u : x);
  });
  const float least = unordered(wave_min(in));
  const float e2 = a.apart(least);
  uint32_t first = T, sure = T;  // scores from `sure` on are in, from `first` on perhaps
  unsigned long long chosen = 0;  // which of the latter, in index order
  if (cnt != need || !(least - unordered(wave_max(outside)) > e2)) {
    const bool finite = e2 < -kNegInf && least > kNegInf;
    if (!finite) return false;
    first = ordered(least - e2);
    sure = ordered(least + e2) + 1;
    const int want = need - scores.count(sure);
    int near = 0;
    scores.each_key([&](int i, uint32_t x) {
      const bool at = x >= first && x < sure;
      const unsigned long long m = __ballot(at);
      const int slot = rank_in(m, near);
      scratch[at ? min(slot, 64) : 64] = c0 + 64 * i + lane;
      near += (int)__popcll(m);
    });
    if (near > 64) return false;
    wave_lds_sync();
    const int block = lane < near ? scratch[lane] : 0;
    wave_lds_sync();
    const unsigned long long set = near < 64 ? (1ull << near) - 1 : ~0ull;
    const int rank = a.template exact_rank<D>(set, block);
    chosen = __ballot(lane < near && rank < want);
  }
  int at = 0, seen = 0;
  scores.each_key([&](int i, uint32_t x) {
    const unsigned long long m = __ballot(x >= first && x < sure);
    const int j = rank_in(m, seen);
    const bool take = x >= sure || (x >= first && j < 64 && (chosen >> j & 1));
    const unsigned long long t = __ballot(take);
    const int slot = rank_in(t, at);
    if (take && slot < need) a.out[slot] = c0 + 64 * i + lane;
    at += (int)__popcll(t);
    seen += (int)__popcll(m);
  });
  return true;
}

// The choice where more than 64 scores may be at the border.
template <int D>
__device__ __forceinline__ void choose_many(const Choice& a) {
  const int lane = threadIdx.x & 63;
  const int c0 = a.c0, c1 = a.c1, need = a.need;
  lds_float* const sc = a.sc;
  const Scores<0> scores{sc, c0, c1, {}};
  uint32_t top = 0;
  scores.each_key([&](int, uint32_t x) { top = max(top, x); });
  top = __builtin_amdgcn_readfirstlane(wave_max(top));
  int cnt = c1 - c0;
  uint32_t T = bisect(kLowest, top, need, cnt, [&](uint32_t t) { return scores.count(t); });
  uint32_t in = 0xffffffffu, outside = 0;
  scores.each_key([&](int, uint32_t x) {
    in = min(in, x >= T ? x : 0xffffffffu);
    outside = max(outside, x >= T ? 0u : x);
  });
  const float least = unordered(wave_min(in));
  const float next = cnt != need ? least : unordered(wave_max(outside));
  const float e2 = a.apart(least);
  if (!(least - next > e2)) {
    // Scores that are -inf (NaN), or 0 because all summaries or all of the
    // position's queries are, need no second look: their indices decide.
    const bool finite = e2 < -kNegInf;
    const bool settled =
        (finite && least == kNegInf) || !a.summaries || all_zero<D>(a.q, a.head_stride, a.G);
    const float lo = settled ? least : finite ? least - e2 : kNegInf;
    const float hi = settled ? least : finite ? least + e2 : -kNegInf;
    int sure = 0;
    for (int base = c0; base < c1; base += 64) {
      const int n = base + lane;
      sure += (int)__popcll(__ballot(n < c1 && sc[min(n, c1 - 1)] > hi));
    }
    int want = need - sure;
    float thr = hi;
    if (settled) {
      for (int base = c0; base < c1; base += 64) {
        const int n = base + lane;
        const bool tie = n < c1 && sc[min(n, c1 - 1)] == least;
        const unsigned long long m = __ballot(tie);
        const int rank = rank_in(m);
        if (tie) sc[n] = rank < want ? -kNegInf : kNegInf;
        want = max(want - (int)__popcll(m), 0);
      }
      wave_lds_sync();
      thr = least == kNegInf ? -3.402823466e+38f : least;
    } else {
      settle_border<D>(sc, c0, c1, lo, hi, want, a.q, a.head_stride, a.G, a.s);
    }
    T = ordered(thr);
  }
  int at = 0;
  scores.each_key([&](int i, uint32_t x) {
    const bool take = x >= T;
    const unsigned long long m = __ballot(take);
    const int slot = rank_in(m, at);
    if (take && slot < need) a.out[slot] = c0 + 64 * i + lane;
    at += (int)__popcll(m);
  });
}

// CT: 16-row tiles of queries per workgroup (G <= 16); 1 with `per` passes for
// G > 16. AHEAD: tiles of summaries a wave requests at once. LDS: floats of the score
// rows, 0: given at launch.
template <int D, int CT, int NW, int AHEAD, int LDS>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2)))
void block_select_kernel(SelectParams a) {
  constexpr int KS = D / 32;  // k-steps of the product
  extern __shared__ __align__(16) float launch_lds[];
  __shared__ __align__(16) float fixed_lds[LDS > 0 ? LDS : 4];
  float* const scores = LDS > 0 ? fixed_lds : launch_lds;  // [pos][stride]
  __shared__ __align__(16) u32x4_t tiles[NW][128];
  __shared__ __align__(16) int scratch[NW][128];
  __shared__ float norms[NW];
  __shared__ uint32_t nonzero[NW];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int bh = blockIdx.x / a.ptiles, pt = blockIdx.x % a.ptiles;
  const int b = bh / a.Hkv, hkv = bh % a.Hkv;
  const int p0 = pt * a.pos, npos = min(a.pos, a.Sq - p0);
  const uint16_t* sh = a.s + (size_t)bh * a.NB * D;
  const uint16_t* qh = a.q + ((size_t)b * a.Hq + (size_t)hkv * a.G) * a.Sq * D;
  const size_t head_stride = (size_t)a.Sq * D;

  const int c = lane & 15, kg = lane >> 4;
  // Summaries of AHEAD tiles of the wave from block n0 on. The first are requested
  // before the sequence's length is there.
  auto fetch = [&](int n0, u32x4_t (&x)[AHEAD][KS]) {
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const int n = n0 + j * NW * 16 + (k & 1) * 8 + (lane >> 3);
        const uint16_t* sp = sh + (size_t)min(n, a.NB - 1) * D + (k >> 1) * 64 + (lane & 7) * 8;
        x[j][k] = *reinterpret_cast<const u32x4_t*>(sp);
      }
  };
  // The lane's part of a tile as the product takes it: block c, elements 32 k + 8 kg on.
  // A load covers eight blocks' 128-byte lines; fragments read straight from memory touch
  // 16 lines in each quarter of a wave (with the score rows written without conditions,
  // one-token choice 15.7 -> 11.6 us, 4096 queries 130 -> 106).
  // The 64-element halves of a tile turn in a 2 KiB buffer of the wave, 16-byte chunks
  // permuted by row against bank conflicts; LDS keeps a wave's operations in order.
  auto turn = [&](const u32x4_t (&x)[KS], u32x4_t (&y)[KS]) {
    lds_chunk* const buf = (lds_chunk*)tiles[wave];
#pragma unroll
    for (int half = 0; half < KS / 2; ++half) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        buf[(i * 8 + (lane >> 3)) * 8 + ((lane & 7) ^ (lane >> 3))] = x[2 * half + i];
      wave_lds_sync();
#pragma unroll
      for (int i = 0; i < 2; ++i) y[2 * half + i] = buf[c * 8 + ((4 * i + kg) ^ (c & 7))];
      wave_lds_sync();
    }
  };
  auto queries = [&](int pass, u32x4_t (&x)[CT][KS]) {
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      const int p = a.per > 1 ? 0 : (t * 16 + c) / a.gp;
      const int g = a.per > 1 ? pass * 16 + c : c % a.gp;
      const uint16_t* qp =
          qh + min(g, a.G - 1) * head_stride + (size_t)(p0 + min(p, npos - 1)) * D + 8 * kg;
#pragma unroll
      for (int k = 0; k < KS; ++k) x[t][k] = *reinterpret_cast<const u32x4_t*>(qp + 32 * k);
    }
  };
  u32x4_t next[AHEAD][KS], qf[CT][KS];
  if (a.NB > 0) fetch(wave * 16, next);
  queries(0, qf);

  const int len = sequence_length(a.lengths, b, a.Skv);
  const long long diag0 = (long long)p0 + len - a.Sq;  // key of the first position
  auto own_block = [&](int p) {  // -1: before the first key
    const long long d = diag0 + p;
    return d < 0 ? -1 : (int)(d >> a.shift);
  };
  // Blocks that some position of the workgroup scores: below the last one's own.
  const int last = own_block(npos - 1);
  const int scored = last + 1 > a.K ? min(last - a.local + 1, a.NB) : 0;
  // Squares of the largest norms; the floor keeps the bound above what underflows.
  constexpr float kTinyNorm = 1e-36f;
  float mnorm = 0.f, qnorm = kTinyNorm;
  if (scored > 0) {
    auto norm2 = [](const u32x4_t (&x)[KS]) {  // of the lane's row (query or summary)
      float n2 = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) n2 = dot2_bf16(x[k][e], x[k][e], n2);
      float u, v;
      lane_pair<16>(n2, u, v);
      lane_pair<32>(u + v, u, v);
      return u + v;
    };
    // The score rows for GP rows to a position, in `per` passes where GP is 16. Rows of
    // the tiles without a position of their own repeat the last one, and lanes that
    // share a maximum write it to the same word, so no write needs a condition.
    auto score = [&](auto gp_tag) {
      constexpr int GP = decltype(gp_tag)::value;
      constexpr int PER = GP < 4 ? 4 / GP : 1;  // positions among a lane's four rows
      lds_float* row[CT][PER];
#pragma unroll
      for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int p = a.per > 1 ? 0 : (t * 16 + 4 * kg + i * GP) / GP;
          row[t][i] = (lds_float*)(scores + min(p, npos - 1) * a.stride + c);
        }
      for (int pass = 0; pass < (GP == 16 ? a.per : 1); ++pass) {
        if (pass > 0) {
          fetch(wave * 16, next);
          queries(pass, qf);
        }
#pragma unroll
        for (int t = 0; t < CT; ++t) qnorm = fmaxf(qnorm, norm2(qf[t]));
        for (int n0 = wave * 16; n0 < scored; n0 += AHEAD * NW * 16) {
          u32x4_t now[AHEAD][KS];
#pragma unroll
          for (int j = 0; j < AHEAD; ++j)
#pragma unroll
            for (int k = 0; k < KS; ++k) now[j][k] = next[j][k];
          if (n0 + AHEAD * NW * 16 < scored) fetch(n0 + AHEAD * NW * 16, next);
#pragma unroll
          for (int j = 0; j < AHEAD; ++j) {
            const int n = n0 + j * NW * 16;  // first block of the tile
            if (AHEAD > 1 && n >= scored) break;
            u32x4_t sf[KS];
            turn(now[j], sf);
            const float n2 = norm2(sf);  // blocks that no position scores may hold anything
            mnorm = fmaxf(mnorm, n + c < scored ? n2 : 0.f);
            floatx4 acc[CT];
#pragma unroll
            for (int t = 0; t < CT; ++t) acc[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
              for (int t = 0; t < CT; ++t)
                acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    __builtin_bit_cast(bf16x8_t, qf[t][k]), __builtin_bit_cast(bf16x8_t, sf[k]),
                    acc[t], 0, 0, 0);
            // Lane: block n + c, rows 4 kg + i of each tile. The maxima pass over NaN and
            // end at -inf.
#pragma unroll
            for (int t = 0; t < CT; ++t)
#pragma unroll
              for (int i = 0; i < PER; ++i) {
                float x = kNegInf;
#pragma unroll
                for (int e = 0; e < 4 / PER; ++e) x = fmaxf(x, acc[t][i * (4 / PER) + e]);
                float u, v;
                if constexpr (GP >= 8) {
                  lane_pair<16>(x, u, v);
                  x = fmaxf(u, v);
                }
                if constexpr (GP >= 16) {
                  lane_pair<32>(x, u, v);
                  x = fmaxf(u, v);
                  if (pass > 0) x = fmaxf(x, row[t][i][n]);
                }
                row[t][i][n] = x;
              }
          }
        }
      }
    };
    switch (a.gp) {
      case 1: score(std::integral_constant<int, 1>{}); break;
      case 2: score(std::integral_constant<int, 2>{}); break;
      case 4: score(std::integral_constant<int, 4>{}); break;
      case 8: score(std::integral_constant<int, 8>{}); break;
      default: score(std::integral_constant<int, 16>{}); break;
    }
    mnorm = wave_max(mnorm);
    qnorm = wave_max(qnorm);
    uint32_t bits = 1;
    if (mnorm == 0.f) {  // zeros, or too small for their squares
      bits = 0;
      for (int n0 = wave * 16; n0 < scored; n0 += NW * 16) {
        const uint32_t* sp = reinterpret_cast<const uint32_t*>(sh + (size_t)n0 * D);
        const int words = min(16, a.NB - n0) * (D / 2);
        for (int i = lane; i < words; i += 64) bits |= sp[i] & 0x7fff7fffu;
      }
    }
    const bool any = __ballot(bits != 0) != 0;
    if (lane == 0) {
      norms[wave] = fmaxf(mnorm, kTinyNorm);
      nonzero[wave] = any;
    }
  }
  __syncthreads();
  bool summaries = false;
  if (scored > 0) {
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      mnorm = fmaxf(mnorm, norms[w]);
      summaries = summaries || nonzero[w] != 0;
    }
  }
  const float bound = 1.01f * 2.f * D * 5.9604645e-8f * sqrtf(qnorm) * sqrtf(mnorm);

  for (int p = wave; p < npos; p += NW) {
    int* out = a.out + ((size_t)bh * a.Sq + p0 + p) * a.K;
    const int cur = own_block(p);
    if (cur + 1 <= a.K) {
      for (int i = lane; i < a.K; i += 64) out[i] = i <= cur ? i : -1;
      continue;
    }
    const int c0 = a.sinks, c1 = cur - a.local + 1;
    const Choice ch{(lds_float*)(scores + p * a.stride), c0, c1, a.K - c0 - a.local, bound,
                    summaries, qh + (size_t)(p0 + p) * D, head_stride, a.G, sh, out + c0};
    for (int i = lane; i < c0; i += 64) out[i] = i;
    for (int i = c1 + lane; i <= cur; i += 64) out[a.K - 1 - (cur - i)] = i;
    if (ch.need == 0) continue;
    lds_int* const words = (lds_int*)scratch[wave];
    const bool done = c1 - c0 <= 64 * 4    ? choose<D, 4>(ch, words)
                      : c1 - c0 <= 64 * 16 ? choose<D, 16>(ch, words)
                                           : choose<D, 0>(ch, words);
    if (!done) choose_many<D>(ch);
  }
}

template <int D, int CT, int NW, int AHEAD, int LDS>
hipError_t launch_one(const SelectParams& a, hipStream_t stream) {
  const size_t lds = LDS > 0 ? 0 : (size_t)a.pos * a.stride * sizeof(float);
  hipLaunchKernelGGL((block_select_kernel<D, CT, NW, AHEAD, LDS>),
                     dim3((unsigned)a.B * a.Hkv * a.ptiles), dim3(NW * 64), lds, stream, a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_d(const SelectParams& a, hipStream_t stream) {
  const int rows = a.per > 1 ? 16 : a.pos * a.gp;
  if (rows > 16) return launch_one<D, 4, 4, 2, kSelectLds / 4>(a, stream);
  if (a.waves == 8) return launch_one<D, 1, 8, 2, 0>(a, stream);
  return launch_one<D, 1, 4, 2, 0>(a, stream);
}

}  // namespace

hipError_t launch_block_select(const SelectParams& a, hipStream_t stream) {
  return a.D == 128 ? launch_d<128>(a, stream) : launch_d<64>(a, stream);
}

}  // namespace ef
