// Block selection: for every query position and kv head the `K` blocks of the
// key axis that its attention reads. The first `sinks` blocks and the last `local`
// ones up to the query's own are always taken; the others compete by
//   score(n) = max over the G query heads of the kv head of <q_g, s_n>,
// s_n the block's summary, ties to the lower index. The result is the one that
// exact arithmetic gives, in ascending order, filled with -1.
//
// Scores: a 16x16x32 bf16 product, 16 summaries (A) times 16 columns of queries
// (B). A position's heads take adjacent columns, padded to a power of two by
// repeating the last head, so the maximum over them is a few DPP moves. A
// workgroup scores `pos` positions against all blocks they may choose from and
// keeps the scores in LDS; each wave then chooses for its own positions.
//
// Choice: the need-th largest score is found by bisection over the bits of the
// scores (as order-preserving integers), counting with ballots. fp32 products
// differ from exact ones by at most E = 2 D 2^-24 max|q| max|s| (2-norms; every
// one of the D additions rounds, or truncates, once; bf16 products are exact), so
// where the last score in and the first one out are more than 2 E apart the choice
// is the exact one. Elsewhere only the blocks within 2 E of the border are scored
// again in 64 bits (products of bf16 are exact there and their sum is to 2^-53),
// in index order, and the best of them complete the list.
#include "ef_long.hpp"
#include "ef_device.hpp"

namespace ef {

namespace {

// Order-preserving integer of a float (no NaN).
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x);
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) x = fmaxf(x, shfl_xor(x, m));
  return x;
}
__device__ __forceinline__ float wave_min(float x) { return -wave_max(-x); }

// LDS written by other lanes of this wave becomes visible to it.
__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// score(n) in 64 bits, by one wave; NaN counts as -inf.
template <int D>
__device__ double exact_score(const uint16_t* q, size_t head_stride, int G, const uint16_t* s) {
  constexpr int E = D / 64;  // elements per lane
  const int lane = threadIdx.x & 63;
  double best = -__builtin_inf();
  double m[E];
#pragma unroll
  for (int e = 0; e < E; ++e) m[e] = (double)__uint_as_float((uint32_t)s[lane + 64 * e] << 16);
  for (int g = 0; g < G; ++g) {
    const uint16_t* qg = q + g * head_stride;
    double x = 0.0;
#pragma unroll
    for (int e = 0; e < E; ++e)
      x += m[e] * (double)__uint_as_float((uint32_t)qg[lane + 64 * e] << 16);
#pragma unroll
    for (int off = 1; off < 64; off *= 2) x += __shfl_xor(x, off, 64);
    if (x > best) best = x;  // false for NaN
  }
  return best;
}

// Whether the queries of all G heads of a position are 0.
template <int D>
__device__ bool all_zero(const uint16_t* q, size_t head_stride, int G) {
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
__device__ void settle_border(float* sc, int c0, int c1, float lo, float hi, int want,
                              const uint16_t* q, size_t head_stride, int G, const uint16_t* s) {
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
      const int j = __builtin_ctzll(todo);
      todo &= todo - 1;
      const int m = base + j;
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

// CT: 16-column tiles of queries per workgroup (G <= 16); 1 with `per` passes
// for G > 16.
template <int D, int CT, int NW>
__global__ __launch_bounds__(NW * 64) void block_select_kernel(SelectParams a) {
  constexpr int KS = D / 32;  // k-steps of the product
  extern __shared__ __align__(16) float scores[];  // [pos][stride]
  __shared__ float norms[NW];
  __shared__ uint32_t nonzero[NW];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int bh = blockIdx.x / a.ptiles, pt = blockIdx.x % a.ptiles;
  const int b = bh / a.Hkv, hkv = bh % a.Hkv;
  const int len = sequence_length(a.lengths, b, a.Skv);
  const int p0 = pt * a.pos, npos = min(a.pos, a.Sq - p0);
  const long long diag0 = (long long)p0 + len - a.Sq;  // key of the first position
  auto own_block = [&](int p) {  // -1: before the first key
    const long long d = diag0 + p;
    return d < 0 ? -1 : (int)(d >> a.shift);
  };
  const uint16_t* sh = a.s + (size_t)bh * a.NB * D;
  const uint16_t* qh = a.q + ((size_t)b * a.Hq + (size_t)hkv * a.G) * a.Sq * D;
  const size_t head_stride = (size_t)a.Sq * D;

  // Blocks that some position of the workgroup scores: below the last one's own.
  const int last = own_block(npos - 1);
  const int scored = last + 1 > a.K ? min(last - a.local + 1, a.NB) : 0;
  // Squares of the largest norms; the floor keeps the bound above what underflows.
  float mnorm = 1e-36f, qnorm = 1e-36f;
  uint32_t mbits = 0;  // whether some summary is not 0
  if (scored > 0) {
    const int c = lane & 15, kg = lane >> 4;
    for (int pass = 0; pass < a.per; ++pass) {
      bf16x8_t qf[CT][KS];
#pragma unroll
      for (int t = 0; t < CT; ++t) {
        const int p = a.per > 1 ? 0 : (t * 16 + c) / a.gp;
        const int g = a.per > 1 ? pass * 16 + c : c % a.gp;
        const uint16_t* qp =
            qh + min(g, a.G - 1) * head_stride + (size_t)(p0 + min(p, npos - 1)) * D;
        float n2 = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const u32x4_t x = *reinterpret_cast<const u32x4_t*>(qp + 32 * k + 8 * kg);
          qf[t][k] = __builtin_bit_cast(bf16x8_t, x);
#pragma unroll
          for (int e = 0; e < 4; ++e) n2 = dot2_bf16(x[e], x[e], n2);
        }
        float u, v;
        lane_pair<16>(n2, u, v);
        lane_pair<32>(u + v, u, v);
        qnorm = fmaxf(qnorm, u + v);
      }
      for (int n0 = wave * 16; n0 < scored; n0 += NW * 16) {
        const uint16_t* sp = sh + (size_t)min(n0 + c, a.NB - 1) * D + 8 * kg;
        bf16x8_t sf[KS];
        float n2 = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const u32x4_t x = *reinterpret_cast<const u32x4_t*>(sp + 32 * k);
          sf[k] = __builtin_bit_cast(bf16x8_t, x);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            n2 = dot2_bf16(x[e], x[e], n2);
            mbits |= x[e];
          }
        }
        float u, v;
        lane_pair<16>(n2, u, v);
        lane_pair<32>(u + v, u, v);
        mnorm = fmaxf(mnorm, u + v);
#pragma unroll
        for (int t = 0; t < CT; ++t) {
          floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < KS; ++k)
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(sf[k], qf[t][k], acc, 0, 0, 0);
          // Lane: column c, blocks n0 + 4 kg + i.
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float x = acc[i] == acc[i] ? acc[i] : kNegInf;
            if (a.gp > 1) x = fmaxf(x, dpp_mov<kDppQuadXor1>(x));
            if (a.gp > 2) x = fmaxf(x, dpp_mov<kDppQuadXor2>(x));
            if (a.gp > 4) x = fmaxf(x, dpp_mov<kDppHalfMirror>(x));
            if (a.gp > 8) x = fmaxf(x, dpp_mov<kDppRowRor8>(x));
            acc[i] = x;
          }
          const int p = a.per > 1 ? 0 : (t * 16 + c) / a.gp;
          if (c % a.gp == 0 && p < npos) {
            float4* dst = reinterpret_cast<float4*>(scores + p * a.stride + n0 + 4 * kg);
            float4 x = make_float4(acc[0], acc[1], acc[2], acc[3]);
            if (pass > 0) {  // the same lane wrote the earlier heads' maximum
              const float4 y = *dst;
              x = make_float4(fmaxf(x.x, y.x), fmaxf(x.y, y.y), fmaxf(x.z, y.z), fmaxf(x.w, y.w));
            }
            *dst = x;
          }
        }
      }
    }
    mnorm = wave_max(mnorm);
    qnorm = wave_max(qnorm);
    const bool any = __ballot((mbits & 0x7fff7fffu) != 0) != 0;
    if (lane == 0) {
      norms[wave] = mnorm;
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
    float* sc = scores + p * a.stride;
    const int c0 = a.sinks, c1 = cur - a.local + 1;
    const int need = a.K - a.sinks - a.local;  // below c1 - c0
    float thr = -kNegInf;  // blocks of [c0, c1) with a score >= thr are taken
    bool none = need == 0;
    if (!none) {
      uint32_t T = 0;
      int cnt = c1 - c0;
      for (int bit = 31; bit >= 0 && cnt != need; --bit) {
        const uint32_t cand = T | (1u << bit);
        int k = 0;
        for (int base = c0; base < c1; base += 64) {
          const int n = base + lane;
          k += (int)__popcll(__ballot(n < c1 && ordered(sc[min(n, c1 - 1)]) >= cand));
        }
        if (k >= need) {
          T = cand;
          cnt = k;
        }
      }
      // Last score in, first one out.
      float in = -kNegInf, outv = kNegInf;
      for (int n = c0 + lane; n < c1; n += 64) {
        const float x = sc[n];
        if (ordered(x) >= T) in = fminf(in, x);
        else outv = fmaxf(outv, x);
      }
      in = wave_min(in);
      outv = wave_max(outv);
      if (cnt != need) outv = in;
      // (in = -inf adds nothing; an infinite bound stays infinite.)
      const float e2 = 2.f * bound + (in == kNegInf ? 0.f : 4.8e-7f * fabsf(in)) + 1e-30f;
      thr = in;
      if (!(in - outv > e2)) {
        // Scores that are -inf (NaN), or 0 because all summaries or all of the
        // position's queries are, need no second look: their indices decide.
        const bool finite = e2 < -kNegInf;
        const bool settled = (finite && in == kNegInf) || !summaries ||
                             all_zero<D>(qh + (size_t)(p0 + p) * D, head_stride, a.G);
        const float lo = settled ? in : finite ? in - e2 : kNegInf;
        const float hi = settled ? in : finite ? in + e2 : -kNegInf;
        int sure = 0;
        for (int base = c0; base < c1; base += 64) {
          const int n = base + lane;
          sure += (int)__popcll(__ballot(n < c1 && sc[min(n, c1 - 1)] > hi));
        }
        int want = need - sure;
        if (settled) {
          for (int base = c0; base < c1; base += 64) {
            const int n = base + lane;
            const bool tie = n < c1 && sc[min(n, c1 - 1)] == in;
            const unsigned long long m = __ballot(tie);
            const int rank = (int)__popcll(m & ((1ull << lane) - 1));
            if (tie) sc[n] = rank < want ? -kNegInf : kNegInf;
            want = max(want - (int)__popcll(m), 0);
          }
          wave_lds_sync();
          thr = in == kNegInf ? -3.402823466e+38f : in;
        } else {
          settle_border<D>(sc, c0, c1, lo, hi, want, qh + (size_t)(p0 + p) * D, head_stride, a.G,
                           sh);
          thr = hi;
        }
      }
    }
    int at = 0;
    for (int base = 0; base <= cur; base += 64) {
      const int n = base + lane;
      const bool take = n <= cur && (n < c0 || n >= c1 || (!none && sc[n] >= thr));
      const unsigned long long m = __ballot(take);
      const int slot = at + (int)__popcll(m & ((1ull << lane) - 1));
      if (take && slot < a.K) out[slot] = n;
      at += (int)__popcll(m);
    }
  }
}

constexpr int kSelectWaves = 8;

template <int D, int CT>
hipError_t launch_ct(const SelectParams& a, hipStream_t stream) {
  const size_t lds = (size_t)a.pos * a.stride * sizeof(float);
  hipLaunchKernelGGL((block_select_kernel<D, CT, kSelectWaves>),
                     dim3((unsigned)a.B * a.Hkv * a.ptiles), dim3(kSelectWaves * 64), lds, stream,
                     a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_d(const SelectParams& a, hipStream_t stream) {
  const int columns = a.per > 1 ? 16 : a.pos * a.gp;
  if (columns <= 16) return launch_ct<D, 1>(a, stream);
  return launch_ct<D, 4>(a, stream);
}

}  // namespace

hipError_t launch_block_select(const SelectParams& a, hipStream_t stream) {
  return a.D == 128 ? launch_d<128>(a, stream) : launch_d<64>(a, stream);
}

}  // namespace ef
