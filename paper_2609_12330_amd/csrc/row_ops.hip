// Rows of new tokens: rotary positions, and the append of keys and values to a paged cache.
//
// A pair (a, b) of a row turns by the angle 2 pi p f, p the token's position, f the pair's turns
// per position: y_a = A (a cos - b sin), y_b = A (b cos + a sin). The turns p f are formed in 64
// bits and only their fraction goes on: at p = 10^6 an fp32 product would be off by 0.06 turns.
// A workgroup takes 1 to 16 tokens and all or a share of their rows. It forms each token's
// cosines and sines once, in LDS, while its rows are on their way; then every lane turns 16
// elements, two 16-byte chunks that hold whole pairs in either layout. A, cos and sin are joined
// in 64 bits and rounded to fp32; products and sums round one by one (no fused ones), so the
// result is the same however the compiler pairs them.
//
// 8-bit rows: the largest magnitude of a row is taken over its D / 16 lanes; the scale is a power
// of two, so x / s is exact and a code carries one rounding.
//
// Bound by HBM (each row read and written once): 11006 tokens of 32 heads of 128 rotated (180 MB)
// 32.7 us, 5.5 TB/s; prompts of 9000 tokens of 32/8 heads of 128 to an 8-bit cache (203 MB) 43 us, 4.7
// TB/s, with the codes' arithmetic. For few tokens by latency: starts, then lengths, then the table's
// entry, with the rows' loads beside them (one token of 16 sequences 3.9 us).
#include "ef_device.hpp"
#include "ef_serve.hpp"

namespace ef {

namespace {

constexpr int kMaxPer = 16;

struct Chunks {
  uint32_t a[4], b[4];  // elements 0 .. 7 and 8 .. 15 of a lane, bf16 pairs
};

// Smallest power of two s >= 2^-100 with top <= 448 s: 448 = 1.75 * 2^8.
__device__ __forceinline__ float power_scale(float top) {
  const uint32_t u = __float_as_uint(top);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return __uint_as_float((uint32_t)(max(e, -100) + 127) << 23);
}

// Codes of four values x / s; not finite ones are NaN (0x7f).
__device__ __forceinline__ uint32_t codes4(const float* x, float inv) {
  int w = 0;
  w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, w, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, w, true);
  uint32_t u = (uint32_t)w;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (!(fabsf(x[i]) < -kNegInf)) u = (u & ~(0xffu << 8 * i)) | 0x7fu << 8 * i;
  return u;
}

template <int D, bool E4M3, bool ONCE>
__global__ __launch_bounds__(256) void rows_kernel(RowsParams a) {
#pragma clang fp contract(off)
  constexpr int LPR = D / 16;  // lanes of a row
  __shared__ float2 turn[kMaxPer][D / 2];
  __shared__ long long pos[kMaxPer];  // position
  __shared__ int seq[kMaxPer];        // sequence, -1: none
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t0 = (int)(blockIdx.x / a.blocks) * a.per;
  const int share = (int)(blockIdx.x % a.blocks);
  const int per = min(a.per, a.T - t0);
  const int rows = a.Hq + 2 * a.Hkv;

  // The tokens' places, one to a lane: starts ascend, so a token's sequence is the first token's
  // or one behind it.
  if (wave == 0) {
    int b = a.positions != nullptr ? 0 : find_sequence(a.starts, a.B, a.T, t0);
    if (lane < per) {
      const int t = t0 + lane;
      long long p = 0;
      if (a.positions != nullptr) {
        p = a.positions[t];
      } else {
        int end = 0;  // first row behind the sequence
        while (b < a.B && (end = sequence_start(a.starts, b + 1, a.B, a.T)) <= t) ++b;
        if (b >= a.B) b = -1;
        // len_b - n_b + (t - start_b), where n_b = end_b - start_b
        if (b >= 0) p = (long long)a.lengths[b] + t - end;
      }
      pos[lane] = p;
      seq[lane] = b;
    }
  }
  // This lane's first row goes out for its elements before the angles are formed.
  const int ch = threadIdx.x % LPR;
  const int rh = a.rot / 2;
  // Offsets of its two chunks.
  const bool turned = a.turns != nullptr && 16 * ch < a.rot;
  const int o1 = turned && !a.interleaved ? 8 * ch : 16 * ch;
  const int o2 = turned && !a.interleaved ? 8 * ch + rh : 16 * ch + 8;
  const int total = per * rows, stride = a.blocks * (256 / LPR);
  int r = share * (256 / LPR) + (int)threadIdx.x / LPR;
  auto source = [&](int i, int& n, int& h) -> const uint16_t* {
    n = i / rows;
    h = i - n * rows;
    const size_t t = (size_t)(t0 + n);
    if (h < a.Hq) return a.q + (t * a.Hq + h) * D;
    const int hk = h - a.Hq;
    return hk < a.Hkv ? a.k + (t * a.Hkv + hk) * D : a.v + (t * a.Hkv + hk - a.Hkv) * D;
  };
  auto fetch = [&](const uint16_t* p, u32x4_t& x, u32x4_t& y) {
    x = *reinterpret_cast<const u32x4_t*>(p + o1);
    y = *reinterpret_cast<const u32x4_t*>(p + o2);
  };
  // Outputs that no cache can hold for their reader stream past them.
  auto store = [&](auto v, auto* p) {
    auto* const q = reinterpret_cast<decltype(v)*>(p);
    if constexpr (ONCE)
      __builtin_nontemporal_store(v, q);
    else
      *q = v;
  };
  u32x4_t x = {0u, 0u, 0u, 0u}, y = x;
  int n = 0, h = 0;
  if (r < total) fetch(source(r, n, h), x, y);

  __syncthreads();
  if (a.turns != nullptr) {
    for (int i = threadIdx.x; i < per * rh; i += 256) {
      const int w = i / rh, j = i - w * rh;
      double f = (double)pos[w] * a.turns[j];
      f -= floor(f);
      double s, c;
      sincospi(2.0 * f, &s, &c);
      const float sf = (float)(s * a.amplitude);
      turn[w][j] = make_float2((float)(c * a.amplitude), a.transpose ? -sf : sf);
    }
    __syncthreads();
  }

  for (; r < total; r += stride) {
    const int cn = n, chd = h;
    float u[8], w[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u[2 * i] = bf16lo_to_f32(x[i]);
      u[2 * i + 1] = bf16hi_to_f32(x[i]);
      w[2 * i] = bf16lo_to_f32(y[i]);
      w[2 * i + 1] = bf16hi_to_f32(y[i]);
    }
    if (r + stride < total) fetch(source(r + stride, n, h), x, y);
    if (turned && chd < a.Hq + a.Hkv) {
      const float2* tw = &turn[cn][8 * ch];
      if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 f = tw[i], g = tw[4 + i];
          const float u0 = u[2 * i], u1 = u[2 * i + 1], w0 = w[2 * i], w1 = w[2 * i + 1];
          u[2 * i] = u0 * f.x - u1 * f.y;
          u[2 * i + 1] = u1 * f.x + u0 * f.y;
          w[2 * i] = w0 * g.x - w1 * g.y;
          w[2 * i + 1] = w1 * g.x + w0 * g.y;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 f = tw[i];
          const float u0 = u[i], w0 = w[i];
          u[i] = u0 * f.x - w0 * f.y;
          w[i] = w0 * f.x + u0 * f.y;
        }
      }
    }
    const int b = seq[cn];
    uint16_t* to = nullptr;  // bf16 row
    size_t cell = 0;         // row of the cache
    bool cached = false;
    const bool isk = chd < a.Hq + a.Hkv;
    if (chd < a.Hq) {
      if (b >= 0) to = a.q_out + ((size_t)(t0 + cn) * a.Hq + chd) * D;
    } else if (b >= 0) {
      const long long p = pos[cn];
      const int hk = isk ? chd - a.Hq : chd - a.Hq - a.Hkv;
      if (p >= 0 && p < (long long)a.c.width << a.c.shift) {
        const int page = a.c.table[(size_t)b * a.c.width + (int)(p >> a.c.shift)];
        if ((unsigned)page < (unsigned)a.c.pages) {
          cell = (((size_t)page * a.Hkv + hk) << a.c.shift) + ((int)p & ((1 << a.c.shift) - 1));
          cached = true;
          if constexpr (!E4M3) to = reinterpret_cast<uint16_t*>(isk ? a.c.k : a.c.v) + cell * D;
        }
      }
    }
    if (E4M3 && chd >= a.Hq) {
      float top = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {  // (fmaxf passes over NaN)
        const float m = fabsf(u[i]), l = fabsf(w[i]);
        top = fmaxf(top, m < -kNegInf ? m : 0.f);
        top = fmaxf(top, l < -kNegInf ? l : 0.f);
      }
      if constexpr (LPR == 8) top = fmaxf(top, dpp_mov<kDppHalfMirror>(top));
      top = fmaxf(top, dpp_mov<kDppQuadXor2>(top));
      top = fmaxf(top, dpp_mov<kDppQuadXor1>(top));
      const float s = power_scale(top), inv = 1.f / s;
      if (cached) {
        char* const row = (isk ? a.c.k : a.c.v) + cell * D;
        const u32x2_t c1 = {codes4(u, inv), codes4(u + 4, inv)};
        const u32x2_t c2 = {codes4(w, inv), codes4(w + 4, inv)};
        store(c1, row + o1);
        store(c2, row + o2);
        if (ch == 0) (isk ? a.c.k_scale : a.c.v_scale)[cell] = s;
      }
    } else if (to != nullptr) {
      u32x4_t p1, p2;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p1[i] = pack_bf16x2(u[2 * i], u[2 * i + 1]);
        p2[i] = pack_bf16x2(w[2 * i], w[2 * i + 1]);
      }
      store(p1, to + o1);
      store(p2, to + o2);
    }
  }
}

template <int D>
hipError_t launch_d(const RowsParams& a, bool e4m3, hipStream_t stream) {
  const dim3 grid((unsigned)((a.T + a.per - 1) / a.per) * a.blocks);
  auto* const kernel = e4m3 ? (a.once ? rows_kernel<D, true, true> : rows_kernel<D, true, false>)
                            : (a.once ? rows_kernel<D, false, true> : rows_kernel<D, false, false>);
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rows(const RowsParams& a, bool e4m3, hipStream_t stream) {
  return a.D == 128 ? launch_d<128>(a, e4m3, stream) : launch_d<64>(a, e4m3, stream);
}

}  // namespace ef
