// Cached keys and values as packed bf16 rows.
//
// A copy: every 16 bytes of output are one lane's, from 16 bytes of a bf16 page or 8 codes and
// their row's scale. A workgroup takes up to 16 packed rows (tokens) of all heads; their sequences
// and pages are found once and kept in LDS. A lane requests four pieces before it stores one.
//
// Bound by HBM: codes and rows read once, rows written once: 179000 positions of 8 heads of 128 in
// bf16 (1.47 GB) 258 us, 5.7 TB/s (one piece at a time 276); 14 contexts of 264 of 32 heads of 64
// 29 -> 13.6 us with the pieces in flight and fewer tokens to a workgroup.
#include "ef_device.hpp"
#include "ef_serve.hpp"

namespace ef {

namespace {

constexpr int kMaxTokens = 16;  // packed rows of a workgroup
constexpr int kPieces = 4;      // a lane's loads in flight

// ONCE: more rows than the caches hold for their reader, stores stream past them.
template <int D, bool E4M3, bool ONCE>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheReadParams a) {
  constexpr int LPR = D / 8;  // lanes of a row
  __shared__ long long cell0[kMaxTokens];  // the token's row of head 0, -1: NaN, -2: no sequence
  const int t0 = blockIdx.x * a.per;
  const int n = min(a.per, a.T - t0);
  if (threadIdx.x < 64) {
    int b = find_sequence(a.starts, a.B, a.T, t0);
    const int lane = threadIdx.x, t = t0 + lane;
    if (lane < n) {
      // starts ascend: the token's sequence is the first token's or one behind it.
      while (b < a.B && sequence_start(a.starts, b + 1, a.B, a.T) <= t) ++b;
      long long c = -2;
      if (b >= 0 && b < a.B) {
        const int p = t - sequence_start(a.starts, b, a.B, a.T);
        c = -1;
        if (p >= 0 && p < (long long)a.c.width << a.c.shift) {
          const int page = a.c.table[(size_t)b * a.c.width + (p >> a.c.shift)];
          if ((unsigned)page < (unsigned)a.c.pages)
            c = (((long long)page * a.Hkv) << a.c.shift) + (p & ((1 << a.c.shift) - 1));
        }
      }
      cell0[lane] = c;
    }
  }
  __syncthreads();
  const int ch = threadIdx.x % LPR;
  const int per = n * a.Hkv;
  constexpr int STEP = 256 / LPR;
  for (int i0 = threadIdx.x / LPR; i0 < 2 * per; i0 += kPieces * STEP) {
    u32x4_t x[kPieces];
    float scale[kPieces];
    uint16_t* to[kPieces];
    bool held[kPieces];
#pragma unroll
    for (int e = 0; e < kPieces; ++e) {
      const int i = i0 + e * STEP;
      const bool isv = i >= per;
      const int j = isv ? i - per : i;
      const int h = (unsigned)j / (unsigned)n, m = j - h * n;
      const long long c = i < 2 * per ? cell0[m] : -2;
      to[e] = c == -2 ? nullptr
                      : (isv ? a.v_out : a.k_out) + ((size_t)(t0 + m) * a.Hkv + h) * D + 8 * ch;
      held[e] = c >= 0;
      x[e] = {0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
      if (c >= 0) {
        const size_t cell = (size_t)c + ((size_t)h << a.c.shift);
        const char* const base = isv ? a.c.v : a.c.k;
        if constexpr (E4M3) {
          const u32x2_t w = __builtin_nontemporal_load(
              reinterpret_cast<const u32x2_t*>(base + cell * D + 8 * ch));
          x[e][0] = w[0];
          x[e][1] = w[1];
          scale[e] = (isv ? a.c.v_scale : a.c.k_scale)[cell];
        } else {
          x[e] = __builtin_nontemporal_load(
              reinterpret_cast<const u32x4_t*>(base + (cell * D + 8 * ch) * 2));
        }
      }
    }
#pragma unroll
    for (int e = 0; e < kPieces; ++e) {
      if (to[e] == nullptr) continue;
      if constexpr (E4M3) {
        if (held[e]) {
          const u32x2_t w = {x[e][0], x[e][1]};
          const float s = scale[e];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            x[e][2 * y] = pack_bf16x2(__builtin_amdgcn_cvt_f32_fp8((int)w[y], 0) * s,
                                      __builtin_amdgcn_cvt_f32_fp8((int)w[y], 1) * s);
            x[e][2 * y + 1] = pack_bf16x2(__builtin_amdgcn_cvt_f32_fp8((int)w[y], 2) * s,
                                          __builtin_amdgcn_cvt_f32_fp8((int)w[y], 3) * s);
          }
        }
      }
      if constexpr (ONCE)
        __builtin_nontemporal_store(x[e], reinterpret_cast<u32x4_t*>(to[e]));
      else
        *reinterpret_cast<u32x4_t*>(to[e]) = x[e];
    }
  }
}

template <int D>
hipError_t launch_d(const CacheReadParams& a, bool e4m3, hipStream_t stream) {
  const dim3 grid((unsigned)((a.T + a.per - 1) / a.per));
  auto* const kernel =
      e4m3 ? (a.once ? cache_read_kernel<D, true, true> : cache_read_kernel<D, true, false>)
           : (a.once ? cache_read_kernel<D, false, true> : cache_read_kernel<D, false, false>);
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_read(const CacheReadParams& a, bool e4m3, hipStream_t stream) {
  return a.D == 128 ? launch_d<128>(a, e4m3, stream) : launch_d<64>(a, e4m3, stream);
}

}  // namespace ef
