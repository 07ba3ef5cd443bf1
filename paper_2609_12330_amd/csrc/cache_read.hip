// Cached keys and values as packed bf16 rows.
//
// A copy: every 16 bytes of output are one lane's, from 16 bytes of a bf16 page or 8 codes and
// their row's scale. A workgroup takes 16 packed rows (tokens) of all heads; their sequences
// and pages are found once and kept in LDS.
//
// Bound by HBM: codes and rows read once, rows written once.
#include "ef_device.hpp"
#include "ef_serve.hpp"

namespace ef {

namespace {

constexpr int kTokens = 16;  // packed rows of a workgroup

template <int D, bool E4M3>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheReadParams a) {
  constexpr int LPR = D / 8;  // lanes of a row
  __shared__ long long cell0[kTokens];  // the token's row of head 0, -1: NaN, -2: no sequence
  const int t0 = blockIdx.x * kTokens;
  const int n = min(kTokens, a.T - t0);
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
  for (int i = threadIdx.x / LPR; i < 2 * per; i += 256 / LPR) {
    const bool isv = i >= per;
    const int j = isv ? i - per : i;
    const int h = j / n, m = j - h * n;
    const long long c = cell0[m];
    if (c == -2) continue;
    u32x4_t x = {0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
    if (c >= 0) {
      const size_t cell = (size_t)c + ((size_t)h << a.c.shift);
      const char* const base = isv ? a.c.v : a.c.k;
      if constexpr (E4M3) {
        const u32x2_t w = __builtin_nontemporal_load(
            reinterpret_cast<const u32x2_t*>(base + cell * D + 8 * ch));
        const float s = (isv ? a.c.v_scale : a.c.k_scale)[cell];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          x[2 * e] = pack_bf16x2(__builtin_amdgcn_cvt_f32_fp8((int)w[e], 0) * s,
                                 __builtin_amdgcn_cvt_f32_fp8((int)w[e], 1) * s);
          x[2 * e + 1] = pack_bf16x2(__builtin_amdgcn_cvt_f32_fp8((int)w[e], 2) * s,
                                     __builtin_amdgcn_cvt_f32_fp8((int)w[e], 3) * s);
        }
      } else {
        x = __builtin_nontemporal_load(
            reinterpret_cast<const u32x4_t*>(base + (cell * D + 8 * ch) * 2));
      }
    }
    uint16_t* const to = (isv ? a.v_out : a.k_out) + ((size_t)(t0 + m) * a.Hkv + h) * D + 8 * ch;
    *reinterpret_cast<u32x4_t*>(to) = x;
  }
}

template <int D>
hipError_t launch_d(const CacheReadParams& a, bool e4m3, hipStream_t stream) {
  const dim3 grid((unsigned)((a.T + kTokens - 1) / kTokens));
  if (e4m3)
    hipLaunchKernelGGL((cache_read_kernel<D, true>), grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((cache_read_kernel<D, false>), grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_read(const CacheReadParams& a, bool e4m3, hipStream_t stream) {
  return a.D == 128 ? launch_d<128>(a, e4m3, stream) : launch_d<64>(a, e4m3, stream);
}

}  // namespace ef
