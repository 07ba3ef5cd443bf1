// Block summaries: the mean key of every block of 64 or 128 keys of a cache,
//   s[b][h][n] = (1 / c) sum of the c valid keys of block n   (0 when c = 0),
// summed in fp32 and rounded to bf16 once (the product that reads it takes bf16).
//
// Bound by HBM, a read of every key once: 8 sequences of 20011 to 32768 keys, 8 heads of
// 128, 441 MB in 71 us, 6.2 TB/s (a large read runs at 6.3 to 6.5). One wave owns a
// block: D / 8 lanes hold a key's 16-byte chunks, so a wave-wide load covers 512 / D
// whole keys and all loads of 64 keys are in flight before the first is used. The loads
// are non-temporal (80 us without) and go through a descriptor of the block's valid
// keys. The lanes that hold the same chunk of other keys meet in registers (DPP and lane
// swaps), and the first D / 8 lanes store the row.
#include "ef_long.hpp"
#include "ef_device.hpp"

namespace ef {

namespace {

constexpr int kSummaryWaves = 4;

template <int OFF>
__device__ __forceinline__ void sum_lanes(float (&x)[8]) {
  if constexpr (OFF < 64) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float a, b;
      lane_pair<OFF>(x[e], a, b);
      x[e] = a + b;
    }
    sum_lanes<2 * OFF>(x);
  }
}

template <int D>
__global__ __launch_bounds__(kSummaryWaves * 64) void block_summary_kernel(SummaryParams a) {
  constexpr int LPR = D / 8;      // lanes per key
  constexpr int KPL = 64 / LPR;   // keys per wave-wide load
  constexpr int LOADS = 64 / KPL;  // loads of 64 keys
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long item = (long long)blockIdx.x * kSummaryWaves + wave;
  if (item >= (long long)a.B * a.Hkv * a.touched) return;
  const int t = (int)(item % a.touched);
  const long long bh = item / a.touched;
  const int len = sequence_length(a.lengths, (int)(bh / a.Hkv), a.Skv);
  int n = t;
  if (a.new_keys > 0) {
    n += max(len - a.new_keys, 0) / a.block;
    if (n >= a.NB || (long long)n * a.block >= len) return;
  }
  const int first = n * a.block;  // below Skv + block
  const int count = min(max(len - first, 0), a.block);
  const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint16_t*>(a.k + ((size_t)bh * a.Skv + (count > 0 ? first : 0)) * D), (short)0,
      count * 2 * D, 0x00020000);
  const int key = lane / LPR, chunk = lane % LPR;
  float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int base = 0; base < count; base += 64) {
    u32x4_t w[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int j = base + i * KPL + key;  // reads as 0 past the last key
      w[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, (j * LPR + chunk) * 16, 0,
                                                   2 /* non-temporal */);
    }
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[2 * e] += bf16lo_to_f32(w[i][e]);
        x[2 * e + 1] += bf16hi_to_f32(w[i][e]);
      }
  }
  sum_lanes<LPR>(x);
  if (key != 0) return;
  const float c = (float)max(count, 1);
  u32x4_t o;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = pack_bf16x2(x[2 * e] / c, x[2 * e + 1] / c);
  reinterpret_cast<u32x4_t*>(a.s + ((size_t)bh * a.NB + n) * D)[chunk] = o;
}

}  // namespace

hipError_t launch_block_summary(const SummaryParams& a, hipStream_t stream) {
  const long long items = (long long)a.B * a.Hkv * a.touched;
  const dim3 grid((unsigned)((items + kSummaryWaves - 1) / kSummaryWaves));
  if (a.D == 128)
    hipLaunchKernelGGL(block_summary_kernel<128>, grid, dim3(kSummaryWaves * 64), 0, stream, a);
  else
    hipLaunchKernelGGL(block_summary_kernel<64>, grid, dim3(kSummaryWaves * 64), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ef
