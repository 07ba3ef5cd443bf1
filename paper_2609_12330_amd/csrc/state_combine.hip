// Combine of stored partial states into bf16 rows: with M = max m_p,
//   o = sum_p e^(m_p - M) acc_p / sum_p e^(m_p - M) l_p   (0 where every m_p is -inf),
// the sums in fp32, one rounding to bf16 at the end.
//
// One wave per row. Lane p holds the reference and sum of state p (64 at a time, a
// running maximum carries over); each group of D / 4 lanes reads the value states of
// every other (D = 128) or fourth (D = 64) partition, 16 bytes a lane, the first ones
// requested before the weights are formed. A state without a key has weight and sum 0 and
// what stands in its value's place does not matter; a sum that is NaN (a query that is)
// makes the row NaN.
//
// Bound by latency: 2048 rows of 10 states of 128 (11 MB) 4.8 us.
#include "ef_device.hpp"
#include "ef_long.hpp"
#include "wave_ops.hpp"

namespace ef {

namespace {

constexpr int kCombineWaves = 4;

template <int D>
__global__ __launch_bounds__(kCombineWaves * 64) void state_combine_kernel(StateCombineParams a) {
  constexpr int LPS = D / 4;    // lanes per state
  constexpr int SPL = 64 / LPS;  // states per wave-wide load
  const int lane = threadIdx.x & 63;
  const int row = blockIdx.x * kCombineWaves + (threadIdx.x >> 6);
  if (row >= a.rows) return;
  const size_t base = (size_t)row * a.P;
  const int grp = lane / LPS, ch = lane % LPS;
  constexpr int BATCH = 8;  // value states of a lane in flight
  float M = kNegInf, L = 0.f;
  floatx4 x = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < a.P; p0 += 64) {
    const int count = min(a.P - p0, 64);
    const float m = lane < count ? a.m[base + p0 + lane] : kNegInf;
    const float l = lane < count ? a.l[base + p0 + lane] : 0.f;
    floatx4 y[BATCH];
    auto fetch = [&](int j) {
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int q = min(j + i * SPL + grp, count - 1);
        y[i] = *reinterpret_cast<const floatx4*>(a.acc + (base + p0 + q) * D + 4 * ch);
      }
    };
    fetch(0);
    const float top = fmaxf(M, wave_max(m));
    const float ref = top == kNegInf ? 0.f : top;
    const float w = exp2_fast((m - ref) * kLog2e);  // 0 where m = -inf
    const float old = exp2_fast((M - ref) * kLog2e);
    L = L * old + wave_sum(w * l);
    M = top;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] *= old;
    for (int j = 0; j < count; j += BATCH * SPL) {
      if (j > 0) fetch(j);
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        // The weight of this group's state (0 from `count` on).
        float wq = 0.f;
#pragma unroll
        for (int g = 0; g < SPL; ++g) {
          const float wg = __int_as_float(__builtin_amdgcn_readlane(
              __float_as_int(w), min(j + i * SPL + g, 63)));
          wq = grp == g ? wg : wq;
        }
        if (j + i * SPL + grp > 63) wq = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = wq > 0.f ? fmaf(wq, y[i][e], x[e]) : x[e];
      }
    }
  }
#pragma unroll
  for (int off = LPS; off < 64; off *= 2)
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += shfl_xor(x[e], off);
  if (grp != 0) return;
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const u32x2_t o = {pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv)};
  *reinterpret_cast<u32x2_t*>(a.o + (size_t)row * D + 4 * ch) = o;
}

}  // namespace

hipError_t launch_state_combine(const StateCombineParams& a, hipStream_t stream) {
  const dim3 grid((a.rows + kCombineWaves - 1) / kCombineWaves);
  if (a.D == 128)
    hipLaunchKernelGGL(state_combine_kernel<128>, grid, dim3(kCombineWaves * 64), 0, stream, a);
  else
    hipLaunchKernelGGL(state_combine_kernel<64>, grid, dim3(kCombineWaves * 64), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ef
