// Combine of stored partial states into bf16 rows: with M = max m_p,
//   o = sum_p e^(m_p - M) acc_p / sum_p e^(m_p - M) l_p   (0 where every m_p is -inf),
// the sums in fp32, one rounding to bf16 at the end.
//
// One wave per row: the lanes first form the weights of up to 64 states at a time
// (a running maximum carries over), then each group of D / 4 lanes reads the value
// states of every other (D = 128) or fourth (D = 64) partition, 16 bytes a lane. A
// state without a key has weight 0 and is not read.
#include "ef_device.hpp"
#include "ef_long.hpp"

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
  float M = kNegInf, L = 0.f;
  floatx4 x = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < a.P; p0 += 64) {
    const int p = p0 + lane;
    const float m = p < a.P ? a.m[base + p] : kNegInf;
    const float l = p < a.P ? a.l[base + p] : 0.f;
    float top = fmaxf(M, m);
#pragma unroll
    for (int off = 1; off < 64; off *= 2) top = fmaxf(top, shfl_xor(top, off));
    const float ref = top == kNegInf ? 0.f : top;
    const float w = exp2_fast((m - ref) * kLog2e);  // 0 where m = -inf
    const float old = exp2_fast((M - ref) * kLog2e);
    float sum = w > 0.f ? w * l : 0.f;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) sum += shfl_xor(sum, off);
    L = L * old + sum;
    M = top;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] *= old;
    const int count = min(a.P - p0, 64);
    for (int j = 0; j < count; j += 4 * SPL) {
      floatx4 y[4];
      float wj[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int q = j + i * SPL + grp;
        wj[i] = __shfl(w, min(q, 63), 64);
        if (q >= count) wj[i] = 0.f;
        y[i] = floatx4{0.f, 0.f, 0.f, 0.f};
        if (wj[i] > 0.f)
          y[i] = *reinterpret_cast<const floatx4*>(a.acc + (base + p0 + q) * D + 4 * ch);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = fmaf(wj[i], y[i][e], x[e]);
    }
  }
#pragma unroll
  for (int off = LPS; off < 64; off *= 2)
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += shfl_xor(x[e], off);
  if (grp != 0) return;
  const float inv = L > 0.f ? 1.f / L : 0.f;
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
