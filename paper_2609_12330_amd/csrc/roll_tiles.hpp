// What the long-context attention kernels share around the rolling loop
// (rolling.hpp): the operand layout of a wave's 32 query rows, the walk over a list
// of key tiles, and the epilogue, which writes bf16 rows or fp32 partial states.
#pragma once

#include "ef_long.hpp"
#include "group_combine.hpp"
#include "rolling.hpp"

namespace ef {

// LDS offsets of a lane's fragment reads inside a stage (see attn_mfma.hip).
template <int D>
struct FragmentReads {
  using Geo = TileGeom<D>;
  int k[D / 16], v[D / 32];
  __device__ __forceinline__ void init(int lane) {
    const int h = lane >> 5, ql = lane & 31;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) k[s] = ql * Geo::ROW + ((2 * s + h) ^ Geo::swz_k(ql)) * 16;
    const int j16 = lane & 15, grp = lane >> 4;
    const int vr = 4 * (grp >> 1) + (j16 >> 2);
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) {
      const int d_off = 32 * dt + 16 * (grp & 1) + 4 * (j16 & 3);
      v[dt] = vr * Geo::ROW + (((d_off >> 3) ^ Geo::swz_v(vr)) * 16) + 2 * (d_off & 7);
    }
  }
};

// A wave's 32 query rows: operands, and the state they carry.
template <int D>
struct Rows {
  static constexpr int DT = D / 32;
  bf16x8_t qf[D / 16];
  floatx16 oacc[DT];
  float mref, lsum;  // reference (base-2 units) and this lane's half of the row sum
  __device__ __forceinline__ void init(const uint16_t* qrow, bool valid, uint32_t flip, int h) {
    const u32x4_t* qp = reinterpret_cast<const u32x4_t*>(qrow);
    const u32x4_t zero = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      const u32x4_t x = (valid ? qp[2 * s + h] : zero) ^ flip;
      qf[s] = __builtin_bit_cast(bf16x8_t, x);
    }
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) oacc[i][j] = 0.f;
    mref = kNoRef;
    lsum = 0.f;
  }
  // A query that is not finite: what this lane holds of it becomes 0, so that its scores are
  // finite, and the row's sum NaN where the row sees a key (`sees`). Left to the scores, an
  // infinite element could make them all -inf, as if no key were visible, and a NaN would
  // pass the offset of rows that do not see a tile. The sum stays NaN through every
  // rescaling and combine.
  template <class Sees>
  __device__ __forceinline__ void guard(Sees sees) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    u16x2 most = {0, 0};  // largest magnitudes, as integers
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      const u32x4_t x = __builtin_bit_cast(u32x4_t, qf[s]);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, x[e] & 0x7fff7fffu));
    }
    const bool bad = most[0] >= 0x7f80 || most[1] >= 0x7f80;
    const bool poison = bad && sees();
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      u32x4_t x = __builtin_bit_cast(u32x4_t, qf[s]);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = bad ? 0u : x[e];
      qf[s] = __builtin_bit_cast(bf16x8_t, x);
    }
    lsum = poison ? __builtin_nanf("") : lsum;
  }
};

// The four stages of a workgroup, objects of their own so that the compiler tells
// the loads into some from the reads of others.
struct Stages {
  char *k0, *k1, *v0, *v1;
};

// Walks the first n tiles of a list with the rolling loop. `tiles` gives each tile
// (at), loads it into a stage (load) and, with SEL, says whether this lane's row
// sees it (on). A wave without rows (`active` false) only loads. Every wave of the
// workgroup makes the call with the same n. The list's last tile may end in its
// first half; any other tile may be ragged. What `mask` and the tiles say of masks need
// not be there before `ready` is called, behind the first loads. `sees` says whether this
// lane's row sees a key in any workgroup (Rows::guard).
template <int D, bool SEL, class Tiles, class Ready, class Sees>
__device__ __forceinline__ void roll_tiles(const Tiles& tiles, int n, bool active,
                                           const Stages& st, const FragmentReads<D>& fr,
                                           Rows<D>& rows, float c, const KeyMask& mask,
                                           Ready ready, Sees sees) {
  if (n <= 0) return;
  constexpr int SUB = TileGeom<D>::SUB;
  Rolling<D, SEL> ro{fr.k, fr.v, rows.qf, rows.oacc, rows.lsum, rows.mref, c};
  floatx16 xa, xb;        // scores of odd and even subtiles
  uint32_t pa[8], pb[8];  // their weights
  float top = 0.f;        // unused without renewals
  auto tile = [&](int t) { return t < n ? tiles.at(t) : TileAt{0, 0, false, false}; };
  TileAt t0 = tile(0), t1 = tile(1), t2;
  const TileAt end = tile(n - 1);
  const int nsub = 2 * n - (end.base + 32 >= end.end ? 1 : 0);
  const int steps = nsub / 2;
  tiles.template load<true>(st.k0, t0);
  tiles.template load<false>(st.v0, t0);
  tiles.template load<true>(st.k1, t1);
  tiles.template load<false>(st.v1, t1);  // all four stages are free: a short walk waits once
  ready();
  t0 = tile(0);
  t1 = tile(1);
  wait_tile_loads();
  __syncthreads();
  if (active) {
    tile_scores<D>(st.k0, fr.k, rows.qf, xb, xa);
    // Keys are finite, so before masks every score of a query that is not is infinite or NaN
    // (an infinite element against a 0): one tells. One token over 16 blocks 9.72 -> 9.86
    // us; a look at every element of the queries takes 9.95.
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(fabsf(xb[0]) < -kNegInf)) != 0, 0)) {
      rows.guard(sees);
      tile_scores<D>(st.k0, fr.k, rows.qf, xb, xa);
    }
    if (t0.masked) {
      mask(xb, t0.base, t0.end);
      mask(xa, t0.base + 32, t0.end);
      t0.masked = false;  // both halves are
    }
    if constexpr (SEL) ro.select(tiles.on(0));
    ro.resume(xb, xa, pb);
  }
  __syncthreads();
  for (int u = 0; u < steps; u += 2) {
    t2 = tile(u + 2);
    tiles.template load<true>(st.k0, t2);
    if (u > 0) tiles.template load<false>(st.v1, t1);
    if (active)
      pair_compute<D, false>(st.k1, st.v0, ro, t0, t1, 2 * u + 2 < nsub, top, mask, xa, xb, pa,
                             pb, tiles.on(u), tiles.on(min(u + 1, n - 1)));
    wait_tile_loads();
    __syncthreads();
    if (u + 1 >= steps) break;
    t0 = tile(u + 3);
    tiles.template load<true>(st.k1, t0);
    tiles.template load<false>(st.v0, t2);
    if (active)
      pair_compute<D, false>(st.k0, st.v1, ro, t1, t2, 2 * u + 4 < nsub, top, mask, xa, xb, pa,
                             pb, tiles.on(u + 1), tiles.on(min(u + 2, n - 1)));
    wait_tile_loads();
    __syncthreads();
    t1 = t0;
    t0 = t2;
  }
  if (active) {
    const int last = nsub - 1;
    const char* vl = (last >> 1 & 1) ? st.v1 : st.v0;
    if (last & 1)
      ro.last_values(pa, vl + SUB);
    else
      ro.last_values(pb, vl);
  }
  __syncthreads();  // the stages may be loaded again
}

// This lane's half of a row (channels 32 dt + 8 q + 4 h .. + 4) as bf16 values of
// the finished row, or as the fp32 state of a partition in `slot`.
template <int D>
__device__ __forceinline__ void store_row(const Rows<D>& rows, int h, uint16_t* orow) {
  const float l = rows.lsum + __shfl_xor(rows.lsum, 32, 64);  // both lane halves of the row
  if (orow == nullptr) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;  // NaN stays NaN
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const floatx16& x = rows.oacc[i];
      const u32x2_t w = {pack_bf16x2(x[4 * q] * inv, x[4 * q + 1] * inv),
                         pack_bf16x2(x[4 * q + 2] * inv, x[4 * q + 3] * inv)};
      *reinterpret_cast<u32x2_t*>(orow + 32 * i + 8 * q + 4 * h) = w;
    }
}
// With `shared` the state is read by another workgroup of the launch: device-scope
// stores (see group_combine.hpp).
template <int D>
__device__ __forceinline__ void store_state(const Rows<D>& rows, int h, bool valid, float* m,
                                            float* l, float* acc, size_t slot, bool shared) {
  const float lt = rows.lsum + __shfl_xor(rows.lsum, 32, 64);
  if (!valid) return;
  const bool none = rows.mref == kNoRef;
  const float mref = none ? kNegInf : rows.mref * kLn2;  // natural-log units
  if (shared) {
    if (h == 0) {
      store_dev(m + slot, mref);
      store_dev(l + slot, lt);
    }
    if (none) return;
    // (Shared states are few: their offsets fit 32 bits.)
    const __amdgpu_buffer_rsrc_t rs =
        __builtin_amdgcn_make_buffer_rsrc(acc, (short)0, -1, 0x00020000);
    const unsigned off = ((unsigned)slot * D + 4 * h) * 4u;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const floatx16& x = rows.oacc[i];
        const floatx4 v = {x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, v), rs,
                                               (int)(off + (32 * i + 8 * q) * 4), 0,
                                               16 /* device scope */);
      }
    return;
  }
  if (h == 0) {
    m[slot] = mref;
    l[slot] = lt;
  }
  if (none) return;
  float* const row = acc + slot * D + 4 * h;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const floatx16& x = rows.oacc[i];
      *reinterpret_cast<float4*>(row + 32 * i + 8 * q) =
          make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
    }
}

// Combine, by the workgroup that stored the last of them, of the P states of rows row0
// .. row0 + nrows - 1 into bf16 rows: what state_combine.hip does, on device-scope
// loads. D / 4 lanes take a row, four channels each; P <= 2 kSharedParts.
template <int D, int NT>
__device__ __forceinline__ void combine_shared(const float* m, const float* l, const float* acc,
                                               uint16_t* o, size_t row0, int nrows, int P) {
  constexpr int LPR = D / 4;  // lanes per row
  static_assert(2 * kSharedParts <= LPR, "a lane for each state's weight");
  static_assert(NT / LPR * D == kSharedElems, "the rows of a round");
  const int ch = threadIdx.x % LPR;
  // Rows are taken in whole waves: the lanes of a wave shuffle together.
  for (int r0 = 0; r0 < nrows; r0 += NT / LPR) {
    const int r = r0 + (int)threadIdx.x / LPR;
    const bool valid = r < nrows;
    const size_t base = (row0 + (valid ? r : 0)) * P;
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<float*>(acc + row0 * P * D), (short)0, nrows * P * D * 4, 0x00020000);
    const int off = ((valid ? r : 0) * P * D + 4 * ch) * 4;
    const float mv = ch < P ? load_dev(m + base + ch) : kNegInf;
    const float lv = ch < P ? load_dev(l + base + ch) : 0.f;
    u32x4_t y[kSharedParts];
#pragma unroll
    for (int j = 0; j < kSharedParts; ++j) y[j] = load16_dev(rs, off + min(j, P - 1) * D * 4);
    float M = mv;
#pragma unroll
    for (int x = 1; x < LPR; x *= 2) M = fmaxf(M, shfl_xor(M, x));
    const float w = exp2_fast((mv - (M == kNegInf ? 0.f : M)) * kLog2e);  // 0: no key, no state
    float L = w * lv;
#pragma unroll
    for (int x = 1; x < LPR; x *= 2) L += shfl_xor(L, x);
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = 0; p0 < P; p0 += kSharedParts) {
      if (p0 > 0) {
#pragma unroll
        for (int j = 0; j < kSharedParts; ++j)
          y[j] = load16_dev(rs, off + min(p0 + j, P - 1) * D * 4);
      }
#pragma unroll
      for (int j = 0; j < kSharedParts; ++j) {
        const float wp = __shfl(w, p0 + j, LPR);
#pragma unroll
        for (int e = 0; e < 4; ++e)  // (a state without a key was not stored)
          s[e] = wp > 0.f ? fmaf(wp, __uint_as_float(y[j][e]), s[e]) : s[e];
      }
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;  // NaN stays NaN
    const u32x2_t x = {pack_bf16x2(s[0] * inv, s[1] * inv), pack_bf16x2(s[2] * inv, s[3] * inv)};
    if (valid) *reinterpret_cast<u32x2_t*>(o + (row0 + r) * D + 4 * ch) = x;
  }
}

// The output rows made visibly invalid, where the arrivals cannot be trusted (a counter
// that was not zero when the launch began: at the number of arrivals or above it every
// workgroup does this and none combines; below it nothing in the launch tells).
template <int D, int NT>
__device__ __forceinline__ void poison_rows(uint16_t* o, size_t row0, int nrows) {
  for (int i = threadIdx.x; i < nrows * D; i += NT) o[row0 * D + i] = 0x7fc0;
}

}  // namespace ef
