// What the long-context attention kernels share around the rolling loop
// (rolling.hpp): the operand layout of a wave's 32 query rows, the walk over a list
// of key tiles, and the epilogue, which writes bf16 rows or fp32 partial states.
#pragma once

#include "ef_long.hpp"
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
// first half; any other tile may be ragged.
template <int D, bool SEL, class Tiles>
__device__ __forceinline__ void roll_tiles(const Tiles& tiles, int n, bool active,
                                           const Stages& st, const FragmentReads<D>& fr,
                                           Rows<D>& rows, float c, const KeyMask& mask) {
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
  wait_tile_loads();
  __syncthreads();
  if (active) {
    tile_scores<D>(st.k0, fr.k, rows.qf, xb, xa);
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
    tiles.template load<false>(st.v1, t1);
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
  const float inv = l > 0.f ? 1.f / l : 0.f;
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
template <int D>
__device__ __forceinline__ void store_state(const Rows<D>& rows, int h, bool valid, float* m,
                                            float* l, float* acc, size_t slot) {
  const float lt = rows.lsum + __shfl_xor(rows.lsum, 32, 64);
  if (!valid) return;
  const bool none = rows.mref == kNoRef;
  if (h == 0) {
    m[slot] = none ? kNegInf : rows.mref;
    l[slot] = lt;
  }
  if (none) return;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const floatx16& x = rows.oacc[i];
      *reinterpret_cast<float4*>(acc + slot * D + 32 * i + 8 * q + 4 * h) =
          make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
    }
}

}  // namespace ef
