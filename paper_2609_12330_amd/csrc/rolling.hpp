// The rolling loop of the matrix-core attention kernels: 64-key tiles of K and V
// in LDS, three 32-key subtiles in flight (scores, softmax, values), and the loads
// that feed it. See attn_mfma.hip for the operand layout.
#pragma once

#include "ef_device.hpp"
#include "ef_kernels.hpp"

namespace ef {

constexpr float kLazySum = 256.f;      // 2^8: a lane's weights whose sum is below are too
constexpr float kNoRef = -3.402823466e+38f;  // rolling loop: no key seen yet (-FLT_MAX)
constexpr float kRenewDepth = 16.f;  // a renewed reference lies at most this far below the top

// Geometry of K and V rows in LDS.
template <int D>
struct TileGeom {
  static constexpr int KCH = D / 8;        // 16-byte chunks per row
  static constexpr int ROW = 2 * D;        // bytes per K or V row (no padding: swizzled)
  static constexpr int RPI = 64 / KCH;     // rows one wave-wide direct load fills (1 KiB)
  static constexpr int SUB = 32 * ROW;     // bytes of 32 rows
  // Streaming loop: V stage 0, V stage 1, K stage 0, K stage 1 of 32 keys each.
  template <int S>
  static constexpr int v_off() { return S * SUB; }
  template <int S>
  static constexpr int k_off() { return (2 + S) * SUB; }
  // Tiles sit row-major in LDS with their 16-byte chunks permuted per row
  // (chunk c of row r at slot c ^ swz(r)), so the fragment reads below hit
  // distinct banks: K rows are read 16 rows at a time at one chunk, V rows four
  // rows at a time at 32 consecutive bytes (transposing reads).
  static __device__ __forceinline__ int swz_k(int r) { return D == 128 ? (r & 15) : ((r >> 1) & 7); }
  static __device__ __forceinline__ int swz_v(int r) {
    return D == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1);
  }
};

// Cross-half exchange: max of x over lanes l and l ^ 32.
__device__ __forceinline__ float max_with_other_half(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Waits for this wave's direct-to-LDS loads (they count as vector memory loads).
__device__ __forceinline__ void wait_tile_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }

// Scores of the keys hidden from this lane's row set to -inf: past the run's end
// or the causal limit `lim`, or at most `lo` (left of the window) and not a sink.
// Element i holds key kb + 4 h + o(i) with a compile-time offset o, so the hidden
// keys become per-lane offset thresholds, clamped to the tile so the arithmetic
// cannot overflow: past `vis`, and inside [wlo, whi]. Selects, not branches.
__device__ __forceinline__ void mask_scores(floatx16& x, int kb, int kend, int lim, int lo,
                                            int sinks, int h) {
  const int base = kb + 4 * h;
  const int vis = min(min(kend - 1, lim), kb + 32) - base;
  const int wlo = max(sinks, kb) - base;
  const int whi = min(max(lo, kb - 1), kb + 32) - base;
  if (__builtin_amdgcn_ballot_w64(whi >= wlo)) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int o = 8 * (i >> 2) + (i & 3);
      const bool hide = (o > vis) | ((o >= wlo) & (o <= whi));
      x[i] = hide ? kNegInf : x[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int o = 8 * (i >> 2) + (i & 3);
      x[i] = o > vis ? kNegInf : x[i];
    }
  }
}

// S^T of both 32-key subtiles of the 64-key tile at kt, their products alternating.
template <int D>
__device__ __forceinline__ void tile_scores(const char* kt, const int* kread, const bf16x8_t* qf,
                                            floatx16& x0, floatx16& x1) {
  constexpr int SUB = TileGeom<D>::SUB;
#pragma unroll
  for (int i = 0; i < 16; ++i) x0[i] = x1[i] = 0.f;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    const u32x4_t k0 = *reinterpret_cast<const u32x4_t*>(kt + kread[s]);
    const u32x4_t k1 = *reinterpret_cast<const u32x4_t*>(kt + SUB + kread[s]);
    x0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k0), qf[s], x0, 0,
                                                0, 0);
    x1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k1), qf[s], x1, 0,
                                                0, 0);
  }
}

// Compile-time loop: f(integral_constant<int, 0>) ... f(integral_constant<int, N - 1>).
template <int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (N > 0) {
    static_for<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}

// The rolling loop's work on one 32-key subtile j: its softmax, beside the
// scores of subtile j + 1 and the values of subtile j - 1.
//
// What bounds it: the matrix core and, on long launches, the power limit (the
// clock falls from 2.4 to about 1.75 GHz under this loop; a library matrix
// product of random bf16 data runs at 1.77 GHz too). Before, a step formed a
// tile's weights and multiplied its values one after the other, took the tile's
// maximum on every step and spent about a hundred scalar instructions on tile
// addresses; its matrix cores were busy 54% of the time on 8192 keys at
// D = 128, whatever order the compiler issued the step in. Here
//  - all products of a subtile are independent of the softmax beside them, and
//    scheduling barriers pin one product, its share of the vector work (3-4
//    instructions) and the fragment reads PF products ahead to each slot;
//  - the maximum is only taken when a lane's sum of weights passes 2^8
//    (soft_end), 57 vector instructions per 16 weights instead of 74;
//  - tile loads keep one address register set for all tiles (StageLoader).
// Together the matrix cores are busy 61.5-63% of the time: 8192 x 8192 keys,
// 32/8 heads, 1064 -> 984 us; causal 4 x 2048, 168.5 -> 156.5 us; 1024 of 32768
// keys, 32 heads, one branch 521 -> 490 us. Tried on top, not kept: fragments
// read 4, 5 or 7 slots ahead (equal); eight waves sharing each tile (clock 1.89
// GHz but 59.6% busy: 8192^2 920 us against 945, causal 4 x 2048 160 against 154);
// 64 rows per wave, one wave per SIMD (half the fragment reads, 2.1 GHz, 51%
// busy: 952 and 171 us); three or four stages per tile (25 us against 20 on a
// 777-token prompt).
//
// With SEL a tile may be hidden from single rows as a whole (a block that other rows
// of the workgroup selected): select() sets the offset of such a row's exponents to
// -inf, so its weights are 0 at the cost of one instruction a subtile.
template <int D, bool SEL = false>
struct Rolling {
  using Geo = TileGeom<D>;
  static constexpr bool SELECTS = SEL;
  static constexpr int KSTEPS = D / 16;
  static constexpr int DT = D / 32;
  static constexpr int NV = 2 * DT;            // value products of a subtile
  static constexpr int SLOTS = KSTEPS + NV;    // products of a subtile
  static constexpr int PF = 6;                 // slots a fragment is read ahead of its product

  // Products of a subtile in issue order: scores and values alternate, so that
  // a product rarely follows the one it accumulates onto. The last two are
  // values, so the scores are complete when the next subtile reads them; that
  // leaves the last two scores one behind the other, the subtile's one dependent
  // pair.
  static constexpr bool is_score(int i) {
    return i < SLOTS - 4 ? i % 2 == 0 : i < SLOTS - 2;
  }
  static constexpr int index_of(int i) {  // k-step of a score slot, number of a value slot
    int n = 0;
    for (int k = 0; k < i; ++k) n += is_score(k) == is_score(i);
    return n;
  }

  // Fragment offsets and operands of the wave, and the state carried along.
  const int* kread;
  const int* vread;
  const bf16x8_t* qf;
  floatx16* oacc;
  float& lsum;
  float& mref;
  float c;
  bool on = true;     // SEL: whether this lane's row sees the tile
  float bias = 0.f;   // SEL: -reference, or -inf where it does not

  __device__ __forceinline__ void select(bool sees) {
    on = sees;
    rebias();
  }
  __device__ __forceinline__ void rebias() {
    if constexpr (SEL) bias = on ? -mref : kNegInf;
  }
  // The largest score of a row counts for its reference only where the row sees it.
  __device__ __forceinline__ float seen(float cand) const {
    return !SEL || on ? cand : kNegInf;
  }

  // Fragment of product i of a subtile, K and V subtiles at kt and vt.
  template <int I>
  __device__ __forceinline__ u32x4_t fragment(const char* kt, const char* vt) const {
    constexpr int n = index_of(I);
    if constexpr (is_score(I)) {
      return *reinterpret_cast<const u32x4_t*>(kt + kread[n]);
    } else {
      typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
      const char* p = vt + vread[n % DT] + 16 * (n / DT) * Geo::ROW;
      const bf16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
          (__attribute__((address_space(3))) bf16x4_t*)(p));
      const bf16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
          (__attribute__((address_space(3))) bf16x4_t*)(p + 8 * Geo::ROW));
      const bf16x8_t vx = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      return __builtin_bit_cast(u32x4_t, vx);
    }
  }

  template <int I>
  __device__ __forceinline__ void product(const u32x4_t& fr, floatx16& y, const uint32_t* pin) {
    constexpr int n = index_of(I);
    if constexpr (is_score(I)) {
      if constexpr (n == 0) {
        floatx16 z;
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = 0.f;
        y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, fr), qf[0], z, 0,
                                                   0, 0);
      } else {
        y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, fr), qf[n], y, 0,
                                                   0, 0);
      }
    } else {
      constexpr int s = n / DT, dt = n % DT;
      const u32x4_t pv = {pin[4 * s], pin[4 * s + 1], pin[4 * s + 2], pin[4 * s + 3]};
      oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          __builtin_bit_cast(bf16x8_t, fr), __builtin_bit_cast(bf16x8_t, pv), oacc[dt], 0, 0, 0);
    }
  }

  // One subtile's softmax (scores x, weights pout) beside the other subtiles'
  // products: slot I's share of the weights 2^(x c - reference) and their sum.
  struct Soft {
    float ps[4];
    float prev;
  };
  template <int I, int N>
  __device__ __forceinline__ void soft_slot(Soft& f, const floatx16& x, uint32_t* pout) const {
    constexpr int lo = 16 * I / N, hi = 16 * (I + 1) / N;
    static_for<hi - lo>([&](auto q) {
      constexpr int e = lo + decltype(q)::value;
      const float p = exp2_fast(fmaf(x[e], c, SEL ? bias : -mref));
      if constexpr (e % 2 == 0) {
        f.prev = p;
      } else {
        pout[e / 2] = pack_bf16x2(f.prev, p);
        if constexpr (e / 2 < 4)
          f.ps[e / 2] = f.prev + p;
        else
          f.ps[e / 2 - 4] += f.prev + p;
        // Keeps the weights' work in this slot (the compiler would sink it past
        // the branch of soft_end, next to its use).
        asm volatile("" : "+v"(pout[e / 2]), "+v"(f.ps[(e / 2) % 4]));
      }
    });
  }
  // The first tile's scores (x0, x1) set the reference to the row's maximum over
  // its 64 keys, and x0's weights are formed. Taken over the first subtile alone,
  // the reference was below more rows' largest score, whose weight then is no
  // longer exactly 1 but rounded to bf16: the error against 64 bits of 64 keys at
  // D = 64 was 1.50e-3 instead of 1.33e-3, of 384 keys 1.62e-3 instead of 1.60e-3.
  __device__ __forceinline__ void start(const floatx16& x0, const floatx16& x1, uint32_t* pout) {
    mref = fmaxf(mref, seen(tile_max(x0, x1)));
    rebias();
    Soft f;
    soft_slot<0, 1>(f, x0, pout);
    lsum += (f.ps[0] + f.ps[1]) + (f.ps[2] + f.ps[3]);
  }
  // start() of a loop that carries a state from an earlier one.
  __device__ __forceinline__ void resume(const floatx16& x0, const floatx16& x1, uint32_t* pout) {
    const float old = mref;
    mref = fmaxf(mref, seen(tile_max(x0, x1)));
    rescale(exp2_fast(old - mref));
    start(x0, x1, pout);
  }
  // A tile that renews the reference: it moves to the maximum of the tile, down as
  // well as up, and the carried sum and value move with it. Down at most
  // kRenewDepth below the largest so far (`top`), so that they grow by 2^kRenewDepth
  // at most; weights further below round to nothing that matters.
  __device__ __forceinline__ void renew(float& top, const floatx16& x0, const floatx16& x1,
                                        uint32_t* pout) {
    const float old = mref;
    top = fmaxf(top, old);
    mref = fmaxf(top - kRenewDepth, tile_max(x0, x1));  // kNoRef - kRenewDepth is kNoRef
    rescale(exp2_fast(old - mref));
    start(x0, x1, pout);
  }
  // Largest score of a row in a 64-key tile, base-2 units.
  __device__ __forceinline__ float tile_max(const floatx16& x0, const floatx16& x1) const {
    float tmax = fmaxf(x0[0], x1[0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) tmax = fmaxf(tmax, fmaxf(x0[i], x1[i]));
    return max_with_other_half(tmax) * c;
  }
  // Moves the carried sum and value to another reference.
  __device__ __forceinline__ void rescale(float rs) {
    lsum *= rs;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int jj = 0; jj < 16; ++jj) oacc[i][jj] *= rs;
  }
  // A lane's weights are all at most 2^8 when their sum is, and then the
  // reference stays. Otherwise (a row's first visible keys past its first tile, or
  // a larger score) the reference moves up to the subtile's maximum, the carried
  // sum and value are rescaled and the weights formed again.
  __device__ __forceinline__ void soft_end(Soft& f, const floatx16& x, uint32_t* pout) {
    float sum = (f.ps[0] + f.ps[1]) + (f.ps[2] + f.ps[3]);
    if (__builtin_amdgcn_ballot_w64(!(sum <= kLazySum))) {
      float tmax = fmaxf(x[0], x[1]);
#pragma unroll
      for (int i = 2; i < 16; ++i) tmax = fmaxf(tmax, x[i]);
      const float cand = max_with_other_half(tmax) * c;
      const float old = mref;
      mref = fmaxf(mref, seen(cand));
      rebias();
      rescale(exp2_fast(old - mref));  // by 1 where the reference stayed
      soft_slot<0, 1>(f, x, pout);
      sum = (f.ps[0] + f.ps[1]) + (f.ps[2] + f.ps[3]);
    }
    lsum += sum;
  }

  // Subtile softmax of x into pout, the next subtile's scores into y (K subtile
  // at kt) and the values of the previous subtile (V subtile at vt, weights pin).
  // With CARRY_IN the first PF fragments are in carry, with CARRY_OUT the next
  // subtile's first PF are left there.
  template <bool CARRY_IN, bool CARRY_OUT>
  __device__ __forceinline__ void subtile(const floatx16& x, floatx16& y, const uint32_t* pin,
                                          uint32_t* pout, const char* kt, const char* vt,
                                          const char* kt2, const char* vt2, u32x4_t* carry) {
    u32x4_t fr[SLOTS];
    static_for<PF>([&](auto i) {
      constexpr int I = decltype(i)::value;
      if constexpr (CARRY_IN) fr[I] = carry[I];
      else fr[I] = fragment<I>(kt, vt);
    });
    __builtin_amdgcn_sched_barrier(0);
    Soft f;
    static_for<SLOTS>([&](auto i) {
      constexpr int I = decltype(i)::value;
      if constexpr (I + PF < SLOTS) {
        fr[I + PF] = fragment<I + PF>(kt, vt);
      } else if constexpr (CARRY_OUT) {
        carry[I + PF - SLOTS] = fragment<I + PF - SLOTS>(kt2, vt2);
      }
      product<I>(fr[I], y, pin);
      soft_slot<I, SLOTS>(f, x, pout);
      __builtin_amdgcn_sched_barrier(0);
    });
    soft_end(f, x, pout);
  }

  // The products of a subtile alone.
  __device__ __forceinline__ void products(floatx16& y, const uint32_t* pin, const char* kt,
                                           const char* vt) {
    u32x4_t fr[SLOTS];
    static_for<PF>([&](auto i) {
      constexpr int I = decltype(i)::value;
      fr[I] = fragment<I>(kt, vt);
    });
    __builtin_amdgcn_sched_barrier(0);
    static_for<SLOTS>([&](auto i) {
      constexpr int I = decltype(i)::value;
      if constexpr (I + PF < SLOTS) fr[I + PF] = fragment<I + PF>(kt, vt);
      product<I>(fr[I], y, pin);
      __builtin_amdgcn_sched_barrier(0);
    });
  }

  // Values of the last subtile.
  __device__ __forceinline__ void last_values(const uint32_t* pin, const char* vt) {
    static_for<SLOTS>([&](auto i) {
      constexpr int I = decltype(i)::value;
      if constexpr (!is_score(I)) {
        floatx16 unused;
        product<I>(fragment<I>(nullptr, vt), unused, pin);
      }
    });
  }
};

// One 64-key tile of the list: its first key, the end of its run, whether some
// key of it is hidden from some row of the workgroup, and whether it renews the
// reference.
struct TileAt {
  int base, end;
  bool masked, renews;
};

// Loads of 64-key tiles into the stages of the rolling loop. Wave w of the NW
// that share the stages loads the rows [64 w / NW, 64 (w + 1) / NW) of a tile, one
// 1 KiB block of whole rows per instruction; block i lies i KiB further both in
// memory and in LDS, so the instruction offset serves both and only the lane
// offsets of K, whose chunk permutation has a period of 16 rows, differ from block
// to block.
//
// The waves that share a V stage are NV, at least the NW that share a K stage: the
// two groups of a differential launch read the same values.
template <int D, int NW, int NV>
struct StageLoader {
  using G = TileGeom<D>;
  static constexpr int INSTS = 64 / G::RPI / NW;
  static constexpr int VINSTS = 64 / G::RPI / NV;
  static_assert(VINSTS >= 1, "whole blocks of V per wave");
  static constexpr int KPER = D == 128 ? 4 : 2;  // blocks of the K permutation's period
  static constexpr int NK = INSTS < KPER ? INSTS : KPER;
  __amdgpu_buffer_rsrc_t krs, vrs;
  unsigned koff[NK], voff;
  int row0, vrow0, slot;  // this lane's row in the wave's block 0 of K and V, its 16-byte slot
  int wbase, vwbase;      // byte offset of the wave's first block in a tile (scalar)

  // wave: index among the NW sharing a K stage; vwave: among the NV sharing a V stage.
  __device__ __forceinline__ void init(const uint16_t* kh, const uint16_t* vh, int wave,
                                       int vwave) {
    const int lane = threadIdx.x & 63;
    krs = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(kh), (short)0, -1, 0x00020000);
    vrs = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(vh), (short)0, -1, 0x00020000);
    wbase = wave * INSTS * 1024;
    vwbase = vwave * VINSTS * 1024;
    row0 = wave * INSTS * G::RPI + lane / G::KCH;
    vrow0 = vwave * VINSTS * G::RPI + lane / G::KCH;
    slot = lane % G::KCH;
#pragma unroll
    for (int i = 0; i < NK; ++i)
      koff[i] = row0 * G::ROW + (slot ^ G::swz_k(row0 + i * G::RPI)) * 16;
    voff = vrow0 * G::ROW + (slot ^ G::swz_v(vrow0)) * 16;
  }
  // Block I of a whole tile. AUX: cache policy of the load (2: non-temporal).
  template <bool ISK, int I, int AUX>
  __device__ __forceinline__ void block(char* l, unsigned soff) const {
    constexpr int hi = I / 4 * 4096;  // past the 12-bit instruction offset
    if constexpr (ISK)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          krs, (__attribute__((address_space(3))) void*)(l + hi), 16, (int)koff[I % NK],
          (int)(soff + hi), I % 4 * 1024, AUX);
    else
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          vrs, (__attribute__((address_space(3))) void*)(l + hi), 16, (int)voff,
          (int)(soff + hi), I % 4 * 1024, AUX);
  }
  template <bool ISK, int AUX = 0>
  __device__ __forceinline__ void load(char* stage, int kb, int kend) const {
    const int nrows = kend - kb;
    if (nrows <= 0) return;  // a tile past the last one
    constexpr int N = ISK ? INSTS : VINSTS;
    char* l = stage + (ISK ? wbase : vwbase);
    const unsigned soff = (unsigned)kb * G::ROW;
    if (nrows >= 64) {
      static_for<N>([&](auto q) { block<ISK, decltype(q)::value, AUX>(l, soff); });
    } else {
      // Ragged tile: rows past the run repeat its last row (masked later).
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int r = (ISK ? row0 : vrow0) + i * G::RPI;
        const int c = slot ^ (ISK ? G::swz_k(r) : G::swz_v(r));
        const int off = min(r, nrows - 1) * G::ROW + c * 16;
        auto* d = (__attribute__((address_space(3))) void*)(l + i * 1024);
        if constexpr (ISK)
          __builtin_amdgcn_raw_ptr_buffer_load_lds(krs, d, 16, off, (int)soff, 0, AUX);
        else
          __builtin_amdgcn_raw_ptr_buffer_load_lds(vrs, d, 16, off, (int)soff, 0, AUX);
      }
    }
  }
};

// Visibility of keys to this lane's row inside a tile (see mask_scores).
struct KeyMask {
  int lim, lo, sinks, h;
  __device__ __forceinline__ void operator()(floatx16& x, int kb, int kend) const {
    mask_scores(x, kb, kend, lim, lo, sinks, h);
  }
};

// The products and the softmax of one step of the rolling loop, tiles t0 = u, t1 =
// u + 1: the softmax of the second half of tile u (scores in xa) and of the first
// half of tile u + 1 (xb, if `second`), beside the scores of tile u + 1 (K stage
// `knext`) and the values of tile u (V stage `vcur`, weights of its first half in pb
// on entry). With RENEW a tile u + 1 may renew the reference: then its weights wait
// for both halves of its scores and all values of tile u. on0, on1: whether this
// lane's row sees the tiles at all (a loop that selects).
template <int D, bool RENEW, class Ro>
__device__ __forceinline__ void pair_compute(char* knext, char* vcur, Ro& ro, const TileAt& t0,
                                             TileAt& t1, bool second, float& top,
                                             const KeyMask& mask, floatx16& xa, floatx16& xb,
                                             uint32_t* pa, uint32_t* pb, bool on0 = true,
                                             bool on1 = true) {
  constexpr int SUB = TileGeom<D>::SUB;
  u32x4_t carry[Ro::PF];
  if (t0.masked) mask(xa, t0.base + 32, t0.end);
  if constexpr (Ro::SELECTS) ro.select(on0);
  ro.template subtile<false, true>(xa, xb, pb, pa, knext, vcur, knext + SUB, vcur + SUB, carry);
  const bool renews = RENEW && __builtin_expect(t1.renews, 0);
  if (second && !renews) {
    if (t1.masked) mask(xb, t1.base, t1.end);
    if constexpr (Ro::SELECTS) ro.select(on1);
    ro.template subtile<true, false>(xb, xa, pa, pb, knext + SUB, vcur + SUB, nullptr, nullptr,
                                     carry);
  }
  if (renews) {
    ro.products(xa, pa, knext + SUB, vcur + SUB);
    if (t1.masked) {
      mask(xb, t1.base, t1.end);
      mask(xa, t1.base + 32, t1.end);
      t1.masked = false;  // both halves are
    }
    ro.renew(top, xb, xa, pb);
  }
}

// One step of the rolling loop: pair_compute while K of tile t2 = u + 2 and V of tile
// u + 1 land in the two stages nobody reads during the step.
template <int D, int NW, int NV, bool RENEW>
__device__ __forceinline__ void pair_step(char* knext, char* kfree, char* vcur, char* vfree,
                                          Rolling<D>& ro, const StageLoader<D, NW, NV>& ld,
                                          const TileAt& t0, TileAt& t1, const TileAt& t2,
                                          bool second, float& top, const KeyMask& mask,
                                          floatx16& xa, floatx16& xb, uint32_t* pa,
                                          uint32_t* pb) {
  ld.template load<true>(kfree, t2.base, t2.end);
  ld.template load<false>(vfree, t1.base, t1.end);
  pair_compute<D, RENEW>(knext, vcur, ro, t0, t1, second, top, mask, xa, xb, pa, pb);
}

}  // namespace ef
