// Tiled rolling attention on bf16 MFMA (form M2 of figure
// "attention-rewrites", section 3; code-generation mapping of section 6.1:
// the query-row tile axis is the grid, the key-tile axis is the loop inside a
// workgroup, and the (max, sum, value) reducer state is loop-carried).
//
// A workgroup holds NW waves and 32*NW query rows of one kv head. Rows are
// packed as r = sq*G + g, so the Hq/Hkv query heads that read the same kv
// head share every K/V tile the workgroup stages (replication by index,
// section 3.1). Each wave owns 32 rows and works on transposed tiles:
//
//   S^T[key][query] = K_tile (A operand, from LDS) * Q^T (B operand, registers)
//   O^T[d][query]  += V^T_tile (A operand, from LDS) * P^T (B operand, registers)
//
// with v_mfma_f32_32x32x16_bf16. In both products lane l owns query l % 32,
// so the row max, the exponentials, the row sum and the rescale of the
// carried value are lane-local, and the score accumulator, converted to bf16,
// is already in the B-operand layout of the second product. Two lanes
// (l and l ^ 32) share a query and exchange one value per tile for the max.
//
// Two loops share this layout and the prologue and epilogue around it:
//
// The rolling loop (struct Rolling; prefill and every launch whose K/V tiles
// are shared or whose rows fill the matrix core) works on 32-key subtiles of
// 64-key tiles. While the vector ALU turns subtile j's scores into weights, the
// matrix core forms subtile j + 1's scores and multiplies subtile j - 1's
// values: three subtiles are in flight, so nothing the wave issues during a
// subtile waits for another kind of its work, and the source fixes the order of
// issue product by product (see struct Rolling). K is staged one tile ahead of
// V, two stages each, one workgroup barrier per 64 keys.
//
// The streaming loop (pipelined_step; the split producer of decode shapes)
// works on 32-key tiles of half the LDS, four workgroups to a compute unit,
// with non-temporal loads: it is bound by the K/V stream. Tile j's weights are
// formed while the matrix core computes tile j + 1's scores, then tile j's
// values are multiplied.
//
// Tiles go from HBM straight into LDS (direct loads, no staging registers),
// row-major with their 16-byte chunks permuted per row so that the fragment
// reads are free of bank conflicts. The V^T operand of the second product comes
// from transposing LDS reads (ds_read_b64_tr_b16) of the row-major V tile, in
// the key order of the P^T fragments.
//
// The exponent reference is only moved up when a weight against it may exceed
// 2^8 (base-2 units), so the carried sum and value are rescaled rarely; the
// final value / sum is unchanged (the repair h(c, s, s') = c * 2^(s - s') is
// exact for any reference point). A negative scale is moved into q (bf16
// negation is exact), so the scale c below is positive.
//
// In split mode the workgroup covers one key partition and stores the
// partition's (reference, sum, value) state instead of value / sum.
//
// Local attention (a causal sliding window of W keys plus S sink keys; the
// sliding-window GQA and attention-sink layers of section 7.3) visits only
// the tiles some row of the workgroup can see: the tiles of the sink run
// [0, S) and those from the window start of the workgroup's first row to its
// causal end. Both runs feed the same rolling reducer, so the sink and window
// keys share one softmax normalisation; the keys in between are never read.
//
// Differential attention (section 7.3), single pass: one launch, two groups of
// waves, one per branch. They meet in LDS, form y = A1 - lambda * A2, mix in
// lambda from the four learned vectors, RMS-normalise the row over D and write
// the result, so neither branch's output reaches HBM.
#include "diff_norm.hpp"
#include "ef_device.hpp"
#include "ef_kernels.hpp"
#include "rolling.hpp"

namespace ef {

namespace {

constexpr float kLazyThreshold = 8.f;  // base-2 headroom before the reference moves
// Key tiles of one workgroup, in visiting order: `na` tiles of the sink run
// starting at key a0 (keys below aend), then the tiles of the window run
// starting at b0 (keys below bend). Without a window the sink run is empty and
// the window run is the whole key range. Tiles past the last one cover no key.
template <int BN>
struct TileList {
  int a0, aend, na, b0, bend, n;
  int full_lo;  // a tile whose last key is at most this is below every row's causal limit
  int win_lo;   // a tile starting at or above this key lies in every row's window
  int sinks;    // keys below this are visible whatever the window
  __device__ __forceinline__ int base(int j) const {
    return j < na ? a0 + j * BN : b0 + (j - na) * BN;
  }
  __device__ __forceinline__ int end(int j) const { return j < na ? aend : bend; }
  // Whether some key of tile j is hidden from some row of the workgroup.
  __device__ __forceinline__ bool masked(int j) const {
    const int kb = base(j);
    return kb + BN > end(j) || kb + BN - 1 > full_lo || (kb < win_lo && kb + BN > sinks);
  }
};

// Loads of the streaming loop's 32-key tiles, straight from HBM to LDS (one
// 16-byte chunk per lane and load, each wave-wide load filling RPI whole rows).
// Rows past the tile's run repeat its last row (their keys are masked, their
// values finite); a tile past the last one loads nothing. Every key is read
// exactly once, so the loads are non-temporal and stream past the caches, which
// lifts the read rate by about a sixth (5.5 to 6.3-6.5 TB/s on the 537 MB of a
// 16 x 8192-key chunked decode).
template <int D, int NW>
struct Loader {
  using G = TileGeom<D>;
  static constexpr int INSTS = 32 / G::RPI / NW;  // direct loads per wave and tile
  static_assert(INSTS * G::RPI * NW == 32, "tile split over the waves");
  int row[INSTS];       // tile row whose chunk this lane loads
  int kchunk[INSTS];    // element offset of that chunk in a K row
  int vchunk[INSTS];    // element offset of that chunk in a V row
  unsigned koff[INSTS];  // byte offset of this lane's K chunk from the tile's first row
  unsigned voff[INSTS];  // the same for V
  int wave;              // wave index, uniform (scalar)

  __device__ __forceinline__ void init() {
    const int lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int i = 0; i < INSTS; ++i) {
      const int blk = wave + NW * i;
      row[i] = blk * G::RPI + lane / G::KCH;
      const int slot = lane % G::KCH;
      kchunk[i] = (slot ^ G::swz_k(row[i])) * 8;
      vchunk[i] = (slot ^ G::swz_v(row[i])) * 8;
      koff[i] = (unsigned)(row[i] * D + kchunk[i]) * 2u;
      voff[i] = (unsigned)(row[i] * D + vchunk[i]) * 2u;
    }
  }

  static __device__ __forceinline__ void load_chunk(const char* g, char* l) {
    __builtin_amdgcn_global_load_lds(g, (__attribute__((address_space(3))) void*)l, 16, 0,
                                     2 /* non-temporal */);
  }
  // The address is a uniform base (the tile's first row) plus a 32-bit lane
  // offset, so the vector ALU only clamps rows of a ragged tile.
  template <bool ISK>
  __device__ __forceinline__ void load(char* stage, const uint16_t* head, int kb, int kend) const {
    const int nrows = kend - kb;
    if (nrows <= 0) return;
    const char* base = reinterpret_cast<const char*>(head + (size_t)kb * D);
    if (nrows >= 32) {
#pragma unroll
      for (int i = 0; i < INSTS; ++i)
        load_chunk(base + (ISK ? koff[i] : voff[i]), stage + (wave + NW * i) * 1024);
    } else {
#pragma unroll
      for (int i = 0; i < INSTS; ++i) {
        const int r = min(row[i], nrows - 1);
        const unsigned off = (unsigned)(r * D + (ISK ? kchunk[i] : vchunk[i])) * 2u;
        load_chunk(base + off, stage + (wave + NW * i) * 1024);
      }
    }
  }
  template <int S>
  __device__ __forceinline__ void load_k(char* smem, const uint16_t* kh, int kb, int kend) const {
    load<true>(smem + G::template k_off<S>(), kh, kb, kend);
  }
  template <int S>
  __device__ __forceinline__ void load_v(char* smem, const uint16_t* vh, int kb, int kend) const {
    load<false>(smem + G::template v_off<S>(), vh, kb, kend);
  }
};

// S^T of the 32-key subtile at kt, every K fragment in registers of its own so
// that the reads run several products ahead.
template <int D>
__device__ __forceinline__ void subtile_scores(const char* kt, const int* kread,
                                               const bf16x8_t* qf, floatx16& sacc) {
  u32x4_t kx[D / 16];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) kx[s] = *reinterpret_cast<const u32x4_t*>(kt + kread[s]);
#pragma unroll
  for (int i = 0; i < 16; ++i) sacc[i] = 0.f;
#pragma unroll
  for (int s = 0; s < D / 16; ++s)
    sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kx[s]), qf[s],
                                                   sacc, 0, 0, 0);
}

// Softmax and value steps of the streaming loop's 32-key tiles.
template <int D>
struct Tile {
  using Geo = TileGeom<D>;
  static constexpr int DT = D / 32;  // 32-wide output tiles along D

  // Masks the scores and updates the rolling reference; returns -reference (0
  // while nothing is visible).
  static __device__ __forceinline__ float prepare(floatx16& x, floatx16* oacc, float& lsum,
                                                  float& mref, float c, int kb, int kend,
                                                  bool masked, int lim, int lo, int sinks,
                                                  int h) {
    if (masked) mask_scores(x, kb, kend, lim, lo, sinks, h);
    float tmax = fmaxf(x[0], x[1]);
#pragma unroll
    for (int i = 2; i < 16; ++i) tmax = fmaxf(tmax, x[i]);
    tmax = max_with_other_half(tmax);
    const float cand = tmax * c;  // tile maximum in base-2 units (c > 0)
    // Move the reference only when the tile exceeds it by the threshold.
    const bool up = cand > mref + kLazyThreshold;
    if (__builtin_amdgcn_ballot_w64(up)) {
      const float rs = up ? exp2_fast(mref - cand) : 1.f;  // 0 when mref = -inf
      mref = up ? cand : mref;
      lsum *= rs;
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int jj = 0; jj < 16; ++jj) oacc[i][jj] *= rs;
    }
    return (mref == kNegInf) ? 0.f : -mref;
  }

  // Weights 2^(x*c - reference) as bf16 pairs (P^T fragments) and their row
  // sum in fp32. (A packed bf16 dot product with (1, 1) per pair would sum the
  // rounded weights in half the instructions, but between matrix products it
  // costs about ten cycles each; the two sums differ by far less than the
  // rounding of the weights themselves.)
  static __device__ __forceinline__ void weights(const floatx16& x, float c, float mneg,
                                                 uint32_t* pk, float& lsum) {
    float ps[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float p0 = exp2_fast(fmaf(x[2 * i], c, mneg));
      const float p1 = exp2_fast(fmaf(x[2 * i + 1], c, mneg));
      pk[i] = pack_bf16x2(p0, p1);
      ps[i & 3] += p0 + p1;
    }
    lsum += (ps[0] + ps[1]) + (ps[2] + ps[3]);
  }

  // O^T += V^T * P^T over the two 16-key steps of the tile in V stage S; the
  // V^T operand (8 keys of one value column per lane) comes from two transposing
  // reads of 4 keys each out of the row-major V tile. The reads are issued from
  // assembly: the compiler cannot tell them from the direct-to-LDS loads into the other
  // stages still in flight, and waits for every outstanding load before the
  // first of them, which leaves the step's loads only its first half to land.
  // The reads of 16-key step s + 1 are requested before the products of step
  // s; LDS operations complete in order, so before step s's products a wait
  // until at most step s + 1's reads are outstanding suffices (other
  // operations counted by the same counter only make it longer). An empty
  // statement that rewrites the operands after the wait keeps the products
  // below it.
  template <int S>
  static __device__ __forceinline__ void values(const char* smem, const int* vread,
                                                    const uint32_t* pk, floatx16* oacc) {
    constexpr int STEPS = 2;
    constexpr int READS = 2 * DT;  // reads per 16-key step
    static_assert(READS <= 15, "outstanding reads exceed the LDS counter");
    const unsigned base = (unsigned)(uintptr_t)(
        (const __attribute__((address_space(3))) char*)(smem + Geo::template v_off<S>()));
    u32x2_t lo[2][DT], hi[2][DT];
    auto read_step = [&](int s, u32x2_t(&l)[DT], u32x2_t(&h)[DT]) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const unsigned addr = base + vread[dt] + 16 * s * Geo::ROW;
        asm volatile("ds_read_b64_tr_b16 %0, %1" : "=v"(l[dt]) : "v"(addr));
        asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2"
                     : "=v"(h[dt])
                     : "v"(addr), "i"(8 * Geo::ROW));
      }
    };
    read_step(0, lo[0], hi[0]);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int b = s & 1;
      if (s + 1 < STEPS) {
        read_step(s + 1, lo[b ^ 1], hi[b ^ 1]);
        asm volatile("s_waitcnt lgkmcnt(%0)" ::"i"(READS) : "memory");
      } else {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) asm volatile("" : "+v"(lo[b][dt]), "+v"(hi[b][dt]));
      // P^T fragment: registers 8*(s%2) .. +8 of score half s/2, i.e. pk[4*s .. 4*s+3].
      const u32x4_t pv = {pk[4 * s], pk[4 * s + 1], pk[4 * s + 2], pk[4 * s + 3]};
      const bf16x8_t pf = __builtin_bit_cast(bf16x8_t, pv);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const u32x4_t vx = {lo[b][dt][0], lo[b][dt][1], hi[b][dt][0], hi[b][dt][1]};
        oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, vx), pf,
                                                          oacc[dt], 0, 0, 0);
      }
    }
  }
};

// One step of the streaming loop on tile j (stage parity S = j % 2). On entry
// sacc[S] holds S^T of tile j, K stage 1-S holds tile j+1 and V stage S holds
// tile j. The step requests K of tile j+2 (into K stage S, last read for tile j's
// scores) and V of tile j+1 (into V stage 1-S, last read for tile j-1's values)
// straight into LDS, computes tile j's weights while the matrix core computes
// tile j+1's scores, multiplies tile j's values, and waits for its loads before
// the workgroup barrier.
template <int D, int NW, int S>
__device__ __forceinline__ void pipelined_step(char* smem, const Loader<D, NW>& ld,
                                               const uint16_t* kh, const uint16_t* vh,
                                               const TileList<32>& tl, int j, int lim, int lo,
                                               int h, const int* kread, const int* vread,
                                               const bf16x8_t* qf, floatx16* sacc, floatx16* oacc,
                                               float& lsum, float& mref, float c) {
  using TileT = Tile<D>;
  ld.template load_k<S>(smem, kh, tl.base(j + 2), tl.end(j + 2));  // nothing past the last tile
  ld.template load_v<1 - S>(smem, vh, tl.base(j + 1), tl.end(j + 1));
  const float mneg = TileT::prepare(sacc[S], oacc, lsum, mref, c, tl.base(j), tl.end(j),
                                    tl.masked(j), lim, lo, tl.sinks, h);
  uint32_t pk[8];
  TileT::weights(sacc[S], c, mneg, pk, lsum);
  // Tile j+1's scores go to the other accumulator, so tile j's stay in place.
  subtile_scores<D>(smem + TileGeom<D>::template k_off<1 - S>(), kread, qf, sacc[1 - S]);
  TileT::template values<S>(smem, vread, pk, oacc);
  // The wait stays behind the products: the scheduler moves it up into them, where
  // the loads have had two thirds of the step to land (8 rows per kv head, 8 x
  // 16384 keys of 64: 65.7 -> 61.3 us; 16 x 12 heads, 8 of 2000 keys of 128: 43.9 ->
  // 41.6 us).
  __builtin_amdgcn_sched_barrier(0);
  wait_tile_loads();
  __syncthreads();
}

// The tiles [first, first + n) of the list that one group of waves walks.
struct GroupTiles {
  const TileList<64>& tl;
  int first, n;
  __device__ __forceinline__ TileAt at(int t, bool renews) const {
    if (t >= n) return {0, 0, false, false};  // nothing to load
    return {tl.base(first + t), tl.end(first + t), tl.masked(first + t), renews};
  }
  // 32-key subtiles; the list's last tile may end within its first half.
  __device__ __forceinline__ int subtiles() const {
    if (n <= 0) return 0;
    return 2 * n - (tl.base(first + n - 1) + 32 >= tl.end(first + n - 1) ? 1 : 0);
  }
};

// Forms of the kernel.
enum Form {
  kStream,    // streaming loop (split producer of decode shapes)
  kRolling,   // rolling loop
  kKeySplit,  // rolling loop, two groups of waves over the two halves of the key tiles
  kDiffPair,  // rolling loop, two groups of waves over the two branches of a
              // differential layer
  kDiffRenew,  // kDiffPair whose rows renew their reference every a.renew tiles
};

// NW waves (of 32 query rows each) per group; the two-group forms hold two
// groups over the same rows, with stages of their own, that meet in LDS at the
// end.
//
// kKeySplit serves grids that leave the chip's SIMDs without a second wave: one
// wave alone reaches 88% of the rate of two on a SIMD, so what such a launch
// waits for is the chain of a workgroup's tiles, and two groups halve it. 8 heads
// of 64, 2048 causal: 28.3 -> 17.7 us; 32/8 heads of 128, 4 x 100 of 1500 keys:
// 30.2 -> 22.5 us (the rule that selects it holds both sides' figures).
//
// kDiffPair runs both branches of a differential layer in one launch: the
// second branch's output stays in registers and LDS instead of going through o
// between two launches, and each V tile is staged once for both. 32/8 heads of
// 128, 1024 causal: 52.5 -> 37.0 us, 4 x 1024: 118.5 -> 105.8 us; 32 heads, 1024 of
// 32768 keys: 1003 us in two split branches, 999 in one launch, 968 with the
// shared V stages. Grids of thousands of row tiles of grouped heads of 64 lose up
// to 3% against a launch per branch, whose four-wave workgroups run three waves to
// a SIMD: 15 x 32/8 heads, 1321 of 2227 keys 715 us before, 734 now, 11 x 64/8, 762
// of 886 245 and 252 (ungrouped heads gain there too: 4 x 32, 1024 87 and 82).
//
// kDiffRenew is kDiffPair where the launch takes the place of a split call: every
// a.renew key tiles, the tiles of one of the split's partitions, a row's reference
// starts again at the maximum of a 64-key tile, as each partition's would, so the
// weights are rounded to bf16 as the split rounds them. The renewal stands behind
// the step in a block of its own: as an else of the step's second half it cost 87
// spilled registers, inside the second half 4% on every step. It costs a step of
// its own, 1-1.5 us: 32 heads, 1024 of 32768 keys, every 256 tiles 986 us without,
// 992 with it; 32/8 heads of 64, 768 of 3000 keys, every 32 tiles 55.7, 57.9; 12
// heads of 64, 128 of 640 keys, every tile 17.6, 22.2.
//
// Occupancy target: two waves per SIMD (two workgroups of four waves per CU, four
// of the streaming loop's two-wave ones, overlap each other's barrier and
// latency stalls; a workgroup of eight waves has both on its own), three at D = 64
// where the registers allow; the four-wave two-group form and the two-wave
// workgroup of the rolling loop serve grids too small for that.
template <int D, int NW, Form F>
__global__ __launch_bounds__(NW * 64 * (F >= kKeySplit ? 2 : 1))
__attribute__((amdgpu_waves_per_eu(NW == 2 && F != kStream         ? 1
                                   : D == 64 && F < kKeySplit ? 3
                                                              : 2)))
void attn_mfma_kernel(MfmaParams a) {
  using Geo = TileGeom<D>;
  constexpr bool STREAM = F == kStream;
  constexpr bool DIFF = F >= kDiffPair, RENEW = F == kDiffRenew;
  constexpr int GROUPS = F >= kKeySplit ? 2 : 1;
  constexpr int KSTEPS = D / 16;
  constexpr int DT = D / 32;
  constexpr int BM = 32 * NW;
  constexpr int BN = STREAM ? 32 : 64;  // keys per tile

  const int lane = threadIdx.x & 63;
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int grp = GROUPS > 1 ? wid / NW : 0;  // group of this wave
  const int wave = wid - grp * NW;            // wave inside the group
  const int h = lane >> 5;   // k-group of the MFMA operands
  const int ql = lane & 31;  // this lane's query inside the wave's 32 rows

  // Workgroup -> (row tile, partition, b*Hkv). Workgroups are dispatched to the
  // chip's 8 XCDs round-robin by linear id; the id is remapped so that each XCD
  // receives a contiguous run of kv heads, and all row tiles of a head, which
  // read the same K/V, share one XCD's L2. Row tiles are visited last-first so
  // causal tiles with the most keys start first: head by head, or (a.interleave)
  // over all heads of the XCD, which leaves only short tiles for the end.
  const unsigned nwg = gridDim.x * gridDim.y * gridDim.z;
  unsigned lin = blockIdx.x + gridDim.x * (blockIdx.y + gridDim.y * blockIdx.z);
  if (nwg % kXcds == 0) lin = (lin % kXcds) * (nwg / kXcds) + lin / kXcds;
  int mt = a.mtiles - 1 - (int)(lin % gridDim.x);
  const int p = (int)((lin / gridDim.x) % gridDim.y);
  int bh = (int)(lin / (gridDim.x * gridDim.y));
  if (a.interleave) {
    const unsigned heads = gridDim.z / kXcds, wgs = nwg / kXcds;  // of one XCD
    mt = a.mtiles - 1 - (int)(lin % wgs / heads);
    bh = (int)(lin / wgs * heads + lin % wgs % heads);
  }
  const int b = bh / a.Hkv, hkv = bh % a.Hkv;

  const size_t kvhead = ((size_t)b * a.Hkv + hkv) * (size_t)a.Skv * D;
  const uint16_t* kh = (DIFF && grp ? a.k2 : a.k) + kvhead;
  const uint16_t* vh = a.v + kvhead;

  // This lane's query row.
  const int r = mt * BM + wave * 32 + ql;
  const bool rvalid = r < a.R;
  const int sq = rvalid ? r / a.G : 0;
  const int g = rvalid ? r % a.G : 0;
  const size_t orow = (((size_t)b * a.Hq + (size_t)hkv * a.G + g) * a.Sq + sq);
  const int off = a.Skv - a.Sq;
  const int lim = !rvalid ? -1 : (a.causal ? sq + off : 0x7fffffff);
  const int W = a.runs.window;
  const int lo = W > 0 ? lim - W : INT_MIN;  // keys at or left of lo are outside the window

  // Key tiles of this workgroup. The partition is a range [v0, v1) of the
  // virtual key axis (the sink run [0, la) followed by the window run from key
  // bs); its part in each run is cut at the last key any row can see and, in
  // the window run, at the first key of the earliest row's window.
  TileList<BN> tl;
  {
    const int la = a.runs.la, bs = a.runs.bs;
    const int v0 = p * a.T;
    const int v1 = min(v0 + a.T, a.runs.lv);
    int cend = 0x7fffffff, wbeg = 0;
    tl.full_lo = 0x7fffffff;
    tl.win_lo = INT_MIN;
    if (a.causal) {
      const int r_lo = mt * BM;
      const int r_hi = min(mt * BM + BM, a.R) - 1;
      tl.full_lo = r_lo / a.G + off;
      cend = r_hi / a.G + off + 1;
      if (W > 0) {
        wbeg = max(0, tl.full_lo - W + 1) / BN * BN;
        tl.win_lo = r_hi / a.G + off - W + 1;
      }
    }
    tl.a0 = v0;
    tl.aend = min(min(v1, la), cend);
    tl.na = tl.aend > tl.a0 ? (tl.aend - tl.a0 + BN - 1) / BN : 0;
    tl.b0 = max(bs + max(v0, la) - la, wbeg);
    tl.bend = min(bs + v1 - la, cend);
    tl.n = tl.na + (tl.bend > tl.b0 ? (tl.bend - tl.b0 + BN - 1) / BN : 0);
    tl.sinks = W > 0 ? a.runs.sinks : 0;
  }
  const int ntiles = tl.n;

  // Q^T fragments (B operand): lane holds q[row][16*s + 8*h .. +8].
  bf16x8_t qf[KSTEPS];
  {
    const u32x4_t* qp =
        reinterpret_cast<const u32x4_t*>((DIFF && grp ? a.q2 : a.q) + orow * D);
    const u32x4_t zero = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int s = 0; s < KSTEPS; ++s) {
      const u32x4_t x = (rvalid ? qp[2 * s + h] : zero) ^ a.qflip;
      qf[s] = __builtin_bit_cast(bf16x8_t, x);
    }
  }

  floatx16 oacc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) oacc[i][j] = 0.f;
  float mref = STREAM ? kNegInf : kNoRef;  // reference maximum, base-2 units
  float lsum = 0.f;      // this lane's half of the row sum
  // The floor keeps a zero scale well defined: every visible key gets weight 1
  // (2^(x c) rounds to 1 for any finite score), while a hidden key's -inf stays
  // -inf instead of becoming -inf * 0 = NaN.
  const float c = fmaxf(a.c_abs, 1e-30f);
  // Per-lane LDS byte offsets of the fragment reads inside a stage: K row ql,
  // chunk 2s + h of k-step s; and, per 32-column tile dt of V^T, the
  // transposing-read pointer of this lane (row 4(lane/32) + (lane%16)/4 of a
  // 16-key step, 8 bytes at column 32 dt + 16 ((lane/16)%2) + 4 (lane%4)).
  int kread[KSTEPS];
#pragma unroll
  for (int s = 0; s < KSTEPS; ++s) kread[s] = ql * Geo::ROW + ((2 * s + h) ^ Geo::swz_k(ql)) * 16;
  int vread[DT];
  {
    const int j16 = lane & 15, grp = lane >> 4;
    const int vr = 4 * (grp >> 1) + (j16 >> 2);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const int d_off = 32 * dt + 16 * (grp & 1) + 4 * (j16 & 3);
      vread[dt] = vr * Geo::ROW + (((d_off >> 3) ^ Geo::swz_v(vr)) * 16) + 2 * (d_off & 7);
    }
  }

  if constexpr (STREAM) {
    // Prologue: K and V of tile 0 into stage 0, K of tile 1 into K stage 1, then
    // tile 0's scores; the second barrier orders those K reads before stage 0 is
    // rewritten by the first step.
    __shared__ __align__(1024) char smem[4 * Geo::SUB];
    Loader<D, NW> ld;
    ld.init();
    floatx16 sacc[2];  // S^T of the current and the next tile
    if (ntiles > 0) {
      ld.template load_k<0>(smem, kh, tl.base(0), tl.end(0));
      ld.template load_v<0>(smem, vh, tl.base(0), tl.end(0));
      ld.template load_k<1>(smem, kh, tl.base(1), tl.end(1));
    }
    wait_tile_loads();
    __syncthreads();
    if (ntiles > 0) subtile_scores<D>(smem + Geo::template k_off<0>(), kread, qf, sacc[0]);
    __syncthreads();
    for (int j = 0; j < ntiles; j += 2) {
      pipelined_step<D, NW, 0>(smem, ld, kh, vh, tl, j, lim, lo, h, kread, vread, qf, sacc, oacc,
                               lsum, mref, c);
      if (j + 1 < ntiles)
        pipelined_step<D, NW, 1>(smem, ld, kh, vh, tl, j + 1, lim, lo, h, kread, vread, qf, sacc,
                                 oacc, lsum, mref, c);
    }
  }

  // Output rows: value / sum, or the state of the partition, of the value tiles
  // [DT0, DT0 + NDT) (32 channels each; lane halves hold alternate 4-channel runs).
  auto store = [&](const floatx16* val, int dt0, auto ndt, float ref, float ltot) {
    constexpr int NDT = decltype(ndt)::value;
    if (!rvalid) return;
    auto put = [&](float* dst, float mul) {
#pragma unroll
      for (int i = 0; i < NDT; ++i)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          *reinterpret_cast<float4*>(dst + (dt0 + i) * 32 + 8 * q4 + 4 * h) =
              make_float4(val[i][4 * q4] * mul, val[i][4 * q4 + 1] * mul, val[i][4 * q4 + 2] * mul,
                          val[i][4 * q4 + 3] * mul);
    };
    if (a.ws_m == nullptr) {
      put(a.o + orow * D, ltot > 0.f ? 1.f / ltot : 0.f);
    } else {
      const size_t slot = orow * (size_t)a.P + p;
      if (h == 0) {
        // Reference in natural-log units, in terms of scale * q.k.
        a.ws_m[slot] = ref == kNegInf || ref == kNoRef ? kNegInf : ref * kLn2;
        a.ws_l[slot] = ltot;
      }
      put(a.ws_acc + slot * D, 1.f);
    }
  };

  if constexpr (STREAM) {
    store(oacc, 0, std::integral_constant<int, DT>{}, mref, lsum + __shfl_xor(lsum, 32, 64));
    return;
  } else {
    // The four stages are objects of their own, and the loads go through buffer
    // descriptors: the compiler then neither waits for a step's loads before its
    // first reads (they cannot alias) nor drains the LDS counter at every read
    // (it does with a flat direct-to-LDS load in flight).
    constexpr int STAGE = 2 * Geo::SUB;  // one group's bytes of a stage
    // The two branches of a differential launch share the V stages.
    constexpr int VGROUPS = DIFF ? 1 : GROUPS, NV = NW * GROUPS / VGROUPS;
    __shared__ __align__(1024) char sk0[GROUPS * STAGE], sk1[GROUPS * STAGE];
    __shared__ __align__(1024) char sv0[VGROUPS * STAGE], sv1[VGROUPS * STAGE];
    char* const k0 = sk0 + grp * STAGE;
    char* const k1 = sk1 + grp * STAGE;
    char* const v0 = sv0 + (VGROUPS > 1 ? grp * STAGE : 0);
    char* const v1 = sv1 + (VGROUPS > 1 ? grp * STAGE : 0);
    // Tiles of this group, and the steps the workgroup's barriers count: those of
    // the first half of the tiles, which is never the shorter one.
    const int first_half = (ntiles + 1) / 2;
    const GroupTiles gt{tl, F == kKeySplit && grp ? first_half : 0,
                        F != kKeySplit ? ntiles : grp ? ntiles - first_half : first_half};
    const int nsub = gt.subtiles();
    const int steps =
        F == kKeySplit ? GroupTiles{tl, 0, first_half}.subtiles() / 2 : nsub / 2;
    floatx16 xa, xb;        // scores of odd and even subtiles
    uint32_t pa[8], pb[8];  // their weights
    Rolling<D> ro{kread, vread, qf, oacc, lsum, mref, c};
    const KeyMask mask{lim, lo, tl.sinks, h};
    if (ntiles > 0) {
      StageLoader<D, NW, NV> ld;
      ld.init(kh, vh, wave, DIFF ? wid : wave);
      int due = RENEW ? a.renew : 0;  // tiles until the next one that renews
      float top = kNoRef;
      auto tile = [&](int t) {  // t = 1, 2, 3, ...
        const bool renews = RENEW && --due == 0;
        if (renews) due = a.renew;
        return gt.at(t, renews);
      };
      TileAt t0 = gt.at(0, false), t1 = tile(1), t2;
      // Prologue: tile 0's K and V and tile 1's K; tile 0's scores, then subtile 0's
      // softmax. The second barrier orders those K reads before stage 0 is rewritten
      // by the first step.
      ld.template load<true>(k0, t0.base, t0.end);
      ld.template load<false>(v0, t0.base, t0.end);
      ld.template load<true>(k1, t1.base, t1.end);
      wait_tile_loads();
      __syncthreads();
      if (GROUPS == 1 || nsub > 0) {
        tile_scores<D>(k0, kread, qf, xb, xa);
        if (t0.masked) {
          mask_scores(xb, t0.base, t0.end, lim, lo, tl.sinks, h);
          mask_scores(xa, t0.base + 32, t0.end, lim, lo, tl.sinks, h);
          t0.masked = false;  // both halves are
        }
        ro.start(xb, xa, pb);
      }
      __syncthreads();
      for (int u = 0; u < steps; u += 2) {
        t2 = tile(u + 2);
        if (GROUPS == 1 || 2 * u + 1 < nsub)
          pair_step<D, NW, NV, RENEW>(k1, k0, v0, v1, ro, ld, t0, t1, t2, 2 * u + 2 < nsub, top,
                                      mask, xa, xb, pa, pb);
        wait_tile_loads();
        __syncthreads();
        if (u + 1 >= steps) break;
        t0 = tile(u + 3);
        if (GROUPS == 1 || 2 * u + 3 < nsub)
          pair_step<D, NW, NV, RENEW>(k0, k1, v1, v0, ro, ld, t1, t2, t0, 2 * u + 4 < nsub, top,
                                      mask, xa, xb, pa, pb);
        wait_tile_loads();
        __syncthreads();
        t1 = t0;
        t0 = t2;
      }
      if (GROUPS == 1 || nsub > 0) {
        const int last = nsub - 1;
        const char* vl = (last >> 1 & 1) ? v1 : v0;
        if (last & 1)
          ro.last_values(pa, vl + Geo::SUB);
        else
          ro.last_values(pb, vl);
      }
    }
    const float ltot = lsum + __shfl_xor(lsum, 32, 64);  // both lane halves of the row
    if constexpr (GROUPS == 1) {
      store(oacc, 0, std::integral_constant<int, DT>{}, mref, ltot);
    } else {
      // The groups meet: each sends the other half of its value tiles (and its
      // reference and sum), and finishes its own half of the channels.
      constexpr int HT = DT / 2;
      const float inv = ltot > 0.f ? 1.f / ltot : 0.f;
      float4* out = reinterpret_cast<float4*>(grp ? sk1 : sk0) + wave * (HT * 4 * 64) + lane;
      const float4* in =
          reinterpret_cast<const float4*>(grp ? sk0 : sk1) + wave * (HT * 4 * 64) + lane;
      float2* ml = reinterpret_cast<float2*>(sv0);  // [group][wave][lane]
      float* sq2 = reinterpret_cast<float*>(sv1);   // [group][wave][lane]
      floatx16 own[HT];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < HT; ++i) {
#pragma unroll
        for (int e = 0; e < 16; ++e) own[i][e] = grp ? oacc[HT + i][e] : oacc[i][e];
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[e] = grp ? oacc[i][4 * q4 + e] : oacc[HT + i][4 * q4 + e];
            if constexpr (DIFF) x[e] *= inv;
          }
          out[(i * 4 + q4) * 64] = make_float4(x[0], x[1], x[2], x[3]);
        }
      }
      ml[(grp * NW + wave) * 64 + lane] = make_float2(mref, ltot);
      __syncthreads();
      if constexpr (F == kKeySplit) {
        const float2 other = ml[((1 - grp) * NW + wave) * 64 + lane];
        const float ref = fmaxf(mref, other.x);
        const float wo = exp2_fast(mref - ref), wi = exp2_fast(other.x - ref);
        const float lt = fmaf(other.y, wi, ltot * wo);
#pragma unroll
        for (int i = 0; i < HT; ++i)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const float4 x = in[(i * 4 + q4) * 64];
            own[i][4 * q4] = fmaf(x.x, wi, own[i][4 * q4] * wo);
            own[i][4 * q4 + 1] = fmaf(x.y, wi, own[i][4 * q4 + 1] * wo);
            own[i][4 * q4 + 2] = fmaf(x.z, wi, own[i][4 * q4 + 2] * wo);
            own[i][4 * q4 + 3] = fmaf(x.w, wi, own[i][4 * q4 + 3] * wo);
          }
        store(own, grp * HT, std::integral_constant<int, HT>{}, ref, lt);
      } else {
        // y = A1 - lambda A2 (the first group holds the first branch), then the
        // RMS normalisation of the row over all channels.
        const float lam = diff_lambda(a.diff, lane, D);
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < HT; ++i)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const float4 x4 = in[(i * 4 + q4) * 64];
            const float x[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float mine = own[i][4 * q4 + e] * inv;
              const float y = fmaf(-lam, grp ? mine : x[e], grp ? x[e] : mine);
              own[i][4 * q4 + e] = y;
              ss = fmaf(y, y, ss);
            }
          }
        ss += __shfl_xor(ss, 32, 64);
        sq2[(grp * NW + wave) * 64 + lane] = ss;
        __syncthreads();
        ss += sq2[((1 - grp) * NW + wave) * 64 + lane];
        const float rn = diff_row_factor(a.diff, ss, D);
        if (!rvalid) return;
        float* orp = a.o + orow * D;
#pragma unroll
        for (int i = 0; i < HT; ++i)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const int d = (grp * HT + i) * 32 + 8 * q4 + 4 * h;
            const float4 gw = *reinterpret_cast<const float4*>(a.diff.gamma + d);
            *reinterpret_cast<float4*>(orp + d) =
                make_float4(rn * gw.x * own[i][4 * q4], rn * gw.y * own[i][4 * q4 + 1],
                            rn * gw.z * own[i][4 * q4 + 2], rn * gw.w * own[i][4 * q4 + 3]);
          }
      }
    }
  }
}

template <int D, int NW, Form F>
hipError_t launch_one(const MfmaParams& a, hipStream_t stream) {
  hipLaunchKernelGGL((attn_mfma_kernel<D, NW, F>), dim3(a.mtiles, a.P, a.B * a.Hkv),
                     dim3(NW * 64 * (F >= kKeySplit ? 2 : 1)), 0, stream, a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_d(const MfmaParams& a, hipStream_t stream) {
  if (a.diff.gamma != nullptr) {
    if (a.renew > 0)
      return a.bm == 64 ? launch_one<D, 2, kDiffRenew>(a, stream)
                        : launch_one<D, 4, kDiffRenew>(a, stream);
    return a.bm == 64 ? launch_one<D, 2, kDiffPair>(a, stream)
                      : launch_one<D, 4, kDiffPair>(a, stream);
  }
  if (a.key_split) return launch_one<D, 2, kKeySplit>(a, stream);
  if (a.bm == 128) return launch_one<D, 4, kRolling>(a, stream);
  // The split producer with one 64-row tile per kv head (decode shapes) streams:
  // its loads assume that every key is read once.
  if (a.mtiles == 1 && a.ws_m != nullptr) return launch_one<D, 2, kStream>(a, stream);
  return launch_one<D, 2, kRolling>(a, stream);
}

}  // namespace

hipError_t launch_mfma_attention(const MfmaParams& a, hipStream_t stream) {
  if (a.bm != 64 && a.bm != 128) return hipErrorInvalidValue;
  return a.D == 128 ? launch_d<128>(a, stream) : launch_d<64>(a, stream);
}

}  // namespace ef
