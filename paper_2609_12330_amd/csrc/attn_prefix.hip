// Attention of a batch of sequences over one shared prefix and their own keys.
//
// Sequence b's keys are Lp prefix keys, the same for all, followed by len_b own
// ones; softmax and values run over both. A softmax state (reference, sum, value)
// over the union of two key sets is the sum of their states at one reference, so
// the prefix is treated apart: the rows of all sequences that share a kv head are
// packed into the matrix core's row tiles and read each prefix key once per 128
// rows, instead of once per sequence. The other workgroups of the launch hold one
// sequence's rows over its own keys, which only it reads. Prefix workgroups are
// bound by the matrix core and the others by HBM; they share the compute units, one
// of each where there are enough of both. A combine then joins each row's states.
//
// Where the sequences' rows fill their tiles and the chip by themselves (`whole`), a
// workgroup walks the prefix and then the own keys of its sequence in one loop and
// writes the finished rows.
//
// What bounds it: with one token each, 64 sequences of 32/8 heads of 128, 32768 prefix
// keys and 64 to 2048 own ones (412 MB, 35 GFLOP) 97 us, 4.3 TB/s, and 5 the combine: two workgroups fit on
// a compute unit (LDS, registers), 64 KiB of loads in flight between them, and a step
// takes as long as its loads, 2.1 to 2.6 us; the prefix alone takes 52 us, the own keys
// alone 63 (long ones of equal length run at 6.2 TB/s). Prompts of 384 tokens of 16
// sequences behind 8192 keys (844 GFLOP) 740-766 us, 1.10 to 1.14 PFLOP/s: the power limit,
// as for plain prefills. A few to about 100 tokens, whose rows do not fill their tiles or
// whose tiles do not fill the chip twice, run at 0.6 to 0.7 (see long_api.hip). Tried and not kept: 256 rows to a workgroup of eight waves, which
// leaves one on a compute unit (99 -> 122 us); the own keys of up to four rows on the
// vector ALU (98); the combine in the same launch (4 sequences over 2011 keys 13.6 ->
// 14.7).
#include "roll_tiles.hpp"
#include "wave_ops.hpp"

namespace ef {

namespace {

// Key tiles of a sequence in one count: the prefix's, then its own, whose keys are
// numbered from Lp on.
template <int D, int NW>
struct TwoRuns {
  StageLoader<D, NW, NW> ld;
  const uint16_t *kp, *vp, *ko, *vo;  // prefix and own keys of the head
  int first;                          // first tile of the walk
  int np, Lp, end;                    // prefix tiles and keys, all keys
  int full_lo;                        // keys up to it are visible to all rows of the wave
  bool once;                          // no other workgroup reads the keys of the walk

  __device__ __forceinline__ TileAt at(int t) const {
    t += first;
    const bool own = t >= np;
    const int base = own ? Lp + (t - np) * 64 : t * 64;
    const int stop = own ? end : min(end, Lp);
    return {base, stop, base + 64 > stop || base + 63 > full_lo, false};
  }
  __device__ __forceinline__ bool on(int) const { return true; }
  template <bool ISK>
  __device__ __forceinline__ void load(char* stage, const TileAt& t) const {
    const bool own = t.base >= Lp;
    const uint16_t* p = ISK ? (own ? ko : kp) : (own ? vo : vp);
    const int off = own ? Lp : 0;
    StageLoader<D, NW, NW> l = ld;
    auto& rs = ISK ? l.krs : l.vrs;
    rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(p), (short)0, -1, 0x00020000);
    if (once)
      l.template load<ISK, 2>(stage, t.base - off, t.end - off);
    else
      l.template load<ISK>(stage, t.base - off, t.end - off);
  }
};

template <int D, int NW>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2)))
void attn_prefix_kernel(PrefixParams a) {
  using Geo = TileGeom<D>;
  constexpr int BM = 32 * NW;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, ql = lane & 31;

  // Workgroup -> work. Ids go round the XCDs; each takes a contiguous run of either
  // kind, row tiles innermost, so that the row tiles that read the same keys share
  // its L2.
  unsigned id = blockIdx.x;
  const bool packed = id < a.n_prefix;
  const unsigned n = packed ? a.n_prefix : a.n_own;
  if (!packed) id -= a.n_prefix;
  if (n % kXcds == 0) id = (id % kXcds) * (n / kXcds) + id / kXcds;
  const unsigned mts = packed ? a.mt1 : a.mt2, parts = packed ? a.P1 : a.P2;
  const int mt = (int)(id % mts), p = (int)(id / mts % parts);
  const int group = (int)(id / mts / parts);  // kv head, or sequence and kv head
  const int hkv = packed ? group : group % a.Hkv;

  // This lane's row.
  const int rows = packed ? a.B * a.R : a.R;
  const int r = mt * BM + wave * 32 + ql;
  const bool valid = r < rows;
  const int bu = packed ? 0 : group / a.Hkv;  // uniform: the sequence of an unpacked workgroup
  const int b = packed ? (valid ? r / a.R : 0) : bu;
  const int rr = valid ? (packed ? r % a.R : r) : 0;
  const int sq = rr / a.G, g = rr % a.G;
  const size_t orow = ((size_t)b * a.Hq + (size_t)hkv * a.G + g) * a.Sq + sq;
  // Tiles of 64 keys of the walk.
  TwoRuns<D, NW> tl;
  tl.Lp = a.Lp;
  tl.np = (a.Lp + 63) / 64;
  tl.kp = a.kp + (size_t)hkv * a.Lp * D;
  tl.vp = a.vp + (size_t)hkv * a.Lp * D;
  const size_t own = ((size_t)bu * a.Hkv + hkv) * (size_t)a.Skv * D;
  tl.ko = packed ? tl.kp : a.k + own;
  tl.vo = packed ? tl.vp : a.v + own;
  tl.full_lo = 0;  // until the rows' lengths are there (see `masks`)
  tl.once = packed ? a.mt1 == 1 : a.mt2 == 1 && !a.whole;
  int last;
  if (packed) {
    tl.end = a.Lp;
    tl.first = p * a.T1;
    last = min(tl.first + a.T1, tl.np);
  } else {
    const int all = a.Lp + sequence_length(a.lengths, bu, a.Skv);  // (checked on the host)
    // Keys behind the last row's are not visited.
    const int top = min(mt * BM + BM, rows) - 1;
    const int seen = a.causal ? min(all, top / a.G + all - a.Sq + 1) : all;
    tl.end = max(seen, 0);
    const int tiles = tl.end <= a.Lp ? (tl.end + 63) / 64 : tl.np + (tl.end - a.Lp + 63) / 64;
    tl.first = a.whole ? 0 : tl.np + p * a.T2;
    last = a.whole ? tiles : min(tl.first + a.T2, tiles);
  }

  Rows<D> row;
  row.init(a.q + orow * D, valid, a.qflip, h);
  FragmentReads<D> fr;
  fr.init(lane);
  constexpr int STAGE = 2 * Geo::SUB;
  __shared__ __align__(1024) char sk0[STAGE], sk1[STAGE], sv0[STAGE], sv1[STAGE];
  tl.ld.init(tl.kp, tl.vp, wave, wave);
  // The masks wait for the rows' lengths, while the first tiles are on their way.
  KeyMask mask{0, INT_MIN, 0, h};
  auto masks = [&] {
    mask.lim = !valid     ? -1
               : a.causal ? sq + a.Lp + sequence_length(a.lengths, b, a.Skv) - a.Sq
                          : 0x7fffffff;  // the last key the row sees
    tl.full_lo =
        __builtin_amdgcn_readfirstlane(wave_min(valid ? mask.lim : 0x7fffffff));
  };
  auto sees = [&] {
    return a.causal ? mask.lim >= 0 : a.Lp + sequence_length(a.lengths, b, a.Skv) > 0;
  };
  // The floor keeps a zero scale well defined (every visible key gets weight 1).
  roll_tiles<D, false>(tl, last - tl.first, mt * BM + wave * 32 < rows, Stages{sk0, sk1, sv0, sv1},
                       fr, row, fmaxf(a.c_abs, 1e-30f), mask, masks, sees);
  if (a.P == 1)
    store_row<D>(row, h, valid ? a.o + orow * D : nullptr);
  else
    store_state<D>(row, h, valid, a.ws_m, a.ws_l, a.ws_acc, orow * a.P + (packed ? p : a.P1 + p),
                   false);
}

}  // namespace

hipError_t launch_attention_prefix(const PrefixParams& a, hipStream_t stream) {
  const dim3 grid(a.n_prefix + a.n_own);
  if (a.D == 128)
    hipLaunchKernelGGL((attn_prefix_kernel<128, 4>), grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((attn_prefix_kernel<64, 4>), grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ef
