// Attention over selected blocks of the key axis: every query position has a list of
// blocks for its kv head, and sees the keys of those blocks up to its own.
//
// A workgroup holds 64 or 128 packed rows of a kv head (r = sq G + g), so the G heads
// of a position and several positions share each staged tile. It walks the union of
// their lists: a bitmap of the blocks, its ranks, and per block a mask of the
// positions that selected it. A row whose position did not select a block takes part
// in its products with weights of exactly 0 (the offset of its exponents is -inf).
// Neighbouring positions select much the same blocks, which makes the union little
// longer than one list; where they do not, the walk is never longer than the plain
// causal one. With few rows the tiles of the union are split over P workgroups.
//
// Lists may be in any order; entries outside 0 .. cur (the position's own block) are
// passed over, repeated ones count once.
//
// What bounds it: one token over 64 blocks of 64 keys, 16 sequences of 32/8 heads of 128
// (267 MB), 48 us, 5.5 TB/s: HBM, less the 3.5 us in which a workgroup makes its list. 4096
// queries over 16 blocks each of 512 (67 GFLOP) 127 to 132 us: the union of 32 positions'
// lists is 1.65 times one list, and about 30 us do not grow with it (with 26, 52 and 104
// blocks in every union 132, 230 and 419 us, the last 1.07 PFLOP/s): the starts and ends of
// two rounds of workgroups. Keys that lie in L2 save 6%. One token of one sequence over 16
// blocks 9.8 us: launch, the list, one tile's loads, and the combine by the last workgroup (3
// us). Tried and not kept: waves
// that pass over tiles none of their rows selected (131 -> 147 us; lists that share
// nothing 580 -> 520); the list from ranks of entries held in registers (3400 -> 2350
// cycles, but the walk slowed with it).
#include "roll_tiles.hpp"

namespace ef {

namespace {

constexpr int kWords = (kMaxBlocks + 31) / 32;
constexpr int kWindow = 512;  // blocks of the union that are walked at a time

// Union of the lists of the workgroup's positions, at most one to a row.
template <int NW>
struct UnionList {
  uint32_t word[kWords];       // bitmap
  int before[kWords];          // blocks below each word
  int block[kWindow];          // the window's blocks, ascending
  uint32_t mask[kWindow][NW];  // positions that selected them
  int waves[NW];
};

template <int D, int NW>
struct ListTiles {
  StageLoader<D, NW, NW> ld;
  const UnionList<NW>* u;
  int shift;    // log2 of the keys per block
  int cend;     // keys any row sees
  int full_lo;  // keys up to it are visible to all rows, as far as selected
  int pos;      // bit of this lane's position
  bool once;    // no other workgroup reads the keys: they stream past the caches

  __device__ __forceinline__ TileAt at(int t) const {
    const int per = shift - 6;
    const int n = __builtin_amdgcn_readfirstlane(u->block[t >> per]);
    const int base = (n << shift) + ((t & ((1 << per) - 1)) << 6);
    const int end = min(cend, (n + 1) << shift);
    return {base, end, base + 64 > end || base + 63 > full_lo, false};
  }
  __device__ __forceinline__ bool on(int t) const {
    return (u->mask[t >> (shift - 6)][pos >> 5] >> (pos & 31)) & 1;
  }
  template <bool ISK>
  __device__ __forceinline__ void load(char* stage, const TileAt& t) const {
    if (once)
      ld.template load<ISK, 2>(stage, t.base, t.end);
    else
      ld.template load<ISK>(stage, t.base, t.end);
  }
};

template <int D, int NW, bool SEL>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(NW == 2 ? 1 : 2)))
void attn_blocks_kernel(BlocksParams a) {
  using Geo = TileGeom<D>;
  constexpr int BM = 32 * NW, NT = 64 * NW;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, ql = lane & 31;

  // Workgroup -> (sequence and kv head, row tile, part). The row tiles of a head read
  // the same keys and run on one XCD, the longest first.
  const unsigned nwg = gridDim.x;
  unsigned id = blockIdx.x;
  if (nwg % kXcds == 0) id = (id % kXcds) * (nwg / kXcds) + id / kXcds;
  const int p = (int)(id % a.P);
  const int mt = a.mtiles - 1 - (int)(id / a.P % a.mtiles);
  const int bh = (int)(id / a.P / a.mtiles);
  const int b = bh / a.Hkv, hkv = bh % a.Hkv;

  const int r = mt * BM + wave * 32 + ql;
  const bool valid = r < a.R;
  const int sq = valid ? r / a.G : 0, g = valid ? r % a.G : 0;
  const size_t orow = ((size_t)b * a.Hq + (size_t)hkv * a.G + g) * a.Sq + sq;
  const int off = sequence_length(a.lengths, b, a.Skv) - a.Sq;
  const int lim = valid ? sq + off : -1;
  const int s0 = mt * BM / a.G, s1 = (min(mt * BM + BM, a.R) - 1) / a.G;  // positions

  Rows<D> row;
  row.init(a.q + orow * D, valid, a.qflip, h);
  FragmentReads<D> fr;
  fr.init(lane);
  constexpr int STAGE = 2 * Geo::SUB;
  __shared__ __align__(1024) char sk0[STAGE], sk1[STAGE], sv0[STAGE], sv1[STAGE];
  __shared__ UnionList<NW> u;
  ListTiles<D, NW> tl;
  const size_t head = (size_t)bh * a.Skv * D;
  tl.ld.init(a.k + head, a.v + head, wave, wave);
  tl.u = &u;
  tl.shift = a.shift;
  tl.cend = s1 + off + 1;
  tl.full_lo = s0 + off;
  tl.pos = valid ? sq - s0 : 0;
  tl.once = a.mtiles == 1;

  // Bitmap of the union: entries of the positions' lists, up to each one's own block.
  const int* lists = a.blocks + ((size_t)bh * a.Sq + s0) * a.K;
  const int entries = (s1 - s0 + 1) * a.K;
  const int words = (a.NB + 31) / 32;
  auto entry = [&](int e) {  // block of an entry, -1: none
    const int n = lists[e], d = s0 + e / a.K + off;
    return n >= 0 && d >= 0 && n <= d >> a.shift ? n : -1;
  };
  for (int i = threadIdx.x; i < words; i += NT) u.word[i] = 0;
  __syncthreads();
  for (int e = threadIdx.x; e < entries; e += NT) {
    const int n = entry(e);
    if (n >= 0) atomicOr(&u.word[n >> 5], 1u << (n & 31));
  }
  __syncthreads();
  // Blocks below each word: every thread takes a run of words.
  const int run = (words + NT - 1) / NT;
  const int w0 = min((int)threadIdx.x * run, words), w1 = min(w0 + run, words);
  int count = 0;
  for (int i = w0; i < w1; ++i) count += __popc(u.word[i]);
  int scan = count;
#pragma unroll
  for (int off2 = 1; off2 < 64; off2 *= 2) {
    const int x = __shfl_up(scan, off2, 64);
    if (lane >= off2) scan += x;
  }
  if (lane == 63) u.waves[wave] = scan;
  __syncthreads();
  int below = scan - count, total = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    if (w < wave) below += u.waves[w];
    total += u.waves[w];
  }
  for (int i = w0; i < w1; ++i) {
    u.before[i] = below;
    below += __popc(u.word[i]);
  }

  // This part's share of the union, a window at a time.
  total = __builtin_amdgcn_readfirstlane(total);
  const int first = (int)((long long)total * p / a.P);
  const int last = (int)((long long)total * (p + 1) / a.P);
  const KeyMask mask{lim, INT_MIN, 0, h};
  auto sees = [&] {  // a listed block up to the position's own holds a key that it sees
    bool any = false;
    for (int e = 0; e < a.K; ++e) any |= entry(tl.pos * a.K + e) >= 0;
    return any;
  };
  for (int f = first; f < last; f += kWindow) {
    const int n = min(last - f, kWindow);
    __syncthreads();
    for (int i = w0; i < w1; ++i) {
      uint32_t bits = u.word[i];
      for (int rank = u.before[i] - f; bits; ++rank, bits &= bits - 1)
        if (rank >= 0 && rank < n) {
          u.block[rank] = 32 * i + __builtin_ctz(bits);
#pragma unroll
          for (int w = 0; w < NW; ++w) u.mask[rank][w] = 0;
        }
    }
    __syncthreads();
    if constexpr (SEL) {
      for (int e = threadIdx.x; e < entries; e += NT) {
        const int m = entry(e), pos = e / a.K;
        if (m < 0) continue;
        const int rank = u.before[m >> 5] + __popc(u.word[m >> 5] & ((1u << (m & 31)) - 1)) - f;
        if (rank >= 0 && rank < n) atomicOr(&u.mask[rank][pos >> 5], 1u << (pos & 31));
      }
      __syncthreads();
    }
    // Tiles of the window; of the last block of all only those with a visible key.
    const int per = a.shift - 6;
    int tiles = n << per;
    const int tail = __builtin_amdgcn_readfirstlane(u.block[n - 1]);
    if (per && (tail << a.shift) + 64 >= tl.cend) --tiles;
    roll_tiles<D, SEL>(tl, tiles, mt * BM + wave * 32 < a.R, Stages{sk0, sk1, sv0, sv1}, fr, row,
                       fmaxf(a.c_abs, 1e-30f), mask, [] {}, sees);
  }
  if (NW == 4 || a.P == 1) {  // (tiles of 128 rows are for launches that need no parts)
    store_row<D>(row, h, valid ? a.o + orow * D : nullptr);
    return;
  }
  if constexpr (NW == 2) {
    const bool shared = a.counters != nullptr;
    store_state<D>(row, h, valid, a.ws_m, a.ws_l, a.ws_acc, orow * a.P + p, shared);
    if (!shared) return;
    // The last part of the head's rows to arrive combines them.
    unsigned* const counter = a.counters + (size_t)bh * kCounterStride;
    const size_t row0 = (size_t)bh * a.R;
    const unsigned ticket = arrival_ticket(counter);
    if (ticket >= (unsigned)a.P) poison_rows<D, NT>(a.o, row0, a.R);
    if (ticket != (unsigned)(a.P - 1)) return;
    combine_shared<D, NT>(a.ws_m, a.ws_l, a.ws_acc, a.o, row0, a.R, a.P);
    if (threadIdx.x == 0) reset_counter(counter);
  }
}

template <int D, int NW>
hipError_t launch_nw(const BlocksParams& a, hipStream_t stream) {
  const dim3 grid((unsigned)a.P * a.mtiles * a.B * a.Hkv);
  if (a.Sq > 1)
    hipLaunchKernelGGL((attn_blocks_kernel<D, NW, true>), grid, dim3(NW * 64), 0, stream, a);
  else
    hipLaunchKernelGGL((attn_blocks_kernel<D, NW, false>), grid, dim3(NW * 64), 0, stream, a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_d(const BlocksParams& a, hipStream_t stream) {
  return a.bm == 128 ? launch_nw<D, 4>(a, stream) : launch_nw<D, 2>(a, stream);
}

}  // namespace

hipError_t launch_attention_blocks(const BlocksParams& a, hipStream_t stream) {
  return a.D == 128 ? launch_d<128>(a, stream) : launch_d<64>(a, stream);
}

}  // namespace ef
