// Attention of packed sequences of different lengths: prompts, or chunks of them behind
// earlier keys.
//
// The rolling loop of the prefill kernel (rolling.hpp) over the rows of one sequence: a workgroup
// of four waves holds 128 rows r = i G + g of a kv head and walks the 64-key tiles that they see.
// Packed rows of K and V are Hkv D elements apart, so a tile's base is formed in 64 bits and
// its rows are loaded at that stride, straight to LDS.
//
// Work: a sequence has ceil(G n / 128) row tiles. Where all sequences' tiles do not fill the
// chip, or one of them has far more keys than its share, a sequence's keys are cut into equal parts
// of at most C tiles, C taken from the sums over the sequences that every workgroup forms for
// itself (64 at a time, a wave-wide sum): parts leave states in the workspace and a second kernel
// joins them. Up to 64 sequences run in the
// order of their parts' keys, longest first, and the tiles of one from its last rows on, so that
// the last workgroups to start are the shortest.
//
// What bounds it: the power limit and the issue of a step, as for the causal prefill kernel. 16 prompts
// of 101 to 4096 tokens of 32/8 heads of 128 (774 GFLOP) 770 to 800 us, 0.97 to 1.01 PFLOP/s: the clock
// is at 1.95 GHz, the matrix cores are busy 49% of the time and waves wait 28% of theirs (the first
// forty calls after a pause take up to 970 us, until the clock has settled); 16 equal ones of 2048 590
// to 603 us, where the prefill kernel on padded tensors takes 620. Chunks of 700 and 1500 tokens of
// 64/8 heads of 64 over 9001 and 16001 keys (382 GFLOP) 400 to 432 us, 0.88 to 0.95: the softmax of a
// score is the same beside half the products (1.93 GHz, matrix cores 45% busy), and 1104 workgroups of
// two lengths share 512 places. Finer parts lose more than they even out: at most a half
// / a third / a quarter of a place's share 410 -> 440 / 490 / 480 us. Three short prompts 11.4 us:
// round trips (sequences, first tiles, rows) and five key tiles.
#include "ef_serve.hpp"
#include "roll_tiles.hpp"
#include "wave_ops.hpp"

namespace ef {

namespace {

constexpr int kRows = 128;

template <int D>
struct PackedTiles {
  static constexpr int NW = 4;
  using G = TileGeom<D>;
  static constexpr int INSTS = 64 / G::RPI / NW;
  static constexpr int KPER = D == 128 ? 4 : 2;  // loads of the K permutation's period
  static constexpr int NK = INSTS < KPER ? INSTS : KPER;
  const char *k, *v;  // first key of the sequence and head
  unsigned stride;    // bytes from key to key
  unsigned koff[NK], voff;
  int row0, slot, wave;
  int first;     // first tile of the walk
  int end;       // keys any row sees
  int full_lo;   // keys up to it are visible to all rows of the wave

  __device__ __forceinline__ void init(const char* kh, const char* vh, unsigned bytes, int w) {
    const int lane = threadIdx.x & 63;
    k = kh;
    v = vh;
    stride = bytes;
    wave = w;
    row0 = w * INSTS * G::RPI + lane / G::KCH;
    slot = lane % G::KCH;
#pragma unroll
    for (int i = 0; i < NK; ++i)
      koff[i] = row0 * bytes + (slot ^ G::swz_k(row0 + i * G::RPI)) * 16;
    voff = row0 * bytes + (slot ^ G::swz_v(row0)) * 16;
  }
  __device__ __forceinline__ TileAt at(int t) const {
    const int base = (first + t) * 64;
    return {base, end, base + 64 > end || base + 63 > full_lo, false};
  }
  __device__ __forceinline__ bool on(int) const { return true; }
  template <bool ISK>
  __device__ __forceinline__ void load(char* stage, const TileAt& t) const {
    const int nrows = t.end - t.base;
    if (nrows <= 0) return;
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char*>((ISK ? k : v) + (size_t)t.base * stride), (short)0, -1, 0x00020000);
    char* const l = stage + wave * INSTS * 1024;
    if (nrows >= 64) {
      static_for<INSTS>([&](auto q) {
        constexpr int I = decltype(q)::value;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rs, (__attribute__((address_space(3))) void*)(l + I * 1024), 16,
            (int)(ISK ? koff[I % NK] : voff), (int)(I * G::RPI * stride), 0, 0);
      });
    } else {
      // Ragged tile: rows past the end repeat the last one (masked later).
#pragma unroll
      for (int i = 0; i < INSTS; ++i) {
        const int r = row0 + i * G::RPI;
        const int c = slot ^ (ISK ? G::swz_k(r) : G::swz_v(r));
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rs, (__attribute__((address_space(3))) void*)(l + i * 1024), 16,
            (int)((unsigned)min(r, nrows - 1) * stride + c * 16), 0, 0, 0);
      }
    }
  }
};

// Rows and keys of a sequence.
struct Extent {
  int start, n, kstart, len;
  __device__ __forceinline__ void load(const PackedParams& a, int b) {
    const int s0 = a.starts[b], s1 = a.starts[b + 1], k0 = a.k_starts[b], k1 = a.k_starts[b + 1];
    start = min(max(s0, 0), a.T);
    n = max(min(max(s1, 0), a.T) - start, 0);
    kstart = min(max(k0, 0), a.Tk);
    len = max(min(max(k1, 0), a.Tk) - kstart, 0);
  }
  __device__ __forceinline__ int row_tiles(const PackedParams& a) const {
    return (int)(((unsigned)(n * a.G) + kRows - 1) / kRows);  // (n G is below 2^31 - 128)
  }
  __device__ __forceinline__ int key_tiles() const { return max((len + 63) / 64, 1); }
  // Keys that some row of row tile mt sees.
  __device__ __forceinline__ int seen(const PackedParams& a, int mt) const {
    if (!a.causal) return len;
    const int top = min(mt * kRows + kRows, n * a.G) - 1;
    return min(max((int)((unsigned)top / (unsigned)a.G) + len - n + 1, 0), len);
  }
};

// 64 sequences, one to a lane: their row tiles, key tiles, and how the keys are cut.
struct Cut {
  Extent x;
  int m, kt;         // row tiles, key tiles
  int parts, each;   // equal parts of the keys, key tiles of one
  int units, split;  // workgroups, and those that leave a state
  __device__ __forceinline__ void load(const PackedParams& a, int b0) {
    const int b = b0 + (int)(threadIdx.x & 63);
    m = kt = 0;
    if (b < a.B) {
      x.load(a, b);
      m = x.row_tiles(a);
      kt = x.key_tiles();
    }
  }
  __device__ __forceinline__ void cut(int most) {
    parts = max((int)(((unsigned)kt + (unsigned)most - 1) / (unsigned)most), 1);
    each = ((unsigned)kt + parts - 1) / (unsigned)parts;
    units = m * parts;
    split = parts > 1 ? units : 0;
  }
};

// Most key tiles of a part, and the row tiles of all sequences. The same in every workgroup of both
// launches. `c` is left with the last 64 sequences.
__device__ __forceinline__ int most_tiles(const PackedParams& a, Cut& c, int& rows) {
  float work = 0.f;
  rows = 0;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    c.load(a, b0);
    rows += __builtin_amdgcn_readlane(wave_scan(c.m), 63);
    work += wave_sum((float)c.m * (float)c.kt);
  }
  if (a.slots == 0) return 0x7fffffff;
  const int places = rows >= a.fill ? a.fill : max(a.fill - rows, (a.fill + 1) / 2);
  // At least work / places, for all that fp32 rounds (half a step for each 64 sequences, 1e-9 of
  // the sum for one): the states' room counts on it.
  const float room = 1.001f + 1e-9f * (float)a.B;
  const int most = (int)fminf(work * room / (float)places + 1.f, 2e9f);
  return max(__builtin_amdgcn_readfirstlane(most), a.least);
}

// States of a kv head that the call makes.
__device__ __forceinline__ int count_states(const PackedParams& a) {
  Cut c;
  int rows, all = 0;
  const int most = most_tiles(a, c, rows);
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    if (a.B > 64) c.load(a, b0);
    c.cut(most);
    all += __builtin_amdgcn_readlane(wave_scan(c.split), 63);
  }
  return min(max(all, 0), a.slots);
}

// What workgroup `id` of a kv head does.
struct Unit {
  Extent e;
  int mt;    // row tile
  int p, P;  // part, parts of the sequence's row tiles (fewer may have keys)
  int C;     // key tiles of a part
  int slot;  // its state, where P > 1
  // Workgroup `id` in the order of the launch, or with SLOTS the one that has state `id`. False:
  // there is none. The same for all waves.
  template <bool SLOTS>
  __device__ __forceinline__ bool find(const PackedParams& a, int id) {
    const int lane = threadIdx.x & 63;
    Cut c;
    int rows;
    const int most = most_tiles(a, c, rows);
    int before = 0, slots = 0;  // of the sequences in front of these 64
    for (int b0 = 0; b0 < a.B; b0 += 64) {
      if (a.B > 64) c.load(a, b0);
      c.cut(most);
      // Units in front of this lane's sequence.
      int front = 0;
      if (a.B <= 64 && rows > a.fill) {  // (in one round the order does not matter)
        for (int i = 0; i < a.B; ++i) {
          const int k = __builtin_amdgcn_readlane(c.each, i);
          const int n = __builtin_amdgcn_readlane(c.units, i);
          front += k > c.each || (k == c.each && i < lane) ? n : 0;
        }
      } else {
        front = wave_scan(c.units) - c.units;
      }
      const int sfront = wave_scan(c.split) - c.split;
      const int lo = SLOTS ? slots + sfront : before + front;
      const auto hit =
          __builtin_amdgcn_ballot_w64(id >= lo && id < lo + (SLOTS ? c.split : c.units));
      if (hit) {
        const int at = __builtin_ctzll(hit);
        e.start = __builtin_amdgcn_readlane(c.x.start, at);
        e.n = __builtin_amdgcn_readlane(c.x.n, at);
        e.kstart = __builtin_amdgcn_readlane(c.x.kstart, at);
        e.len = __builtin_amdgcn_readlane(c.x.len, at);
        P = __builtin_amdgcn_readlane(c.parts, at);
        C = __builtin_amdgcn_readlane(c.each, at);
        const int tiles = __builtin_amdgcn_readlane(c.m, at);
        const int in = id - __builtin_amdgcn_readlane(lo, at);
        mt = tiles - 1 - (int)((unsigned)in / (unsigned)P);
        p = (int)((unsigned)in % (unsigned)P);
        slot = slots + __builtin_amdgcn_readlane(sfront, at) + in;
        return P == 1 || (unsigned)slot < (unsigned)a.slots;  // (always, where starts ascend)
      }
      before += __builtin_amdgcn_readlane(wave_scan(c.units), 63);
      slots += __builtin_amdgcn_readlane(wave_scan(c.split), 63);
    }
    return false;
  }
  // Parts of this row tile that have keys.
  __device__ __forceinline__ int used(const PackedParams& a) const {
    const int t = (e.seen(a, mt) + 63) / 64;
    return P == 1 ? 1 : max((t + C - 1) / C, 1);
  }
};

template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
void attn_packed_kernel(PackedParams a) {
  using Geo = TileGeom<D>;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, ql = lane & 31;
  const int hk = (int)(blockIdx.x % a.Hkv);
  Unit u;
  if (blockIdx.x == gridDim.x - 1 && a.slots > 0) {  // one more than the others
    const int states = count_states(a);
    if (threadIdx.x == 0) *a.split = states;
    return;
  }
  if (!u.find<false>(a, (int)(blockIdx.x / a.Hkv))) return;
  const Extent& e = u.e;
  const int rows = e.n * a.G;
  const int r = u.mt * kRows + wave * 32 + ql;
  const bool valid = r < rows;
  const int i = valid ? (unsigned)r / (unsigned)a.G : 0, g = valid ? r - i * a.G : 0;
  const size_t orow = ((size_t)(e.start + i) * a.Hq + (size_t)hk * a.G + g) * D;

  PackedTiles<D> tl;
  const size_t key0 = ((size_t)e.kstart * a.Hkv + hk) * (2 * D);
  tl.init(reinterpret_cast<const char*>(a.k) + key0, reinterpret_cast<const char*>(a.v) + key0,
          (unsigned)a.Hkv * (2 * D), wave);
  tl.end = e.seen(a, u.mt);
  const int tiles = (tl.end + 63) / 64;
  tl.first = u.P == 1 ? 0 : u.p * u.C;
  const int last = u.P == 1 ? tiles : min(tiles, tl.first + u.C);
  if (u.p > 0 && tl.first >= tiles) return;

  Rows<D> row;
  row.init(a.q + orow, valid, a.qflip, h);
  FragmentReads<D> fr;
  fr.init(lane);
  constexpr int STAGE = 2 * Geo::SUB;
  __shared__ __align__(1024) char sk0[STAGE], sk1[STAGE], sv0[STAGE], sv1[STAGE];
  KeyMask mask{!valid ? -1 : a.causal ? i + e.len - e.n : 0x7fffffff, INT_MIN, 0, h};
  tl.full_lo = __builtin_amdgcn_readfirstlane(wave_min(valid ? mask.lim : 0x7fffffff));
  auto sees = [&] { return mask.lim >= 0 && e.len > 0; };
  roll_tiles<D, false>(tl, last - tl.first, u.mt * kRows + wave * 32 < rows,
                       Stages{sk0, sk1, sv0, sv1}, fr, row, fmaxf(a.c_abs, 1e-30f), mask, [] {},
                       sees);
  if (u.P == 1) {
    store_row<D>(row, h, valid ? a.o + orow : nullptr);
  } else {
    const size_t slot = ((size_t)hk * a.slots + u.slot) * kRows + wave * 32 + ql;
    store_state<D>(row, h, valid, a.ws_m, a.ws_l, a.ws_acc, slot, false);
  }
}

// Joins the parts of split row tiles: kShares workgroups for each of a tile's P states, one wave a
// row, D / 4 lanes a state.
constexpr int kShares = 4;
template <int D>
__global__ __launch_bounds__(256) void packed_combine_kernel(PackedParams a) {
  constexpr int LPS = D / 4, SPL = 64 / LPS, BATCH = 8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // (Often nothing is split: the first launch counted the states.)
  if ((int)(blockIdx.x / kShares / a.Hkv) >= *a.split) return;
  const int share = (int)(blockIdx.x % kShares);
  const int hk = (int)(blockIdx.x / kShares % a.Hkv);
  Unit u;
  if (!u.find<true>(a, (int)(blockIdx.x / kShares / a.Hkv))) return;
  const int rows = min(kRows, u.e.n * a.G - u.mt * kRows);
  const int P = u.used(a);
  const size_t slot0 = (size_t)hk * a.slots + u.slot - u.p;  // state of part 0
  const int grp = lane / LPS, ch = lane % LPS;
  for (int r = u.p + u.P * (4 * share + wave); r < rows; r += u.P * 4 * kShares) {
    auto state = [&](int p) { return (slot0 + p) * kRows + r; };
    float M = kNegInf, L = 0.f;
    floatx4 x = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = 0; p0 < P; p0 += 64) {
      const int count = min(P - p0, 64);
      const float m = lane < count ? a.ws_m[state(p0 + lane)] : kNegInf;
      const float l = lane < count ? a.ws_l[state(p0 + lane)] : 0.f;
      const float top = fmaxf(M, wave_max(m));
      const float ref = top == kNegInf ? 0.f : top;
      const float wt = exp2_fast((m - ref) * kLog2e);
      const float old = exp2_fast((M - ref) * kLog2e);
      L = L * old + wave_sum(wt * l);
      M = top;
#pragma unroll
      for (int c = 0; c < 4; ++c) x[c] *= old;
      for (int j = 0; j < count; j += BATCH * SPL) {
        floatx4 y[BATCH];
#pragma unroll
        for (int q = 0; q < BATCH; ++q)
          y[q] = *reinterpret_cast<const floatx4*>(
              a.ws_acc + state(p0 + min(j + q * SPL + grp, count - 1)) * D + 4 * ch);
#pragma unroll
        for (int q = 0; q < BATCH; ++q) {
          const int s = j + q * SPL + grp;
          const float ws = __shfl(wt, min(s, 63), 64);
          // (a state without a key was not stored)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            x[c] = s < count && ws > 0.f ? fmaf(ws, y[q][c], x[c]) : x[c];
        }
      }
    }
#pragma unroll
    for (int off = LPS; off < 64; off *= 2)
#pragma unroll
      for (int c = 0; c < 4; ++c) x[c] += shfl_xor(x[c], off);
    if (grp == 0) {
      const int rr = u.mt * kRows + r;
      const float inv = L == 0.f ? 0.f : 1.f / L;
      const size_t orow =
          ((size_t)(u.e.start + rr / a.G) * a.Hq + (size_t)hk * a.G + rr % a.G) * D;
      const u32x2_t o = {pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv)};
      *reinterpret_cast<u32x2_t*>(a.o + orow + 4 * ch) = o;
    }
  }
}

template <int D>
hipError_t launch_d(const PackedParams& a, hipStream_t stream) {
  const dim3 grid((unsigned)a.per_head * a.Hkv + (a.slots > 0 ? 1 : 0));
  hipLaunchKernelGGL(attn_packed_kernel<D>, grid, dim3(256), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.slots == 0) return e;
  hipLaunchKernelGGL(packed_combine_kernel<D>, dim3((unsigned)a.slots * a.Hkv * kShares), dim3(256),
                     0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attention_packed(const PackedParams& a, hipStream_t stream) {
  return a.D == 128 ? launch_d<128>(a, stream) : launch_d<64>(a, stream);
}

}  // namespace ef
