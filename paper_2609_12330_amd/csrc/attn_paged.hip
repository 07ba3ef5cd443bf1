// Attention of a few new tokens of every sequence over a paged cache.
//
// The G heads of a kv head and a sequence's tokens make rows r = i G + g, 16 or 32 of which a
// workgroup holds (one or two column tiles of the matrix core). Its four waves take keys of
// their own, KT of them a step, and carry a softmax state (reference, sum, value) over them;
// the states of the waves are joined in LDS at the end. A step is, for 16 keys at a time,
//
//   S^T[key][row] = K (A operand) Q^T (B operand),   O^T[d][row] += V^T (A) P^T (B)
//
// with v_mfma_f32_16x16x32_bf16. K goes from memory to registers as the A operand; the second
// product's sum over keys may run in any order, so the scores of two 16-key tiles, turned to
// weights and packed, are its B operand where they stand; V goes to LDS without passing
// registers and is read transposed. No wave waits for another before the end.
//
// 8-bit caches: e4m3 codes are exact in bf16, and scales factor out of both products, a key's of
// its score and a value's of its weight (16 keys at a time, four floats a lane).
//
// Work: the keys of all sequences, in units of 64, make one list for each kv head (and row
// tile), which W workgroups cut into equal runs, whatever the lengths. A run holds the end of
// one sequence, whole ones, and the beginning of another; what is cut leaves a state in the
// workspace (two slots a workgroup), and the last of a row's parts joins them, or a second kernel.
//
// What bounds it: HBM where there is work: 32 sequences of 2001 to 32768 keys of 8 heads of 128, one
// token of 32 heads each (2.28 GB) 350 us, 6.5 TB/s. With 32 rows and 8-bit keys the matrix core
// and the conversions have their share: 16 sequences of 501 to 16384 keys, 1 to 4 tokens of 64/8
// heads (286 MB) 58 us and 5 the second kernel; with loads alone 4 less, so what is left is the start
// (6 us until the first keys are there), and workgroups with the end of one sequence and the start of
// another. One sequence of 777 keys 12 us: lengths, table, keys, join of the waves, ticket, join of
// seven parts, a round trip each. What made it fast: the next step's loads in flight over a step's
// products, always the same number of them so that the wait can tell them apart (89 -> 81 us);
// sequences that count what changing to them costs (81 -> 69); table entries requested before rows
// (69 -> 63). Tried and not kept: workgroups of their own for sequences of equal lengths (8 of 8192
// keys, 8 tokens each, 60.5 -> 56.3 us, but 0.2 to 0.4 us more for every other call).
#include <algorithm>

#include "ef_device.hpp"
#include "ef_serve.hpp"
#include "group_combine.hpp"
#include "wave_ops.hpp"

namespace ef {

namespace {

constexpr int kUnit = 64;             // keys of a unit of work
// Bytes of keys that a sequence counts beside its own: what a workgroup takes from one sequence to
// the next (rows, table, the first loads' way, the join of its waves). 31 sequences of 1122 keys of
// 4 heads, e4m3, 64 / 128 / 192 / 256 KiB 16.7 / 17.5 / 18.6 / 20.5 us; 41 of 5098 of 8 heads 98.5 /
// 99.8 / 98.6 / 97.0; 32 long ones 350 / 352 / 353 / 354.
constexpr int kExtraBytes = 64 * 1024;
constexpr int kWideChannels = 32;  // of a row that a workgroup joins from hundreds of parts
constexpr float kHeadroom = 8.f;   // base-2 headroom before the reference moves
constexpr int kStageBytes = 8192;  // keys, and values, of a wave's step

// A value that is the same in all lanes, for the compiler to see.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
// Waits until at most N of the wave's loads are on their way.
template <int N>
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4) << 14);
}

typedef int v2i __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
#define EF_LDS(T, p) (__attribute__((address_space(3))) T*)(p)

template <int D, bool E4M3>
struct Geo {
  static constexpr int ROWB = D * (E4M3 ? 1 : 2);  // bytes of a cached row
  static constexpr int KCH = ROWB / 16;
  static constexpr int KT = kStageBytes / ROWB;  // keys of a wave's step
  static constexpr int T16 = KT / 16;
  static constexpr int SUBS = KT / 32;
  static constexpr int KL = ROWB / 64;    // 16-byte loads a lane makes for 16 keys
  static constexpr int RPI = 64 / KCH;    // rows of a wave-wide load
  static constexpr int DT = D / 16;
  // Slot of a value row's 16-byte chunk c is c ^ swz(row): the transposing reads take 8 rows
  // (bf16, 32 bytes of each) or 16 (e4m3, 16 bytes) from different banks.
  static __device__ __forceinline__ int swz(int r) {
    return E4M3 ? (D == 128 ? (r >> 1) & 7 : (r >> 2) & 3)
                : (D == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3));
  }
};

// Sequences 64 at a time, one to a lane.
struct Sequences {
  int base;             // first one
  int start, n, len;    // rows and keys of this lane's sequence
  int keys;             // units that hold keys of its rows in this row tile, at least one
  int units;            // these, and EXTRA
  int scan;             // units up to and with it, from sequence `base` on
  template <int EXTRA>
  __device__ __forceinline__ void load(const PagedParams& a, int from, int row0, int rows) {
    base = from;
    const int b = from + (int)(threadIdx.x & 63);
    start = n = len = units = keys = 0;
    if (b < a.B) {
      // Three loads at once, whether there are starts or not.
      const int* const p = a.starts != nullptr ? a.starts + b : a.lengths + b;
      const int s0 = p[0], s1 = p[a.starts != nullptr ? 1 : 0], l = a.lengths[b];
      start = a.starts != nullptr ? min(max(s0, 0), a.T) : b * a.even;
      n = a.starts != nullptr ? max(min(max(s1, 0), a.T) - start, 0) : a.even;
      len = min(max(l, 0), a.c.width << a.c.shift);
      if (row0 < min(n, a.max_queries) * a.G) {
        keys = max((last_key(a, row0, rows) + kUnit) / kUnit, 1);
        units = keys + EXTRA;
      }
    }
    scan = wave_scan(units);
  }
  // Last key that any of the tile's rows sees (-1: none).
  __device__ __forceinline__ int last_key(const PagedParams& a, int row0, int rows) const {
    const int top = min(row0 + rows, min(n, a.max_queries) * a.G) - 1;
    return max((int)((unsigned)top / (unsigned)a.G) + len - n, -1);
  }
};

// Parts p0 .. p1 - 1 of a row joined by one wave: the value's channels c0 .. c0 + CH - 1 (CH / 4
// lanes, four each, the same in every group of them) and the sum against the reference M (base-2
// units).
struct Joined {
  floatx4 x;
  float M, L;
};
template <int D, int CH, int BATCH, bool SHARED, class State>
__device__ __forceinline__ Joined join_parts(const PagedParams& a, int p0, int p1, int c0,
                                             State state) {
  constexpr int LPS = CH / 4, SPL = 64 / LPS;  // lanes of a state, states of a wave-wide load
  const int lane = threadIdx.x & 63, grp = lane / LPS, ch = lane % LPS;
  const __amdgpu_buffer_rsrc_t rs =
      __builtin_amdgcn_make_buffer_rsrc(a.ws_acc, (short)0, -1, 0x00020000);
  auto value = [&](int p) -> floatx4 {
    const size_t at = state(p) * D + c0 + 4 * ch;
    if constexpr (SHARED) return __builtin_bit_cast(floatx4, load16_dev(rs, (int)(at * 4)));
    return *reinterpret_cast<const floatx4*>(a.ws_acc + at);
  };
  Joined j = {{0.f, 0.f, 0.f, 0.f}, kNegInf, 0.f};
  for (; p0 < p1; p0 += 64) {
    const int count = min(p1 - p0, 64);
    float m = kNegInf, l = 0.f;
    if (lane < count) {
      m = load_dev(a.ws_m + state(p0 + lane));
      l = load_dev(a.ws_l + state(p0 + lane));
    }
    floatx4 y[BATCH];
    auto fetch = [&](int q) {
#pragma unroll
      for (int i = 0; i < BATCH; ++i) y[i] = value(p0 + min(q + i * SPL + grp, count - 1));
    };
    fetch(0);
    const float top = fmaxf(j.M, wave_max(m));
    const float ref = top == kNegInf ? 0.f : top;
    const float wt = exp2_fast(m - ref);  // 0 from -inf
    const float old = exp2_fast(j.M - ref);
    j.L = j.L * old + wave_sum(wt * l);
    j.M = top;
#pragma unroll
    for (int e = 0; e < 4; ++e) j.x[e] *= old;
    for (int q = 0; q < count; q += BATCH * SPL) {
      if (q > 0) fetch(q);
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int s = q + i * SPL + grp;
        const float ws = __shfl(wt, min(s, 63), 64);
#pragma unroll
        for (int e = 0; e < 4; ++e) j.x[e] = s < count ? fmaf(ws, y[i][e], j.x[e]) : j.x[e];
      }
    }
  }
#pragma unroll
  for (int off = LPS; off < 64; off *= 2)
#pragma unroll
    for (int e = 0; e < 4; ++e) j.x[e] += shfl_xor(j.x[e], off);
  return j;
}
template <int CH>
__device__ __forceinline__ void store_joined(const Joined& j, float inv, uint16_t* o) {
  const int lane = threadIdx.x & 63;
  if (lane >= CH / 4) return;
  const u32x2_t p = {pack_bf16x2(j.x[0] * inv, j.x[1] * inv),
                     pack_bf16x2(j.x[2] * inv, j.x[3] * inv)};
  *reinterpret_cast<u32x2_t*>(o + 4 * lane) = p;
}

// (A function beside the kernel: the host's compiler reads a kernel's body too, and does not know
// buffers.)
template <int D, bool E4M3, int RT, int NT>
__device__ __forceinline__ void attend_pages(const PagedParams& a) {
  using G = Geo<D, E4M3>;
  constexpr int ROWS = 16 * RT, KT = G::KT, DT = G::DT;
  constexpr int LEAST = 4 * KT / kUnit;  // units of a run: a step of each wave
  constexpr int EXTRA = kExtraBytes / (2 * kUnit * G::ROWB);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, l16 = lane & 15;

  // Workgroup -> (kv head, row tile), place in its list. The row tiles of a head read the same
  // keys and run on one XCD.
  unsigned id = blockIdx.x;
  if (gridDim.x % kXcds == 0) id = (id % kXcds) * (gridDim.x / kXcds) + id / kXcds;
  const int mt = (int)(id % a.mtiles);
  const int hk = (int)(id / a.mtiles % a.Hkv);
  const int w = (int)(id / a.heads);
  const int head = hk * a.mtiles + mt;
  const int row0 = mt * ROWS;

  __shared__ __align__(1024) char sv0[4][kStageBytes], sv1[4][kStageBytes];
  // Scales of keys and values, objects of their own for each stage like the values', so that the
  // compiler tells the loads into one from the reads of the other.
  __shared__ __align__(16) float sks0[4][KT], sks1[4][KT], svs0[4][KT], svs1[4][KT];
  __shared__ float sm[4][ROWS], sl[4][ROWS];

  // This workgroup's run of the list.
  Sequences s;
  s.template load<EXTRA>(a, 0, row0, ROWS);
  int total = __builtin_amdgcn_readlane(s.scan, 63);
  for (int b = 64; b < a.B; b += 64) {
    s.template load<EXTRA>(a, b, row0, ROWS);
    total += __builtin_amdgcn_readlane(s.scan, 63);
  }
  const int T = max((int)(((unsigned)total + a.W - 1) / (unsigned)a.W), LEAST);
  int u = (int)min((long long)w * T, (long long)total);
  const int u_end = (int)min((long long)u + T, (long long)total);
  if (u >= u_end) return;
  // Its first sequence.
  int before = 0;  // units in front of the sequences of `s`
  if (a.B > 64) s.template load<EXTRA>(a, 0, row0, ROWS);
  auto skip = [&] {
    while (s.base + 64 < a.B && before + __builtin_amdgcn_readlane(s.scan, 63) <= u) {
      before += __builtin_amdgcn_readlane(s.scan, 63);
      s.template load<EXTRA>(a, s.base + 64, row0, ROWS);
    }
  };

  while (u < u_end) {
    skip();
    const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(before + s.scan > u));
    const int b = s.base + at;
    const int units = __builtin_amdgcn_readlane(s.keys, at);
    const int behind = before + __builtin_amdgcn_readlane(s.scan, at);  // the next one's first unit
    const int first = behind - units - EXTRA;  // its first unit
    if (u >= first + units) {  // nothing of its keys
      u = min(u_end, behind);
      continue;
    }
    const int len = __builtin_amdgcn_readlane(s.len, at);
    const int n = __builtin_amdgcn_readlane(s.n, at);
    const int start = __builtin_amdgcn_readlane(s.start, at);
    const int nrows = min(ROWS, min(n, a.max_queries) * a.G - row0);
    const int end_seen =  // keys any row sees
        (int)((unsigned)(row0 + nrows - 1) / (unsigned)a.G) + len - n + 1;
    const int k0 = uniform((u - first) * kUnit);
    const int u_next = min(u_end, first + units);
    const int k1 = min((u_next - first) * kUnit, end_seen);

    // This wave's steps.
    const int steps = k1 > k0 ? (k1 - k0 + KT - 1) / KT : 0;
    const int j0 = uniform(steps * wave / 4), j1 = uniform(steps * (wave + 1) / 4);
    int wend = uniform(min(k1, k0 + j1 * KT));  // keys it may read
    int bad_from = 0x7fffffff;                  // first key of a page that is none
    const int page_mask = (1 << a.c.shift) - 1;
    // Table entries p0 .. p0 + 63, one to a lane (from the last one on, that one).
    const int* const table = a.c.table + (size_t)b * a.c.width;
    int p0 = uniform((k0 + j0 * KT) >> a.c.shift), pv = 0;
    auto entries = [&] { return table[min(p0 + lane, max((wend - 1) >> a.c.shift, 0))]; };
    auto check_entries = [&] {
      const bool bad = (unsigned)pv >= (unsigned)a.c.pages;
      const auto none = __builtin_amdgcn_ballot_w64(bad);
      if (none) {  // the walk ends in front of it
        const int from = (p0 + __builtin_ctzll(none)) << a.c.shift;
        if (from < wend) bad_from = from;
        wend = uniform(min(wend, from));
        pv = bad ? 0 : pv;
      }
    };
    const bool some = k1 > k0;  // (else the rows see no key at all)
    if (some) pv = entries();

    // Rows: queries, the last key they see.
    bf16x8_t qf[RT][D / 32];
    int lim[RT];
    size_t orow[RT];
    int full = 0x7fffffff;  // last key that every row sees
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int r = row0 + 16 * t + l16;
      const bool valid = 16 * t + l16 < nrows;
      const int i = valid ? (unsigned)r / (unsigned)a.G : 0, hq = valid ? r - i * a.G : 0;
      lim[t] = valid ? i + len - n : -1;
      full = min(full, valid ? lim[t] : full);
      orow[t] = ((size_t)(start + i) * a.Hq + (size_t)hk * a.G + hq) * D;
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        // Element order of an 8-bit key's 16-byte load: two steps' operands side by side.
        const int d = E4M3 ? 64 * (x / 2) + 16 * g + 8 * (x % 2) : 32 * x + 8 * g;
        // (Rows that are none read row 0 of the sequence, and are zeroed below.)
        qf[t][x] = __builtin_bit_cast(bf16x8_t,
                                      *reinterpret_cast<const u32x4_t*>(a.q + orow[t] + d));
      }
    }
    full = wave_min(full);

    // State.
    floatx4 oacc[RT][DT];
    float mref[RT], lsum[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      mref[t] = kNegInf;
      lsum[t] = 0.f;
#pragma unroll
      for (int i = 0; i < DT; ++i) oacc[t][i] = floatx4{0.f, 0.f, 0.f, 0.f};
    }

    u32x4_t kx[2][8];
    // First row of 16 keys (which lie in one page) in the cache of this head.
    auto cell_of = [&](int key) -> size_t {
      const int page = __builtin_amdgcn_readlane(pv, (key >> a.c.shift) - p0);
      return (((size_t)(unsigned)page * a.Hkv + hk) << a.c.shift) + (unsigned)(key & page_mask);
    };
    auto load = [&](auto stage, int j) {
      constexpr int S = decltype(stage)::value;
      const int kb = k0 + j * KT;
      if (((min(kb + KT, wend) - 1) >> a.c.shift) - p0 >= 64) {
        p0 = uniform(kb >> a.c.shift);
        pv = entries();
        check_entries();
      }
      // Each 16 keys have a buffer of their own that ends behind the last one the wave may read:
      // rows past it are zeros (masked later), and a step past it as a whole moves nothing, but
      // its loads count: the same number is in flight whichever way the walk goes, so that waits
      // can leave the next step's there.
      char* const vs = S == 0 ? sv0[wave] : sv1[wave];
      auto buffer = [&](const char* base, int t) {
        const int key = kb + 16 * t;
        const int rows = min(max(wend - key, 0), 16);
        const uint64_t p = (uint64_t)(uintptr_t)base + cell_of(key) * G::ROWB;
        const uint64_t q = (uint64_t)(unsigned)uniform((int)(p >> 32)) << 32 |
                           (unsigned)uniform((int)p);
        return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<char*>((uintptr_t)q), (short)0,
                                                 uniform(rows * G::ROWB), 0x00020000);
      };
#pragma unroll
      for (int t = 0; t < G::T16; ++t) {
        const __amdgpu_buffer_rsrc_t rs = buffer(a.c.k, t);
#pragma unroll
        for (int x = 0; x < G::KL; ++x)
          kx[S][t * G::KL + x] =
              __builtin_amdgcn_raw_buffer_load_b128(rs, l16 * G::ROWB + g * 16 + 64 * x, 0, NT);
      }
#pragma unroll
      for (int t = 0; t < G::T16; ++t) {
        const __amdgpu_buffer_rsrc_t rs = buffer(a.c.v, t);
        constexpr int N = 16 / G::RPI;  // loads of 16 rows
#pragma unroll
        for (int x = 0; x < N; ++x) {
          const int r = x * G::RPI + lane / G::KCH;
          __builtin_amdgcn_raw_ptr_buffer_load_lds(
              rs, EF_LDS(void, vs + (t * N + x) * 1024), 16,
              r * G::ROWB + ((lane % G::KCH) ^ G::swz(r)) * 16, 0, 0, NT);
        }
      }
      if constexpr (E4M3) {
#pragma unroll
        for (int x = 0; x < KT / 64; ++x) {
          const int key = min(kb + 64 * x + lane, wend - 1);
          const int page = __shfl(pv, (key >> a.c.shift) - p0, 64);
          const size_t cell = (((size_t)(unsigned)page * a.Hkv + hk) << a.c.shift) +
                              (unsigned)(key & page_mask);
          float* const ks = (S == 0 ? sks0 : sks1)[wave] + 64 * x;
          float* const vsc = (S == 0 ? svs0 : svs1)[wave] + 64 * x;
          __builtin_amdgcn_global_load_lds(a.c.k_scale + cell, EF_LDS(void, ks), 4, 0, 0);
          __builtin_amdgcn_global_load_lds(a.c.v_scale + cell, EF_LDS(void, vsc), 4, 0, 0);
        }
      }
    };
    // Waits for a step's loads, the next step's being the only ones behind them. (In the source:
    // the compiler was seen to leave out the wait for one of the stages in LDS.)
    constexpr int LOADS = 16 + (E4M3 ? 2 * (KT / 64) : 0);  // of a step
    auto landed = [] {
      asm volatile("" ::: "memory");  // (no load of the next step sinks below the wait)
      __builtin_amdgcn_sched_barrier(0);
      wait_loads<LOADS>();
      __builtin_amdgcn_sched_barrier(0);
    };
    // This lane's transposing reads of values: 16-byte chunk c of its row, at slot c ^ swz(row).
    // Chunks are 2 i (and the next) of bf16 rows, i of e4m3 ones, so i turns the offset by an
    // exclusive or.
    constexpr int SLOT = E4M3 ? 16 : 32;
    const int r8 = l16 >> 1;
    const int vrow = E4M3 ? 16 * (r8 >> 2) + 4 * g + (r8 & 3) : 4 * g + (l16 >> 2);
    const int vlow = vrow * G::ROWB + 8 * (l16 & 1) + (E4M3 ? 0 : 16 * ((l16 & 3) >> 1));
    const int vturn = 16 * G::swz(vrow);
    // Fragment i of the 32 keys at byte `at` of a stage.
    auto value = [&](const char* vs, int turn, int at, int i) -> bf16x8_t {
      const char* const p = vs + vlow + ((i * SLOT) ^ turn) + at;
      if constexpr (E4M3) {
        const v2i c = __builtin_amdgcn_ds_read_tr8_b64_v2i32(EF_LDS(v2i, p));
        const u32x4_t f = {(uint32_t)c[0], (uint32_t)c[1], 0u, 0u};
        return __builtin_bit_cast(bf16x8_t, f);
      } else {
        const bf16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(EF_LDS(bf16x4_t, p));
        const bf16x4_t hi =
            __builtin_amdgcn_ds_read_tr16_b64_v4bf16(EF_LDS(bf16x4_t, p + 16 * G::ROWB));
        return bf16x8_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      }
    };
    // Eight e4m3 codes as bf16.
    auto widen = [](uint32_t c0, uint32_t c1) -> bf16x8_t {
      const uint32_t c[2] = {c0, c1};
      u32x4_t f;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        f[2 * e] = __builtin_bit_cast(uint32_t,
                                      __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[e], 1.f, false));
        f[2 * e + 1] = __builtin_bit_cast(
            uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[e], 1.f, true));
      }
      return __builtin_bit_cast(bf16x8_t, f);
    };
    auto compute = [&](auto stage, int j) {
      constexpr int S = decltype(stage)::value;
      const int kb = k0 + j * KT;
      landed();
      if (kb >= wend) return;
      const char* const vs = S == 0 ? sv0[wave] : sv1[wave];
      // Scores: element i of tile t is key 16 t + 4 g + i.
      floatx4 x[RT][G::T16];
#pragma unroll
      for (int t = 0; t < G::T16; ++t) {
#pragma unroll
        for (int r = 0; r < RT; ++r) x[r][t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int y = 0; y < G::KL; ++y) {
          const u32x4_t kv = kx[S][t * G::KL + y];
          if constexpr (E4M3) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const bf16x8_t c = widen(kv[2 * e], kv[2 * e + 1]);
#pragma unroll
              for (int r = 0; r < RT; ++r)
                x[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c, qf[r][2 * y + e], x[r][t], 0,
                                                                 0, 0);
            }
          } else {
#pragma unroll
            for (int r = 0; r < RT; ++r)
              x[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kv),
                                                               qf[r][y], x[r][t], 0, 0, 0);
          }
        }
        if constexpr (E4M3) {
          const floatx4 ks = *reinterpret_cast<const floatx4*>(
              (S == 0 ? sks0 : sks1)[wave] + 16 * t + 4 * g);
#pragma unroll
          for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[r][t][e] *= ks[e];
        }
      }
      if (kb + KT - 1 > full || kb + KT > wend) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const int vis = min(lim[r], wend - 1) - kb - 4 * g;
#pragma unroll
          for (int t = 0; t < G::T16; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[r][t][e] = 16 * t + e > vis ? kNegInf : x[r][t][e];
        }
      }
      // Reference, weights, sums.
      uint32_t pk[RT][G::SUBS][4];
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        float top = x[r][0][0];
#pragma unroll
        for (int t = 0; t < G::T16; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) top = fmaxf(top, x[r][t][e]);
        float y, z;
        lane_pair<16>(top, y, z);
        top = fmaxf(y, z);
        lane_pair<32>(top, y, z);
        top = fmaxf(y, z) * a.c_abs;
        const bool up = top > mref[r] + kHeadroom;
        if (__builtin_amdgcn_ballot_w64(up)) {
          const float rs = up ? exp2_fast(mref[r] - top) : 1.f;  // 0 from -inf
          mref[r] = up ? top : mref[r];
          lsum[r] *= rs;
#pragma unroll
          for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) oacc[r][i][e] *= rs;
        }
        const float neg = mref[r] == kNegInf ? 0.f : -mref[r];
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < G::T16; ++t) {
          float p[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) p[e] = exp2_fast(fmaf(x[r][t][e], a.c_abs, neg));
          sum += (p[0] + p[1]) + (p[2] + p[3]);
          if constexpr (E4M3) {
            const floatx4 vsc = *reinterpret_cast<const floatx4*>(
                (S == 0 ? svs0 : svs1)[wave] + 16 * t + 4 * g);
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] *= vsc[e];
          }
          pk[r][t / 2][2 * (t % 2)] = pack_bf16x2(p[0], p[1]);
          pk[r][t / 2][2 * (t % 2) + 1] = pack_bf16x2(p[2], p[3]);
        }
        lsum[r] += sum;
      }
      // Values: the fragments of BATCH products are read while the ones before are multiplied.
      constexpr int BATCH = RT == 2 && !E4M3 ? 2 : 4, NB = DT / BATCH * G::SUBS;
      bf16x8_t vx[2][BATCH];
      int turn = vturn;
      asm volatile("" : "+v"(turn));  // (offsets formed here take no registers outside)
      auto fetch = [&](int n) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i)
          vx[n & 1][i] = value(vs, turn, n / (DT / BATCH) * 32 * G::ROWB,
                               n % (DT / BATCH) * BATCH + i);
      };
      fetch(0);
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        if (n + 1 < NB) fetch(n + 1);
        __builtin_amdgcn_sched_barrier(0);
        const int y = n / (DT / BATCH);
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
          bf16x8_t f = vx[n & 1][i];
          if constexpr (E4M3) {
            const u32x4_t c = __builtin_bit_cast(u32x4_t, f);
            f = widen(c[0], c[1]);
          }
          const int d = n % (DT / BATCH) * BATCH + i;
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            const u32x4_t pw = {pk[r][y][0], pk[r][y][1], pk[r][y][2], pk[r][y][3]};
            oacc[r][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                f, __builtin_bit_cast(bf16x8_t, pw), oacc[r][d], 0, 0, 0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    constexpr std::integral_constant<int, 0> s0{};
    constexpr std::integral_constant<int, 1> s1{};
    // (A stage is loaded again only when its reads have returned.)
    auto reads_done = [] { __builtin_amdgcn_s_waitcnt(0xc07f /* lgkmcnt(0) */); };
    check_entries();
    load(s0, j0);
    // A query that is not finite: zero here, its row NaN where it sees a key.
    bool poison[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      unsigned most = 0;
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        const u32x4_t v = __builtin_bit_cast(u32x4_t, qf[t][x]) ^ a.qflip;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          most = max(most, v[e] & 0x7fffu);
          most = max(most, v[e] >> 16 & 0x7fffu);
        }
        qf[t][x] = __builtin_bit_cast(bf16x8_t, v);
      }
      // (bit patterns of bf16 magnitudes order as floats)
      float y, z;
      lane_pair<16>(__uint_as_float(most), y, z);
      most = max(__float_as_uint(y), __float_as_uint(z));
      lane_pair<32>(__uint_as_float(most), y, z);
      most = max(__float_as_uint(y), __float_as_uint(z));
      const bool bad = most >= 0x7f80u;
      poison[t] = bad && lim[t] >= 0;
      const bool drop = bad || 16 * t + l16 >= nrows;
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        u32x4_t v = __builtin_bit_cast(u32x4_t, qf[t][x]);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = drop ? 0u : v[e];
        qf[t][x] = __builtin_bit_cast(bf16x8_t, v);
      }
    }
    for (int j = j0; j < j1; j += 2) {
      load(s1, j + 1);
      compute(s0, j);
      reads_done();
      load(s0, j + 2);
      compute(s1, j + 1);
      reads_done();
    }
    wait_loads<0>();

    // The waves' states meet in LDS: values in a wave's own stages, each lane's at its place.
    static_assert(ROWS * D * 4 <= 2 * kStageBytes && RT * DT * 1024 == ROWS * D * 4, "they fit");
    constexpr int HALF = kStageBytes / 1024;  // fragments of a stage
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      float y, z;
      lane_pair<16>(lsum[t], y, z);
      float l = y + z;
      lane_pair<32>(l, y, z);
      l = y + z;
      if (poison[t] || lim[t] >= bad_from) l = __builtin_nanf("");
      if (g == 0) {
        sm[wave][16 * t + l16] = mref[t];
        sl[wave][16 * t + l16] = l;
      }
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        const int f = t * DT + i;
        reinterpret_cast<floatx4*>(f < HALF ? sv0[wave] : sv1[wave])[f % HALF * 64 + lane] =
            oacc[t][i];
      }
    }
    __syncthreads();
    const bool whole = u == first && u_next == first + units;
    const size_t slot = ((size_t)head * a.W + w) * 2 + (u == first ? 1 : 0);
    const __amdgpu_buffer_rsrc_t acc_rs =
        __builtin_amdgcn_make_buffer_rsrc(a.ws_acc, (short)0, -1, 0x00020000);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int r = 16 * t + l16;
      float M = sm[0][r];
#pragma unroll
      for (int x = 1; x < 4; ++x) M = fmaxf(M, sm[x][r]);
      const float ref = M == kNegInf ? 0.f : M;
      float wt[4], L = 0.f;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        wt[x] = exp2_fast(sm[x][r] - ref);
        L = fmaf(wt[x], sl[x][r], L);
      }
      const bool valid = r < nrows;
      const float inv = L == 0.f ? 0.f : 1.f / L;  // NaN stays NaN
#pragma unroll
      for (int c = 0; c < DT / 4; ++c) {
        const int i = 4 * c + wave;  // this wave's share of the row
        floatx4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int f = t * DT + i;
          const floatx4 z = reinterpret_cast<const floatx4*>(
              f < HALF ? sv0[x] : sv1[x])[f % HALF * 64 + lane];
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = fmaf(wt[x], z[e], y[e]);
        }
        if (!valid) continue;
        if (whole) {
          const u32x2_t p = {pack_bf16x2(y[0] * inv, y[1] * inv),
                             pack_bf16x2(y[2] * inv, y[3] * inv)};
          *reinterpret_cast<u32x2_t*>(a.o + orow[t] + 16 * i + 4 * g) = p;
        } else if (RT == 1 && a.counters != nullptr) {  // read by another workgroup of the launch
          __builtin_amdgcn_raw_buffer_store_b128(
              __builtin_bit_cast(u32x4_t, y), acc_rs,
              (int)(((unsigned)(slot * ROWS + r) * D + 16 * i + 4 * g) * 4), 0,
              16 /* device scope */);
        } else {
          *reinterpret_cast<floatx4*>(a.ws_acc + (slot * ROWS + r) * D + 16 * i + 4 * g) = y;
        }
      }
      if (!whole && valid && wave == 0 && g == 0) {
        store_dev(a.ws_m + slot * ROWS + r, M);
        store_dev(a.ws_l + slot * ROWS + r, L);
      }
    }
    // The sequence's first workgroup, and how many have keys of it.
    const int w0 = (unsigned)first / (unsigned)T;
    const int P = (unsigned)(first + units - 1) / (unsigned)T - w0 + 1;
    if (RT == 2 || a.counters == nullptr) {
      // The sequence's first part says where the others are.
      if (u == first && threadIdx.x == 0) a.parts[(size_t)b * a.heads + head] = make_int2(w0, P);
    } else if constexpr (RT == 1) if (!whole) {
      // The last part to arrive joins them, a wave a row.
      unsigned* const counter = a.counters + ((size_t)head * a.W + w0) * a.counter_stride;
      const unsigned ticket = arrival_ticket(counter);
      if (ticket >= (unsigned)(P - 1)) {
        for (int r = wave; r < nrows; r += 4) {
          const size_t slot0 = ((size_t)head * a.W + w0) * 2;
          Joined j = {{0.f, 0.f, 0.f, 0.f}, 0.f, 0.f};
          if (ticket == (unsigned)(P - 1))
            j = join_parts<D, D, 8, true>(a, 0, P, 0, [&](int p) {
              return (slot0 + 2 * p + (p == 0 ? 1 : 0)) * ROWS + r;
            });
          // (A counter that was not zero: NaN.)
          const float inv = ticket > (unsigned)(P - 1) ? __builtin_nanf("")
                            : j.L == 0.f               ? 0.f
                                                       : 1.f / j.L;
          const int rr = row0 + r;
          store_joined<D>(j, inv, a.o + ((size_t)(start + rr / a.G) * a.Hq +
                                         (size_t)hk * a.G + rr % a.G) * D);
        }
        if (ticket == (unsigned)(P - 1) && threadIdx.x == 0) reset_counter(counter);
      }
    }
    u = min(u_end, behind);
    __syncthreads();  // the stages may be loaded again
  }
}

// NT: cache policy of the loads of keys and values.
template <int D, bool E4M3, int RT, int NT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
void attn_paged_kernel(PagedParams a) {
  attend_pages<D, E4M3, RT, NT>(a);
}

// Joins the parts of a row that several workgroups share: a wave a row, or (WIDE) four waves for 32
// channels of it, each a quarter of the parts. Sequences from b0 on.
template <int D, int ROWS, bool WIDE>
__global__ __launch_bounds__(256) void paged_combine_kernel(PagedParams a, int tiles, int b0) {
  constexpr int CH = WIDE ? kWideChannels : D;  // channels of a wave
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int x = (int)(blockIdx.x % tiles);
  const int r = WIDE ? x / (D / CH) : x * 4 + wave, c0 = WIDE ? x % (D / CH) * CH : 0;
  const int head = (int)(blockIdx.x / tiles % a.heads);
  const int b = b0 + (int)(blockIdx.x / tiles / a.heads);
  const int mt = head % a.mtiles, hk = head / a.mtiles;
  const int2 part = a.parts[(size_t)b * a.heads + head];
  const int start = sequence_start(a.starts, b, a.B, a.T);
  const int n = min(max(sequence_start(a.starts, b + 1, a.B, a.T) - start, 0), a.T);
  const int row = mt * ROWS + r;
  // (Without rows in this tile nothing wrote `part`. All waves of a row end here, or none.)
  if (r >= ROWS || row >= min(n, a.max_queries) * a.G || part.y < 2) return;
  const int P = part.y;
  const size_t slot0 = ((size_t)head * a.W + part.x) * 2;
  Joined j = join_parts<D, CH, 8, false>(a, WIDE ? P * wave / 4 : 0, WIDE ? P * (wave + 1) / 4 : P,
                                         c0, [&](int p) {
    return (slot0 + 2 * p + (p == 0 ? 1 : 0)) * ROWS + r;
  });
  if constexpr (WIDE) {
    __shared__ float sx[4][CH], sm[4], sl[4];
    if (lane < CH / 4) *reinterpret_cast<floatx4*>(&sx[wave][4 * lane]) = j.x;
    if (lane == 0) {
      sm[wave] = j.M;
      sl[wave] = j.L;
    }
    __syncthreads();
    if (wave != 0) return;
    const float M = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
    const float ref = M == kNegInf ? 0.f : M;
    j = {{0.f, 0.f, 0.f, 0.f}, M, 0.f};
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const float wt = exp2_fast(sm[y] - ref);
      j.L = fmaf(wt, sl[y], j.L);
      if (lane < CH / 4)
#pragma unroll
        for (int e = 0; e < 4; ++e) j.x[e] = fmaf(wt, sx[y][4 * lane + e], j.x[e]);
    }
  }
  store_joined<CH>(
      j, j.L == 0.f ? 0.f : 1.f / j.L,
      a.o + ((size_t)(start + row / a.G) * a.Hq + (size_t)hk * a.G + row % a.G) * D + c0);
}

constexpr int kOnce = 2, kAgain = 0;  // non-temporal, cached

template <int D, bool E4M3, int RT, int NT>
hipError_t launch(const PagedParams& a, hipStream_t stream) {
  hipLaunchKernelGGL((attn_paged_kernel<D, E4M3, RT, NT>), dim3((unsigned)a.heads * a.W), dim3(256),
                     0, stream, a);
  hipError_t e = hipGetLastError();
  // (One workgroup for all of a head's keys cuts nothing.)
  if (e != hipSuccess || a.counters != nullptr || a.W == 1) return e;
  // A wave a row where the parts may be few; where there may be hundreds, four waves for every 32
  // channels of a row.
  const int rows = a.mtiles > 1 ? 16 * RT : a.rows;
  const bool wide = a.W > 128;
  const int tiles = wide ? rows * (D / kWideChannels) : (rows + 3) / 4;
  auto* const combine = wide ? paged_combine_kernel<D, 16 * RT, true>
                             : paged_combine_kernel<D, 16 * RT, false>;
  // Sequences of a launch. (W > 1 leaves at most 1024 heads of 8 tiles, or 16 of 128.)
  const int most = (int)(kMaxGroups / ((long long)a.heads * tiles));
  for (int b0 = 0; b0 < a.B && e == hipSuccess; b0 += most) {
    const dim3 grid((unsigned)std::min(most, a.B - b0) * a.heads * tiles);
    hipLaunchKernelGGL(combine, grid, dim3(256), 0, stream, a, tiles, b0);
    e = hipGetLastError();
  }
  return e;
}

template <int D, bool E4M3>
hipError_t launch_rt(const PagedParams& a, hipStream_t stream) {
  if (a.rt == 1) return launch<D, E4M3, 1, kOnce>(a, stream);
  // Several row tiles read the same keys, out of the L2 cache but for the first (8 sequences of 16
  // tokens of 64/8 heads of 128 over 8192 keys, non-temporal / cached 137 / 94 us; one row tile
  // reads them once, 64 sequences of one token of 32/8 heads of 64 over 4096 85 / 94).
  return a.mtiles == 1 ? launch<D, E4M3, 2, kOnce>(a, stream)
                       : launch<D, E4M3, 2, kAgain>(a, stream);
}

template <int D>
hipError_t launch_d(const PagedParams& a, bool e4m3, hipStream_t stream) {
  return e4m3 ? launch_rt<D, true>(a, stream) : launch_rt<D, false>(a, stream);
}

}  // namespace

hipError_t launch_attention_paged(const PagedParams& a, bool e4m3, hipStream_t stream) {
  return a.D == 128 ? launch_d<128>(a, e4m3, stream) : launch_d<64>(a, e4m3, stream);
}

}  // namespace ef
