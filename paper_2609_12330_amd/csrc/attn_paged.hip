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
// Work: the keys of all sequences, in steps of 64, make one list for each kv head (and row
// tile), which W workgroups cut into equal runs, whatever the lengths. A run holds the end of
// one sequence, whole ones, and the beginning of another; what is cut leaves a state in the
// workspace (two slots a workgroup), and a second kernel joins the states of a row.
#include "ef_device.hpp"
#include "ef_serve.hpp"
#include "group_combine.hpp"
#include "wave_ops.hpp"

namespace ef {

namespace {

constexpr int kUnit = 64;             // keys of a unit of work
constexpr float kHeadroom = 8.f;      // base-2 headroom before the reference moves
constexpr int kStageBytes = 8192;     // keys, and values, of a wave's step

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
  int units;            // units of work of its rows in this row tile
  int scan;             // units up to and with it, from sequence `base` on
  __device__ __forceinline__ void load(const PagedParams& a, int from, int row0, int rows) {
    base = from;
    const int b = from + (int)(threadIdx.x & 63);
    start = n = len = units = 0;
    if (b < a.B) {
      start = sequence_start(a.starts, b, a.B, a.T);
      n = min(max(sequence_start(a.starts, b + 1, a.B, a.T) - start, 0), a.T);
      len = (int)min((long long)max(a.lengths[b], 0), (long long)a.c.width << a.c.shift);
      if (row0 < min(n, a.max_queries) * a.G) units = max((last_key(a, row0, rows) + kUnit) / kUnit, 1);
    }
    scan = wave_scan(units);
  }
  // Last key that any of the tile's rows sees (-1: none).
  __device__ __forceinline__ int last_key(const PagedParams& a, int row0, int rows) const {
    const int top = min(row0 + rows, min(n, a.max_queries) * a.G) - 1;
    return max(top / a.G + len - n, -1);
  }
};

template <int D, bool E4M3, int RT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
void attn_paged_kernel(PagedParams a) {
  using G = Geo<D, E4M3>;
  constexpr int ROWS = 16 * RT, KT = G::KT, DT = G::DT;
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
  __shared__ __align__(16) float sks[2][4][KT], svs[2][4][KT];  // scales of keys and values
  __shared__ float sm[4][ROWS], sl[4][ROWS];

  // This workgroup's run of the list.
  Sequences s;
  s.load(a, 0, row0, ROWS);
  int total = __builtin_amdgcn_readlane(s.scan, 63);
  for (int b = 64; b < a.B; b += 64) {
    s.load(a, b, row0, ROWS);
    total += __builtin_amdgcn_readlane(s.scan, 63);
  }
  constexpr int LEAST = 4 * KT / kUnit;  // a step of each wave
  const int T = max((int)(((long long)total + a.W - 1) / a.W), LEAST);
  int u = (int)min((long long)w * T, (long long)total);
  const int u_end = (int)min((long long)u + T, (long long)total);
  if (u >= u_end) return;
  // Its first sequence.
  int before = 0;  // units in front of the sequences of `s`
  if (a.B > 64) s.load(a, 0, row0, ROWS);
  auto skip = [&] {
    while (s.base + 64 < a.B && before + __builtin_amdgcn_readlane(s.scan, 63) <= u) {
      before += __builtin_amdgcn_readlane(s.scan, 63);
      s.load(a, s.base + 64, row0, ROWS);
    }
  };

  while (u < u_end) {
    skip();
    const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(before + s.scan > u));
    const int b = s.base + at;
    const int units = __builtin_amdgcn_readlane(s.units, at);
    const int first = before + __builtin_amdgcn_readlane(s.scan, at) - units;  // its first unit
    const int len = __builtin_amdgcn_readlane(s.len, at);
    const int n = __builtin_amdgcn_readlane(s.n, at);
    const int start = __builtin_amdgcn_readlane(s.start, at);
    const int nrows = min(ROWS, min(n, a.max_queries) * a.G - row0);
    const int end_seen = (row0 + nrows - 1) / a.G + len - n + 1;  // keys any row sees
    const int k0 = (u - first) * kUnit;
    const int u_next = min(u_end, first + units);
    const int k1 = min((u_next - first) * kUnit, end_seen);

    // Rows: queries, the last key they see.
    bf16x8_t qf[RT][D / 32];
    int lim[RT];
    size_t orow[RT];
    bool poison[RT];
    int full = 0x7fffffff;  // last key that every row sees
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int r = row0 + 16 * t + l16;
      const bool valid = 16 * t + l16 < nrows;
      const int i = valid ? r / a.G : 0, hq = valid ? r % a.G : 0;
      lim[t] = valid ? i + len - n : -1;
      full = min(full, valid ? lim[t] : full);
      orow[t] = ((size_t)(start + i) * a.Hq + (size_t)hk * a.G + hq) * D;
      unsigned most = 0;
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        // Element order of an 8-bit key's 16-byte load: two steps' operands side by side.
        const int d = E4M3 ? 64 * (x / 2) + 16 * g + 8 * (x % 2) : 32 * x + 8 * g;
        u32x4_t v = {0u, 0u, 0u, 0u};
        if (valid) v = *reinterpret_cast<const u32x4_t*>(a.q + orow[t] + d) ^ a.qflip;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          most = max(most, v[e] & 0x7fffu);
          most = max(most, v[e] >> 16 & 0x7fffu);
        }
        qf[t][x] = __builtin_bit_cast(bf16x8_t, v);
      }
      // A query that is not finite: zero here, its row NaN where it sees a key.
      most = max(most, (unsigned)__shfl_xor((int)most, 16, 64));
      most = max(most, (unsigned)__shfl_xor((int)most, 32, 64));
      const bool bad = most >= 0x7f80u;
      poison[t] = bad && lim[t] >= 0;
      if (bad) {
        const u32x4_t zero = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int x = 0; x < D / 32; ++x) qf[t][x] = __builtin_bit_cast(bf16x8_t, zero);
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

    // This wave's steps.
    const int steps = k1 > k0 ? (k1 - k0 + KT - 1) / KT : 0;
    const int j0 = steps * wave / 4, j1 = steps * (wave + 1) / 4;
    int wend = min(k1, k0 + j1 * KT);  // keys it may read
    int bad_from = 0x7fffffff;         // first key of a page that is none
    int pv = 0, p0 = -0x10000000;      // table entries p0 .. p0 + 63, one to a lane
    const int* const table = a.c.table + (size_t)b * a.c.width;
    const int page_mask = (1 << a.c.shift) - 1;

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
        p0 = kb >> a.c.shift;
        const int last = (wend - 1) >> a.c.shift;
        const bool used = p0 + lane <= last;
        pv = used ? table[p0 + lane] : 0;
        const auto none = __builtin_amdgcn_ballot_w64(used && (unsigned)pv >= (unsigned)a.c.pages);
        if (none) {  // the walk ends in front of it
          bad_from = (p0 + __builtin_ctzll(none)) << a.c.shift;
          wend = min(wend, bad_from);
        }
      }
      if (kb >= wend) return;
      char* const vs = S == 0 ? sv0[wave] : sv1[wave];
#pragma unroll
      for (int t = 0; t < G::T16; ++t) {
        // Rows past the end repeat the last one (masked later).
        const int key = min(kb + 16 * t, (wend - 1) & ~15);
        const int left = wend - 1 - key;
        const size_t cell = cell_of(key);
        const char* const kp = a.c.k + cell * G::ROWB;
        const unsigned off = (unsigned)(min(l16, left) * G::ROWB + g * 16);
#pragma unroll
        for (int x = 0; x < G::KL; ++x)
          kx[S][t * G::KL + x] = __builtin_nontemporal_load(
              reinterpret_cast<const u32x4_t*>(kp + off + 64 * x));
      }
#pragma unroll
      for (int t = 0; t < G::T16; ++t) {
        const int key = min(kb + 16 * t, (wend - 1) & ~15);
        const int left = wend - 1 - key;
        const size_t cell = cell_of(key);
        const char* const vp = a.c.v + cell * G::ROWB;
        constexpr int N = 16 / G::RPI;  // loads of 16 rows
#pragma unroll
        for (int x = 0; x < N; ++x) {
          const int r = x * G::RPI + lane / G::KCH;
          const unsigned off =
              (unsigned)(min(r, left) * G::ROWB + ((lane % G::KCH) ^ G::swz(r)) * 16);
          __builtin_amdgcn_global_load_lds(vp + off, EF_LDS(void, vs + (t * N + x) * 1024), 16, 0,
                                           2 /* non-temporal */);
        }
      }
      if constexpr (E4M3) {
#pragma unroll
        for (int x = 0; x < KT / 64; ++x) {
          const int key = min(kb + 64 * x + lane, wend - 1);
          const int page = __shfl(pv, (key >> a.c.shift) - p0, 64);
          const size_t cell = (((size_t)(unsigned)page * a.Hkv + hk) << a.c.shift) +
                              (unsigned)(key & page_mask);
          __builtin_amdgcn_global_load_lds(a.c.k_scale + cell, EF_LDS(void, &sks[S][wave][64 * x]),
                                           4, 0, 0);
          __builtin_amdgcn_global_load_lds(a.c.v_scale + cell, EF_LDS(void, &svs[S][wave][64 * x]),
                                           4, 0, 0);
        }
      }
    };
    // Offsets of this lane's transposing reads of values.
    int vread[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) {
      if constexpr (E4M3) {
        const int r8 = l16 >> 1, r = 16 * (r8 >> 2) + 4 * g + (r8 & 3);
        vread[i] = r * G::ROWB + ((i ^ G::swz(r)) * 16) + 8 * (l16 & 1);
      } else {
        const int r = 4 * g + (l16 >> 2);
        vread[i] = r * G::ROWB + (((2 * i + ((l16 & 3) >> 1)) ^ G::swz(r)) * 16) + 8 * (l16 & 1);
      }
    }
    auto compute = [&](auto stage, int j) {
      constexpr int S = decltype(stage)::value;
      const int kb = k0 + j * KT;
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
              u32x4_t c;
#pragma unroll
              for (int f = 0; f < 2; ++f) {
                c[2 * f] = __builtin_bit_cast(
                    uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(kv[2 * e + f], 1.f, false));
                c[2 * f + 1] = __builtin_bit_cast(
                    uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(kv[2 * e + f], 1.f, true));
              }
#pragma unroll
              for (int r = 0; r < RT; ++r)
                x[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    __builtin_bit_cast(bf16x8_t, c), qf[r][2 * y + e], x[r][t], 0, 0, 0);
            }
          } else {
#pragma unroll
            for (int r = 0; r < RT; ++r)
              x[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kv),
                                                               qf[r][y], x[r][t], 0, 0, 0);
          }
        }
        if constexpr (E4M3) {
          const floatx4 ks = *reinterpret_cast<const floatx4*>(&sks[S][wave][16 * t + 4 * g]);
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
            const floatx4 vsc = *reinterpret_cast<const floatx4*>(&svs[S][wave][16 * t + 4 * g]);
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] *= vsc[e];
          }
          pk[r][t / 2][2 * (t % 2)] = pack_bf16x2(p[0], p[1]);
          pk[r][t / 2][2 * (t % 2) + 1] = pack_bf16x2(p[2], p[3]);
        }
        lsum[r] += sum;
      }
      // Values.
#pragma unroll
      for (int y = 0; y < G::SUBS; ++y)
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          const char* const p = vs + vread[i] + 32 * y * G::ROWB;
          bf16x8_t vx;
          if constexpr (E4M3) {
            const v2i c = __builtin_amdgcn_ds_read_tr8_b64_v2i32(EF_LDS(v2i, p));
            u32x4_t f;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              f[2 * e] = __builtin_bit_cast(
                  uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)c[e], 1.f, false));
              f[2 * e + 1] = __builtin_bit_cast(
                  uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)c[e], 1.f, true));
            }
            vx = __builtin_bit_cast(bf16x8_t, f);
          } else {
            const bf16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(EF_LDS(bf16x4_t, p));
            const bf16x4_t hi =
                __builtin_amdgcn_ds_read_tr16_b64_v4bf16(EF_LDS(bf16x4_t, p + 16 * G::ROWB));
            vx = bf16x8_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
          }
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            const u32x4_t pw = {pk[r][y][0], pk[r][y][1], pk[r][y][2], pk[r][y][3]};
            oacc[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                vx, __builtin_bit_cast(bf16x8_t, pw), oacc[r][i], 0, 0, 0);
          }
        }
    };
    constexpr std::integral_constant<int, 0> s0{};
    constexpr std::integral_constant<int, 1> s1{};
    // (A stage is loaded again only when its reads have returned.)
    auto reads_done = [] { __builtin_amdgcn_s_waitcnt(0xc07f /* lgkmcnt(0) */); };
    if (j0 < j1) load(s0, j0);
    for (int j = j0; j < j1; j += 2) {
      if (j + 1 < j1) load(s1, j + 1);
      compute(s0, j);
      reads_done();
      if (j + 2 < j1) load(s0, j + 2);
      if (j + 1 < j1) compute(s1, j + 1);
      reads_done();
    }

    // The waves' states meet in LDS, each lane's values at its own place.
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      float l = lsum[t];
      l += shfl_xor(l, 16);
      l += shfl_xor(l, 32);
      if (poison[t] || lim[t] >= bad_from) l = __builtin_nanf("");
      if (g == 0) {
        sm[wave][16 * t + l16] = mref[t];
        sl[wave][16 * t + l16] = l;
      }
    }
    __syncthreads();  // (all reads of values are done too)
    floatx4* const so = reinterpret_cast<floatx4*>(wave < 2 ? sv0 : sv1) + (wave & 1) * (ROWS * D / 4);
    static_assert(2 * ROWS * D * 4 <= 4 * kStageBytes, "two waves' values in a stage");
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int i = 0; i < DT; ++i) so[(t * DT + i) * 64 + lane] = oacc[t][i];
    __syncthreads();
    const bool whole = u == first && u_next == first + units;
    const size_t slot = ((size_t)head * a.W + w) * 2 + (u == first ? 1 : 0);
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
          const floatx4 z = reinterpret_cast<const floatx4*>(x < 2 ? sv0 : sv1)[(
              (x & 1) * (ROWS * D / 4)) + (t * DT + i) * 64 + lane];
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = fmaf(wt[x], z[e], y[e]);
        }
        if (!valid) continue;
        if (whole) {
          const u32x2_t p = {pack_bf16x2(y[0] * inv, y[1] * inv),
                             pack_bf16x2(y[2] * inv, y[3] * inv)};
          *reinterpret_cast<u32x2_t*>(a.o + orow[t] + 16 * i + 4 * g) = p;
        } else {
          *reinterpret_cast<floatx4*>(a.ws_acc + (slot * ROWS + r) * D + 16 * i + 4 * g) = y;
        }
      }
      if (!whole && valid && wave == 0 && g == 0) {
        a.ws_m[slot * ROWS + r] = M;
        a.ws_l[slot * ROWS + r] = L;
      }
    }
    // The sequence's first part says where the others are.
    if (u == first && threadIdx.x == 0) {
      const int last = (first + units - 1) / T;
      a.parts[(size_t)b * a.heads + head] = make_int2(w, last - w + 1);
    }
    u = u_next;
    __syncthreads();  // the stages may be loaded again
  }
}

// Joins the parts of a row that several workgroups share: one wave a row, D / 4 lanes a state.
template <int D, int ROWS>
__global__ __launch_bounds__(256) void paged_combine_kernel(PagedParams a) {
  constexpr int LPS = D / 4, SPL = 64 / LPS, BATCH = 8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  constexpr int WGS = ROWS / 4;  // workgroups of a sequence's row tile
  const int r = (int)(blockIdx.x % WGS) * 4 + wave;
  const int head = (int)(blockIdx.x / WGS % a.heads);
  const int b = (int)(blockIdx.x / WGS / a.heads);
  const int mt = head % a.mtiles, hk = head / a.mtiles;
  const int start = sequence_start(a.starts, b, a.B, a.T);
  const int n = min(max(sequence_start(a.starts, b + 1, a.B, a.T) - start, 0), a.T);
  const int row = mt * ROWS + r;
  if (row >= min(n, a.max_queries) * a.G) return;
  const int2 part = a.parts[(size_t)b * a.heads + head];
  const int w0 = part.x, P = part.y;
  if (P < 2) return;
  auto state = [&](int p) {  // row of part p
    return ((((size_t)head * a.W + w0 + p) * 2 + (p == 0 ? 1 : 0)) * ROWS + r);
  };
  const int grp = lane / LPS, ch = lane % LPS;
  float M = kNegInf, L = 0.f;
  floatx4 x = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < P; p0 += 64) {
    const int count = min(P - p0, 64);
    const bool have = lane < count;
    const float m = have ? a.ws_m[state(p0 + lane)] : kNegInf;
    const float l = have ? a.ws_l[state(p0 + lane)] : 0.f;
    const float top = fmaxf(M, wave_max(m));
    const float ref = top == kNegInf ? 0.f : top;
    const float wt = exp2_fast(m - ref);  // base-2 units
    const float old = exp2_fast(M - ref);
    L = L * old + wave_sum(wt * l);
    M = top;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] *= old;
    for (int j = 0; j < count; j += BATCH * SPL) {
      floatx4 y[BATCH];
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int q = min(j + i * SPL + grp, count - 1);
        y[i] = *reinterpret_cast<const floatx4*>(a.ws_acc + state(p0 + q) * D + 4 * ch);
      }
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int q = j + i * SPL + grp;
        const float wq = __shfl(wt, min(q, 63), 64);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = q < count ? fmaf(wq, y[i][e], x[e]) : x[e];
      }
    }
  }
#pragma unroll
  for (int off = LPS; off < 64; off *= 2)
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += shfl_xor(x[e], off);
  if (grp != 0) return;
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const size_t orow =
      ((size_t)(start + row / a.G) * a.Hq + (size_t)hk * a.G + row % a.G) * D;
  const u32x2_t o = {pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv)};
  *reinterpret_cast<u32x2_t*>(a.o + orow + 4 * ch) = o;
}

template <int D, bool E4M3, int RT>
hipError_t launch(const PagedParams& a, hipStream_t stream) {
  hipLaunchKernelGGL((attn_paged_kernel<D, E4M3, RT>), dim3((unsigned)a.heads * a.W), dim3(256), 0,
                     stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.counters != nullptr) return e;
  const dim3 grid((unsigned)a.B * a.heads * (16 * RT / 4));
  hipLaunchKernelGGL((paged_combine_kernel<D, 16 * RT>), grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

template <int D, bool E4M3>
hipError_t launch_rt(const PagedParams& a, hipStream_t stream) {
  return a.rt == 1 ? launch<D, E4M3, 1>(a, stream) : launch<D, E4M3, 2>(a, stream);
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
