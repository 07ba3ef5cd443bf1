// Host side of the long-context entry points of include/ef_attention.h: argument
// validation, launch shapes and workspace arithmetic.
#include <algorithm>
#include <cmath>

#include "ef_attention.h"
#include "ef_long.hpp"
#include "ef_device.hpp"
#include "host_checks.hpp"

namespace {

using namespace ef::host;

static_assert(ef::kMaxBlocks == EF_MAX_BLOCKS && ef::kMaxTopk == EF_MAX_TOPK,
              "the limits of the header are the kernels' ones");

// Blocks of a key axis, or -1 where block_size or their number is refused.
int num_blocks(int Skv, int block_size) {
  if (block_size != 64 && block_size != 128) return -1;
  const int nb = (int)(((long long)Skv + block_size - 1) / block_size);
  return nb <= ef::kMaxBlocks ? nb : -1;
}

// Most bytes of LDS a launch may ask for: any list of EF_MAX_BLOCKS scores fits.
constexpr int kLaunchLds = 64 * 1024;

// A launch holds fewer than 2^32 threads. Where a call may need more it is made in several,
// none of more than half of that.
constexpr long long kMaxThreads = (1LL << 32) - 1;
constexpr long long kLaunchThreads = 1LL << 31;

}  // namespace

extern "C" {

ef_status ef_block_summary(const void* k, const int* lengths, void* summary, int B, int Hkv,
                           int Skv, int D, int block_size, int new_keys, void* stream) {
  const Shape s{B, Hkv, Hkv, 1, Skv, D};
  const ef_status st = check_shape(s);
  if (st != EF_OK) return st;
  const int nb = num_blocks(Skv, block_size);
  if (nb < 0 || new_keys < 0) return EF_ERR_INVALID_BLOCKS;
  if (B == 0 || nb == 0) return EF_OK;
  if (k == nullptr || summary == nullptr) return EF_ERR_NULL_POINTER;
  if (misaligned(k) || misaligned(summary)) return EF_ERR_MISALIGNED;
  ef::SummaryParams a{};
  a.k = static_cast<const uint16_t*>(k);
  a.lengths = lengths;
  a.s = static_cast<uint16_t*>(summary);
  a.B = B; a.Hkv = Hkv; a.Skv = Skv; a.D = D;
  a.NB = nb;
  a.block = block_size;
  a.new_keys = new_keys;
  // The last new_keys keys lie in at most this many blocks.
  a.touched = new_keys == 0
                  ? nb
                  : (int)std::min<long long>(nb, ((long long)new_keys + block_size - 2) /
                                                         block_size + 1);
  return from_hip(ef::launch_block_summary(a, static_cast<hipStream_t>(stream)));
}

ef_status ef_block_select(const void* q, const void* summary, const int* lengths, int* blocks,
                          int B, int Hq, int Hkv, int Sq, int Skv, int D, int block_size,
                          int topk, int sink_blocks, int local_blocks, void* stream) {
  const Shape s{B, Hq, Hkv, Sq, Skv, D};
  const ef_status st = check_shape(s);
  if (st != EF_OK) return st;
  const int nb = num_blocks(Skv, block_size);
  if (nb < 0 || topk < 1 || topk > ef::kMaxTopk || sink_blocks < 0 || local_blocks < 1 ||
      (long long)sink_blocks + local_blocks > topk)
    return EF_ERR_INVALID_BLOCKS;
  if (s.rows() == 0) return EF_OK;
  if (q == nullptr || blocks == nullptr || (nb > 0 && summary == nullptr))
    return EF_ERR_NULL_POINTER;
  if (misaligned(q) || misaligned(summary) || misaligned(blocks)) return EF_ERR_MISALIGNED;
  ef::SelectParams a{};
  a.q = static_cast<const uint16_t*>(q);
  a.s = static_cast<const uint16_t*>(summary);
  a.lengths = lengths;
  a.out = blocks;
  a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.Sq = Sq; a.Skv = Skv; a.D = D;
  a.G = Hq / Hkv;
  a.NB = nb;
  a.shift = block_size == 64 ? 6 : 7;
  a.K = topk;
  a.sinks = sink_blocks;
  a.local = local_blocks;
  a.gp = 1;
  while (a.gp < a.G && a.gp < 16) a.gp *= 2;
  a.per = (a.G + 15) / 16;
  // Rows of four floats more than whole tiles: the rows of a tile's positions start in
  // different banks.
  a.stride = (nb + 15) / 16 * 16 + 4;
  // Positions per workgroup: four row tiles, which share the summaries' loads and norms,
  // where the LDS has room for the scores of at least three of them, there are positions
  // for more than one, the grid still fills the chip and scores are most of the work; else
  // one tile, with more workgroups on a compute unit for the choices, and fewer positions
  // where they do not fit. One / four tiles (us; 4096 queries of 8 kv heads of 128; G x
  // blocks): 4 x 1024 155 / 108, 8 x 256 171 / 117, 4 x 256 69 / 62, 4 x 128 57 / 56, 2 x 128
  // 43 / 46, 1 x 128 36 / 40; 546 of 2 x 32 heads of 64, 1 x 56 30 / 51. Few queries of 64
  // sequences of 8 kv heads of 128, G x blocks: 4 x 512, 1 of them 16.2 / 18.2, 5 26.3 / 21.8;
  // 4 x 1024, 4 of them [one tile] 29.7 / 31.3, 6 44.3 / 34.3; 2 x 512, 8 of them [one tile]
  // 20.5 / 22.0, 9 33.0 / 24.3.
  const long long heads = (long long)B * Hkv;
  const int row = a.stride * 4, tile = a.per > 1 ? 1 : 16 / a.gp;
  a.pos = std::min(std::min(tile, std::max(1, kLaunchLds / row)), Sq);
  const int wide = std::min(4 * tile, ef::kSelectLds / row);
  if (a.per == 1 && wide > 2 * tile && Sq > tile && a.gp * nb >= 512 &&
      heads * ((Sq + wide - 1) / wide) >= 512)
    a.pos = wide;
  // Eight waves share the blocks of a workgroup where the grid leaves room for them.
  a.waves = heads * ((Sq + a.pos - 1) / a.pos) <= 256 ? 8 : 4;
  const long long ptiles = ((long long)Sq + a.pos - 1) / a.pos;
  a.ptiles = (int)ptiles;
  // Sequences per launch.
  const int most = (int)std::min<long long>(B, kLaunchThreads / (64 * a.waves) / (Hkv * ptiles));
  if (most < 1) return EF_ERR_INVALID_SHAPE;
  for (int b = 0; b < B; b += most) {
    ef::SelectParams c = a;
    c.B = std::min(most, B - b);
    c.q += (size_t)b * Hq * Sq * D;
    c.s += (size_t)b * Hkv * nb * D;
    c.lengths = lengths == nullptr ? nullptr : lengths + b;
    c.out += (size_t)b * Hkv * Sq * topk;
    const ef_status ls = from_hip(ef::launch_block_select(c, static_cast<hipStream_t>(stream)));
    if (ls != EF_OK) return ls;
  }
  return EF_OK;
}

}  // extern "C"

namespace {

// A workspace of partial states: the arrival counters (a region of fixed place and size,
// as in every workspace of the library), then m, l [rows][P] and acc [rows][P][D].
struct StateLayout {
  size_t m_off, l_off, acc_off, bytes;
};

StateLayout state_layout(long long rows, long long P, int D) {
  StateLayout w;
  const size_t a = ef::ws_align256((size_t)(rows * P) * sizeof(float));
  w.m_off = ef::kCounterRegionBytes;
  w.l_off = w.m_off + a;
  w.acc_off = w.l_off + a;
  w.bytes = w.acc_off + (size_t)(rows * P) * D * sizeof(float);
  return w;
}

template <class Params>
void set_states(Params& a, const StateLayout& w, void* workspace) {
  char* ws = static_cast<char*>(workspace);
  a.ws_m = reinterpret_cast<float*>(ws + w.m_off);
  a.ws_l = reinterpret_cast<float*>(ws + w.l_off);
  a.ws_acc = reinterpret_cast<float*>(ws + w.acc_off);
}

template <class Params>
ef_status combine_states(const Params& a, long long rows, hipStream_t stream) {
  constexpr long long most = kLaunchThreads / 64;  // rows per launch, one wave each
  for (long long r = 0; r < rows; r += most) {
    ef::StateCombineParams c{};
    c.m = a.ws_m + r * a.P;
    c.l = a.ws_l + r * a.P;
    c.acc = a.ws_acc + r * a.P * a.D;
    c.o = a.o + r * a.D;
    c.rows = (int)std::min(most, rows - r);
    c.P = a.P;
    c.D = a.D;
    const ef_status st = from_hip(ef::launch_state_combine(c, stream));
    if (st != EF_OK) return st;
  }
  return EF_OK;
}

// Workgroups that fill the chip: two of the matrix-core kernels fit on a compute unit (with
// heads of 64 three do, but more parts mean more lists and states). 512 / 640 / 768 /
// 1024 (us): one token over 64 blocks, 16 sequences of 32/8 heads of 128 48 / 61 / 56 / 54, 8
// of them 29 / 40 / 37 / 36; 5 tokens over 24 blocks, 8 sequences of 64/8 heads of 64 29 /
// 28 / 27 / 36, one token of them 16.4 / 17.7 / 18.0 / 24.0.
constexpr long long kFillWgs = 512;

// Launch shape of attention over selected blocks. The rows of a kv head are cut into
// tiles of `bm`; where these are few, P workgroups share a tile's blocks.
//
// 128 rows share a staged tile between four waves where such tiles fill the chip
// twice; otherwise 64 do, whose lists' union is shorter. 64 / 128 rows (us; 16 blocks
// of 512, 32/8 heads of 128; lists of neighbours alike, then independent): 4096 queries
// 180 / 131, 2048 [512 workgroups of 128] 89 / 69 and 479 / 580, 1024 [256] 46.6 / 45.0
// and 251 / 378, 512 38.8 / 38.6 and 138 / 200.
//
// `fused`: the last of P workgroups to store a state combines its head's rows, where one
// round of its loads takes all states (4 rows of 128 or 8 of 64, 8 states of each), or two
// do and each part is one block; otherwise a second kernel does. Two launches cost the host
// 2 us more, which binds a loop of short calls (11.3 to 12.5 us a call); on the GPU the second
// one is worth two rounds. One launch / two, us a call of calls in a row, then of calls in a
// graph: one token of 32/8 heads of 128 over 8 blocks [P = 8] 9.3 / 11.5, 8.7 / 8.5; 8 sequences
// of it 11.7 / 12.3, 11.1 / 11.4; 16 over 64 [4] 50.2 / 50.6, 50.0 / 50.4; 64/8 heads of 64 over 8
// [8] 8.1 / 10.4, 7.7 / 8.5. Two rounds: one token over 16 blocks [16] 9.9 / 12.5, 9.6 / 8.6; 64/8
// heads of 128 over 8 [8] 10.6 / 11.8, 10.1 / 9.1; where parts have more blocks, 16 sequences of
// those over 16 [4] 21.1 / 20.2, 20.8 / 20.0. More: one token over 32, 64 blocks [32, 64] 11.8 /
// 11.8, 15.5 / 12.9 and 11.4 / 10.2, 15.3 / 12.4; four tokens over 4, 16 [4, 16] 12.8 / 11.9, 16.0
// / 11.8 and 12.5 / 9.4, 15.8 / 10.3.
struct BlocksPlan {
  int bm, mtiles, P;
  bool fused;
};

BlocksPlan blocks_plan(const Shape& s, int nb, int topk) {
  BlocksPlan p;
  const long long R = (long long)(s.Hq / s.Hkv) * s.Sq;
  p.bm = (long long)s.B * s.Hkv * (R / 128) >= kFillWgs ? 128 : 64;
  p.mtiles = (int)((R + p.bm - 1) / p.bm);
  const long long groups = (long long)s.B * s.Hkv * p.mtiles;
  const long long most = std::max(1, std::min(std::min(nb, topk), 64));
  p.P = (int)std::min(std::max(kFillWgs / std::max(groups, 1LL), 1LL), most);  // 1 for 128 rows
  const long long rounds = (R * s.D + ef::kSharedElems - 1) / ef::kSharedElems *
                           ((p.P + ef::kSharedParts - 1) / ef::kSharedParts);
  static_assert(kFillWgs / 2 <= ef::kCounterSlots, "a counter for every head whose P is 2 or more");
  p.fused = p.mtiles == 1 && (rounds == 1 || (rounds == 2 && p.P == std::min(nb, topk)));
  return p;
}

ef_status check_blocks(const Shape& s, int block_size, int topk) {
  const ef_status st = check_shape(s);
  if (st != EF_OK) return st;
  if (num_blocks(s.Skv, block_size) < 0 || topk < 1 || topk > ef::kMaxTopk)
    return EF_ERR_INVALID_BLOCKS;
  return s.rows() < (1LL << 31) ? EF_OK : EF_ERR_INVALID_SHAPE;
}

// Launch shape of attention over a shared prefix: see PrefixParams.
struct PrefixPlan {
  bool whole;
  int P1, T1, mt1, P2, T2, mt2, P;
  long long n_prefix, n_own;
};

constexpr int kPrefixRows = 128;  // rows per workgroup

// `tiles` tiles in at most `parts` parts: tiles per part.
int tiles_per_part(long long tiles, long long parts) {
  const long long p = std::max(parts, 1LL);
  return (int)((tiles + p - 1) / p);
}

PrefixPlan prefix_plan(const Shape& s, int Lp) {
  PrefixPlan p{};
  const long long R = (long long)(s.Hq / s.Hkv) * s.Sq, heads = (long long)s.B * s.Hkv;
  const long long np = (Lp + 63) / 64, no = ((long long)s.Skv + 63) / 64;
  p.mt1 = (int)((s.B * R + kPrefixRows - 1) / kPrefixRows);
  p.mt2 = (int)((R + kPrefixRows - 1) / kPrefixRows);
  // `whole` spares the states and their combine, which take a row about as long as 32
  // tiles do, but walks the prefix for the empty rows of its tiles too, and needs rows
  // for the chip (192 workgroups of the 512 that fit, 0.62 PFLOP/s, are where it begins to be
  // the shorter one). Split / whole (us; 32/8 heads of 128; sequences x tokens, prefix + 256 or
  // 1024 keys): 24 x 32 over 2048 62 / 49, over 16384 343 / 330; 16 x 32 over 2048 42 / 46,
  // over 16384 191 / 301; 64 x 64 over 2048 258 / 163; with half of the rows empty 64 x 16
  // over 2048 73 / 65, over 16384 392 / 485, 32 x 16 over 2048 42 / 45; 16 x 100 over 700
  // 70 / 39, over 9000 290 / 316.
  p.whole = np + no == 0 ||
            (heads * R >= 192LL * kPrefixRows &&
             (p.mt2 * (long long)kPrefixRows - R) * np <= 32 * R);
  if (p.whole) {
    p.P2 = p.P = 1;
    p.n_own = heads * p.mt2;
    return p;
  }
  // Workgroups of the prefix: one to a compute unit; half as many where the own keys have
  // most of the work, which then get three of four places; two where the prefix is nearly
  // all, long and read by one row tile. (With more row tiles two were not measured; one, at
  // one wave to a SIMD, leaves the matrix cores at 0.60 to 0.72 PFLOP/s: 24 x 16 tokens over
  // 16384 keys 173 us, 64 x 16 392.) 256 / 128 workgroups (us; 32/8 heads of
  // 128, own keys half of the capacity in the mean; the prefix's part of the tiles in
  // brackets): 64 sequences, 32768 + 2048 keys [0.33] 106 / 98, 16384 + 1024 [0.33] 57.7 /
  // 54.9, 32 of them [0.33] 41 / 35, 16 [0.5] 27.2 / 28.0, 8 [0.67] 19.6 / 26.1, 64 over
  // 32768 + 64 [0.94] 52 / 83. 256 / 512: 16 sequences, 64000 + 64 keys [31 tiles to each
  // of 256] 70 / 59, 32 of them 73 / 63, 16 over 16000 + 100 [8] 20.0 / 24.0.
  const long long w1 = np * s.Hkv * p.mt1, w2 = no * heads * p.mt2;
  const bool mostly = 5 * w1 >= 3 * (w1 + w2);
  const long long n1 = !mostly ? kFillWgs / 4
                       : p.mt1 == 1 && w1 >= 24 * (kFillWgs / 2) ? kFillWgs
                                                                 : kFillWgs / 2;
  if (np > 0) {
    p.T1 = tiles_per_part(np, n1 / (s.Hkv * (long long)p.mt1));
    p.P1 = (int)((np + p.T1 - 1) / p.T1);
    p.n_prefix = (long long)s.Hkv * p.mt1 * p.P1;
  }
  if (no > 0) {
    p.T2 = tiles_per_part(no, (kFillWgs - p.n_prefix) / (heads * p.mt2));
    p.P2 = (int)((no + p.T2 - 1) / p.T2);
    p.n_own = heads * p.mt2 * p.P2;
  }
  p.P = p.P1 + p.P2;
  return p;
}

ef_status check_prefix(const Shape& s, int Lp) {
  const ef_status st = check_shape(s);
  if (st != EF_OK) return st;
  if (Lp < 0 || (long long)Lp * s.D >= (1LL << 31)) return EF_ERR_INVALID_SHAPE;
  // Rows are counted over the whole batch.
  return s.rows() < (1LL << 31) ? EF_OK : EF_ERR_INVALID_SHAPE;
}

}  // namespace

extern "C" {

size_t ef_attention_blocks_workspace_size(int B, int Hq, int Hkv, int Sq, int Skv, int D,
                                          int block_size, int topk) {
  const Shape s{B, Hq, Hkv, Sq, Skv, D};
  if (check_blocks(s, block_size, topk) != EF_OK || s.rows() == 0) return 0;
  const BlocksPlan p = blocks_plan(s, num_blocks(Skv, block_size), topk);
  return p.P == 1 ? 0 : state_layout(s.rows(), p.P, D).bytes;
}

ef_status ef_attention_blocks(const void* q, const void* k, const void* v, const int* blocks,
                              const int* lengths, void* o, int B, int Hq, int Hkv, int Sq,
                              int Skv, int D, float scale, int block_size, int topk,
                              void* workspace, size_t workspace_bytes, void* stream) {
  const Shape s{B, Hq, Hkv, Sq, Skv, D};
  ef_status st = check_blocks(s, block_size, topk);
  if (st != EF_OK) return st;
  st = check_io(s, q, k, v, o, scale);
  if (st != EF_OK) return st;
  if (s.rows() == 0) return EF_OK;
  if (blocks == nullptr) return EF_ERR_NULL_POINTER;
  if (misaligned(blocks)) return EF_ERR_MISALIGNED;
  const BlocksPlan p = blocks_plan(s, num_blocks(Skv, block_size), topk);
  ef::BlocksParams a{};
  if (p.P > 1) {
    const StateLayout w = state_layout(s.rows(), p.P, D);
    if (workspace == nullptr || workspace_bytes < w.bytes) return EF_ERR_WORKSPACE_TOO_SMALL;
    if (misaligned(workspace)) return EF_ERR_MISALIGNED;
    set_states(a, w, workspace);
    a.counters = p.fused ? static_cast<unsigned*>(workspace) : nullptr;
  }
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.blocks = blocks;
  a.lengths = lengths;
  a.o = static_cast<uint16_t*>(o);
  a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.Sq = Sq; a.Skv = Skv; a.D = D;
  a.G = Hq / Hkv;
  a.R = a.G * Sq;
  a.NB = num_blocks(Skv, block_size);
  a.shift = block_size == 64 ? 6 : 7;
  a.K = topk;
  a.P = p.P;
  a.bm = p.bm;
  a.mtiles = p.mtiles;
  a.c_abs = std::fabs(scale) * ef::kLog2e;
  a.qflip = scale < 0.f ? 0x80008000u : 0u;
  if ((long long)B * Hkv * p.mtiles * p.P * 2 * p.bm > kMaxThreads) return EF_ERR_INVALID_SHAPE;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  st = from_hip(ef::launch_attention_blocks(a, hs));
  return st != EF_OK || p.P == 1 || p.fused ? st : combine_states(a, s.rows(), hs);
}

size_t ef_attention_shared_prefix_workspace_size(int B, int Hq, int Hkv, int Sq, int Lp, int Skv,
                                                 int D) {
  const Shape s{B, Hq, Hkv, Sq, Skv, D};
  if (check_prefix(s, Lp) != EF_OK || s.rows() == 0) return 0;
  const PrefixPlan p = prefix_plan(s, Lp);
  return p.P == 1 ? 0 : state_layout(s.rows(), p.P, D).bytes;
}

ef_status ef_attention_shared_prefix(const void* q, const void* k_prefix, const void* v_prefix,
                                     const void* k, const void* v, const int* lengths, void* o,
                                     int B, int Hq, int Hkv, int Sq, int Lp, int Skv, int D,
                                     float scale, int causal, void* workspace,
                                     size_t workspace_bytes, void* stream) {
  const Shape s{B, Hq, Hkv, Sq, Skv, D};
  ef_status st = check_prefix(s, Lp);
  if (st != EF_OK) return st;
  st = check_io(s, q, k, v, o, scale);
  if (st != EF_OK) return st;
  if (s.rows() == 0) return EF_OK;
  if (Lp > 0 && (k_prefix == nullptr || v_prefix == nullptr)) return EF_ERR_NULL_POINTER;
  if (misaligned(k_prefix) || misaligned(v_prefix)) return EF_ERR_MISALIGNED;
  const PrefixPlan p = prefix_plan(s, Lp);
  ef::PrefixParams a{};
  if (p.P > 1) {
    const StateLayout w = state_layout(s.rows(), p.P, D);
    if (workspace == nullptr || workspace_bytes < w.bytes) return EF_ERR_WORKSPACE_TOO_SMALL;
    if (misaligned(workspace)) return EF_ERR_MISALIGNED;
    set_states(a, w, workspace);
  }
  a.q = static_cast<const uint16_t*>(q);
  a.kp = static_cast<const uint16_t*>(k_prefix);
  a.vp = static_cast<const uint16_t*>(v_prefix);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.lengths = lengths;
  a.o = static_cast<uint16_t*>(o);
  a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.Sq = Sq; a.Skv = Skv; a.Lp = Lp; a.D = D;
  a.G = Hq / Hkv;
  a.R = a.G * Sq;
  a.causal = causal ? 1 : 0;
  a.whole = p.whole ? 1 : 0;
  a.P1 = p.P1; a.T1 = p.T1; a.mt1 = p.mt1;
  a.P2 = p.P2; a.T2 = p.T2; a.mt2 = p.mt2;
  a.P = p.P;
  if ((p.n_prefix + p.n_own) * 2 * kPrefixRows > kMaxThreads) return EF_ERR_INVALID_SHAPE;
  a.n_prefix = (unsigned)p.n_prefix;
  a.n_own = (unsigned)p.n_own;
  a.c_abs = std::fabs(scale) * ef::kLog2e;
  a.qflip = scale < 0.f ? 0x80008000u : 0u;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  st = from_hip(ef::launch_attention_prefix(a, hs));
  return st != EF_OK || p.P == 1 ? st : combine_states(a, s.rows(), hs);
}

}  // extern "C"
