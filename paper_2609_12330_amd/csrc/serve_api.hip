// Host side of the serving entry points of include/ef_attention.h: argument validation,
// launch shapes and workspace arithmetic.
#include <algorithm>
#include <cmath>

#include "ef_attention.h"
#include "ef_device.hpp"
#include "ef_serve.hpp"
#include "host_checks.hpp"

namespace {

using namespace ef::host;

using ef::kMaxGroups;

bool misaligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

ef_status check_heads(int T, int B, int Hq, int Hkv, int D) {
  if (T < 0 || B < 0 || Hq < 1 || Hkv < 1) return EF_ERR_INVALID_SHAPE;
  if (Hq % Hkv != 0) return EF_ERR_GQA_RATIO;
  if (D != 64 && D != 128) return EF_ERR_UNSUPPORTED_HEAD_DIM;
  // Rows of a token or a kv head and byte offsets inside a 64-row tile stay below 2^31.
  if (Hkv > kMaxGridYZ || Hq > (1 << 30) || B > (1 << 30) || (long long)T * (Hq / Hkv) >= (1LL << 31) - 128)
    return EF_ERR_INVALID_SHAPE;
  return EF_OK;
}

// With starts = NULL every sequence has T / B tokens.
bool uneven(const int* starts, int T, int B) { return starts == nullptr && T % B != 0; }

ef_status check_pages(int pages, int page, int width, int format) {
  if (pages < 1 || width < 0 || (format != EF_CACHE_BF16 && format != EF_CACHE_E4M3) ||
      (page != 16 && page != 32 && page != 64 && page != 128 && page != 256) ||
      (long long)width * page >= (1LL << 31) - 4096)  // (steps past the end count on)
    return EF_ERR_INVALID_PAGES;
  return EF_OK;
}

ef_status check_rope(int rot, int D, double amplitude) {
  return rot >= 16 && rot <= D && rot % 16 == 0 && std::isfinite(amplitude)
             ? EF_OK
             : EF_ERR_INVALID_ROPE;
}

ef_status set_pages(ef::PagesParams& c, const void* k, const void* v, const float* ks,
                    const float* vs, const int* table, int pages, int page, int width,
                    int format) {
  if (k == nullptr || v == nullptr || (width > 0 && table == nullptr)) return EF_ERR_NULL_POINTER;
  if (format == EF_CACHE_E4M3 && (ks == nullptr || vs == nullptr)) return EF_ERR_NULL_POINTER;
  if (misaligned(k) || misaligned(v) || misaligned4(table)) return EF_ERR_MISALIGNED;
  if (format == EF_CACHE_E4M3 && (misaligned(ks) || misaligned(vs))) return EF_ERR_MISALIGNED;
  c.k = static_cast<char*>(const_cast<void*>(k));
  c.v = static_cast<char*>(const_cast<void*>(v));
  c.k_scale = const_cast<float*>(ks);
  c.v_scale = const_cast<float*>(vs);
  c.table = table;
  c.pages = pages;
  c.width = width;
  c.shift = 4;
  while (1 << c.shift < page) ++c.shift;
  return EF_OK;
}

// What the eight L2 caches hold: larger outputs stream past them (11000 tokens of 32 heads of 128
// rotated 35.2 -> 32.9 us).
constexpr long long kCacheBytes = 32LL << 20;

// Tokens to a workgroup, and workgroups to these tokens' rows. Cosines and sines are formed once
// a workgroup, so it takes tokens for up to three rounds of its lanes where that leaves a thousand
// workgroups, and one token with fewer rows each where there are few.
ef_status run_rows(ef::RowsParams& a, bool e4m3, void* stream) {
  const int rows = a.Hq + 2 * a.Hkv, round = 256 / (a.D / 16);
  a.per = 1;
  while (a.per < 16 && 2LL * a.per * rows <= 3 * round && a.T / (2 * a.per) >= 1024) a.per *= 2;
  const int rounds = (a.per * rows + round - 1) / round;
  a.blocks = (int)std::min<long long>(rounds, std::max<long long>(1, 1024 / std::max(a.T, 1)));
  if (((long long)a.T + a.per - 1) / a.per * a.blocks > kMaxGroups) return EF_ERR_INVALID_SHAPE;
  a.once = (long long)a.T * rows * a.D * 2 > kCacheBytes ? 1 : 0;
  return from_hip(ef::launch_rows(a, e4m3, static_cast<hipStream_t>(stream)));
}

// Workgroups that fill the chip: two of either attention kernel fit on a compute unit.
constexpr int kFillWgs = 512;

// Launch shape of attention over pages: see PagedParams. W workgroups share the keys of each
// (kv head, row tile): the chip's 512 places, or one to a sequence where that is more.
struct PagedPlan {
  int rt, mtiles, heads, W, rows;
  bool fused;
  size_t parts_off, m_off, l_off, acc_off, bytes;
};

constexpr int kMostWgs = 2048;
static_assert(kMostWgs * 64 <= ef::kCounterRegionBytes, "a counter for every workgroup");
// The last of a row's parts joins them in the same launch where rows are few (two of 128 to a wave)
// and their parts not hundreds, or up to 16 rows where the table bounds the parts to a handful, that
// is where mostly nothing is cut at all; a second launch otherwise, which costs 4 us and the
// host 2 (one sequence of 166 keys of 8/2 heads of 128, second launch / same 11.1 / 8.4 us).
constexpr int kJoinElems = 1024;
constexpr int kJoinParts = 128;
constexpr int kFewParts = 4;
constexpr int kLeastKeys = 128;  // keys of a part, at least

// `positions`: the table's, which bound the parts of a row (0 for the workspace's size, which does
// not depend on them).
ef_status paged_plan(PagedPlan& p, int T, int B, int Hq, int Hkv, int D, int max_queries,
                     long long positions) {
  const ef_status st = check_heads(T, B, Hq, Hkv, D);
  if (st != EF_OK) return st;
  if (max_queries < 0) return EF_ERR_INVALID_SHAPE;
  const long long rows = (long long)std::min(max_queries, T) * (Hq / Hkv);
  p.rows = (int)rows;
  p.rt = rows <= 16 ? 1 : 2;
  const long long tile = 16 * p.rt, mtiles = (rows + tile - 1) / tile;
  if (mtiles * Hkv > kMaxGroups) return EF_ERR_INVALID_SHAPE;
  p.mtiles = (int)mtiles;
  p.heads = (int)mtiles * Hkv;
  if (p.heads == 0) return EF_OK;
  p.W = std::max(1, std::max(kFillWgs / p.heads, std::min(B, kMostWgs / p.heads)));
  if ((long long)p.heads * p.W > kMaxGroups) return EF_ERR_INVALID_SHAPE;
  const long long parts = std::min<long long>(p.W, positions / kLeastKeys + 2);
  p.fused = p.rt == 1 && p.heads * p.W <= kMostWgs &&
            ((rows * D <= kJoinElems && parts <= kJoinParts) || parts <= kFewParts);
  // Two states a workgroup where keys are cut (W > 1), or as many as any smaller call has: a
  // workspace for the largest one serves them all.
  const long long most =
      B == 1 ? kFillWgs
             : std::max<long long>(kFillWgs, std::min<long long>((long long)B * p.heads, kMostWgs));
  const size_t states = (size_t)most * 2 * tile;
  p.parts_off = ef::kCounterRegionBytes;
  p.m_off = p.parts_off + ef::ws_align256((size_t)B * p.heads * sizeof(int2));
  p.l_off = p.m_off + ef::ws_align256(states * sizeof(float));
  p.acc_off = p.l_off + ef::ws_align256(states * sizeof(float));
  p.bytes = p.acc_off + states * D * sizeof(float);
  return EF_OK;
}

// Launch shape of attention of packed sequences: see PackedParams. Row tiles of a kv head are at
// most G T / 128 + B, and their keys are cut into parts of at least `least` tiles: 128 rows' states
// cost as much as ten tiles, with the second launch that joins them, those of a few rows little
// more than that launch. At least 4 / 16 tiles: one prompt of 777 tokens of 32/8 heads of 128 [13
// tiles] 38.7 / 19.0 us; one token of 16 sequences of 4 heads over 90 to 2311 keys 16.5 / 23.3, 15 of
// one of 32/8 heads over 5000 18.0 / 24.3. Between the border (64 rows of a sequence) and a full tile
// either may be faster: 24 tokens of 32/8 heads over 5000 keys 19.5 / 26.7, over 32768 41.5 / 36.2, 25
// of 4 sequences over 8000 37.9 / 33.7, 19 to 44 of 9 of 16/4 heads over 2747 to 7262 37.2 / 39.4, the
// longer chunks over the shorter contexts 35.6 / 33.7.
constexpr int kLeastFull = 16, kLeastFew = 4, kFewRows = 64;
// Key tiles of a call that are not cut, whatever the rows: the second launch costs more than two parts
// save (one token over 320 keys of 32/8 heads of 128, cut / whole 11.1 / 9.1 us, over 512 11.9 / 11.7,
// of 64/8 heads of 64 10.8 / 9.3; over 777 12.2 / 16.0).
constexpr int kWholeTiles = 8;

struct PackedPlan {
  int fill, least, slots, per_head;
  size_t split_off, m_off, l_off, acc_off;
  size_t need, bytes;  // of this call, and of one of as many or more rows, keys and sequences
};

// Bytes of a workspace with `slots` states of a kv head.
size_t packed_layout(PackedPlan& p, int slots, int Hkv, int D) {
  const size_t states = (size_t)Hkv * slots * 128;
  // The counters that other calls keep at the start of a workspace are left alone.
  p.split_off = ef::kCounterRegionBytes;
  p.m_off = p.split_off + 256;
  p.l_off = p.m_off + ef::ws_align256(states * sizeof(float));
  p.acc_off = p.l_off + ef::ws_align256(states * sizeof(float));
  return slots == 0 ? 0 : p.acc_off + states * D * sizeof(float);
}

ef_status packed_plan(PackedPlan& p, int T, int Tk, int B, int Hq, int Hkv, int D) {
  const ef_status st = check_heads(T, B, Hq, Hkv, D);
  if (st != EF_OK) return st;
  if (Tk < 0) return EF_ERR_INVALID_SHAPE;
  constexpr long long kRows = 128;
  const long long G = Hq / Hkv;
  // (a sequence of one token has one tile)
  const long long tiles = std::min(T * G / kRows + B, (long long)T * ((G + kRows - 1) / kRows));
  p.fill = std::max(kFillWgs / Hkv, 1);
  const long long key_tiles = ((long long)Tk + 63) / 64;
  p.least = (long long)T * G >= (long long)kFewRows * B ? kLeastFull : kLeastFew;
  // A sequence of m row tiles and t > C key tiles has m ceil(t / C) < 2 m t / C units, and the
  // sum of m t over C is at most `fill`.
  auto states = [&](int least) {
    const long long parts = (key_tiles + least - 1) / least;
    return key_tiles <= kWholeTiles || parts <= 1
               ? 0
               : (int)std::min<long long>(2LL * p.fill, tiles * parts);
  };
  // (More rows may be cut less, so a workspace has room for the shortest parts: one for the largest
  // call serves all smaller ones.)
  p.bytes = packed_layout(p, states(kLeastFew), Hkv, D);
  p.slots = states(p.least);
  const long long per_head = tiles + p.slots;
  if (per_head * Hkv > kMaxGroups || 4LL * p.slots * Hkv > kMaxGroups) return EF_ERR_INVALID_SHAPE;
  p.per_head = (int)per_head;
  p.need = packed_layout(p, p.slots, Hkv, D);
  return EF_OK;
}

}  // namespace

extern "C" {

ef_status ef_rope(const void* x, const int* positions, const double* turns, void* out, int T,
                  int H, int D, int rot, int interleaved, double amplitude, int transpose,
                  void* stream) {
  ef_status st = check_heads(T, 1, H, 1, D);
  if (st != EF_OK) return st;
  st = check_rope(rot, D, amplitude);
  if (st != EF_OK) return st;
  if (T == 0) return EF_OK;
  if (x == nullptr || positions == nullptr || turns == nullptr || out == nullptr)
    return EF_ERR_NULL_POINTER;
  if (misaligned(x) || misaligned(turns) || misaligned(out) || misaligned4(positions))
    return EF_ERR_MISALIGNED;
  ef::RowsParams a{};
  a.q = static_cast<const uint16_t*>(x);
  a.q_out = static_cast<uint16_t*>(out);
  a.turns = turns;
  a.positions = positions;
  a.T = T; a.B = 1; a.Hq = H; a.D = D;
  a.rot = rot;
  a.interleaved = interleaved ? 1 : 0;
  a.amplitude = amplitude;
  a.transpose = transpose ? 1 : 0;
  return run_rows(a, false, stream);
}

ef_status ef_cache_write(const void* k, const void* v, const void* q, const double* turns,
                         void* k_cache, void* v_cache, float* k_scale, float* v_scale,
                         const int* table, const int* lengths, const int* starts, void* q_out,
                         int T, int B, int Hq, int Hkv, int D, int pages, int page, int width,
                         int format, int rot, int interleaved, double amplitude, void* stream) {
  ef_status st = check_heads(T, B, Hq == 0 ? Hkv : Hq, Hkv, D);
  if (st != EF_OK) return st;
  if (Hq < 0) return EF_ERR_INVALID_SHAPE;
  st = check_pages(pages, page, width, format);
  if (st != EF_OK) return st;
  if (turns != nullptr) {
    st = check_rope(rot, D, amplitude);
    if (st != EF_OK) return st;
  }
  if (T == 0 || B == 0) return EF_OK;
  if (uneven(starts, T, B)) return EF_ERR_INVALID_SHAPE;
  if (k == nullptr || v == nullptr || lengths == nullptr || (q == nullptr) != (q_out == nullptr))
    return EF_ERR_NULL_POINTER;
  if (misaligned(k) || misaligned(v) || misaligned(q) || misaligned(q_out) || misaligned(turns) ||
      misaligned4(lengths) || misaligned4(starts))
    return EF_ERR_MISALIGNED;
  ef::RowsParams a{};
  st = set_pages(a.c, k_cache, v_cache, k_scale, v_scale, table, pages, page, width, format);
  if (st != EF_OK) return st;
  a.q = static_cast<const uint16_t*>(q);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.turns = turns;
  a.lengths = lengths;
  a.starts = starts;
  a.T = T; a.B = B; a.Hq = q == nullptr ? 0 : Hq; a.Hkv = Hkv; a.D = D;
  a.rot = turns == nullptr ? 0 : rot;
  a.interleaved = interleaved ? 1 : 0;
  a.amplitude = amplitude;
  return run_rows(a, format == EF_CACHE_E4M3, stream);
}

ef_status ef_cache_read(const void* k_cache, const void* v_cache, const float* k_scale,
                        const float* v_scale, const int* table, const int* starts, void* k_out,
                        void* v_out, int T, int B, int Hkv, int D, int pages, int page, int width,
                        int format, void* stream) {
  ef_status st = check_heads(T, B, Hkv, Hkv, D);
  if (st != EF_OK) return st;
  st = check_pages(pages, page, width, format);
  if (st != EF_OK) return st;
  if (T == 0 || B == 0) return EF_OK;
  if (starts == nullptr || k_out == nullptr || v_out == nullptr) return EF_ERR_NULL_POINTER;
  if (misaligned(k_out) || misaligned(v_out) || misaligned4(starts)) return EF_ERR_MISALIGNED;
  ef::CacheReadParams a{};
  st = set_pages(a.c, k_cache, v_cache, k_scale, v_scale, table, pages, page, width, format);
  if (st != EF_OK) return st;
  a.starts = starts;
  a.k_out = static_cast<uint16_t*>(k_out);
  a.v_out = static_cast<uint16_t*>(v_out);
  a.T = T; a.B = B; a.Hkv = Hkv; a.D = D;
  // Tokens for two rounds of the four pieces of every lane, fewer where there are few.
  a.per = 16;
  while (a.per > 1 && (2LL * a.per * Hkv * (D / 8) > 2 * 4 * 256 || T / a.per < 512)) a.per /= 2;
  a.once = 4LL * T * Hkv * D > kCacheBytes ? 1 : 0;
  if (((long long)T + a.per - 1) / a.per > kMaxGroups) return EF_ERR_INVALID_SHAPE;
  return from_hip(ef::launch_cache_read(a, format == EF_CACHE_E4M3,
                                        static_cast<hipStream_t>(stream)));
}

size_t ef_attention_paged_workspace_size(int T, int B, int Hq, int Hkv, int D, int max_queries) {
  PagedPlan p{};
  if (paged_plan(p, T, B, Hq, Hkv, D, max_queries, 0) != EF_OK || B == 0) return 0;
  return p.bytes;
}

ef_status ef_attention_paged(const void* q, const void* k_cache, const void* v_cache,
                             const float* k_scale, const float* v_scale, const int* table,
                             const int* lengths, const int* starts, void* o, int T, int B, int Hq,
                             int Hkv, int D, int max_queries, int pages, int page, int width,
                             int format, float scale, void* workspace, size_t workspace_bytes,
                             void* stream) {
  PagedPlan p{};
  ef_status st = check_pages(pages, page, width, format);
  if (st != EF_OK) return st;
  st = paged_plan(p, T, B, Hq, Hkv, D, max_queries, (long long)width * page);
  if (st != EF_OK) return st;
  // The units of work of a head are counted in 32 bits.
  if ((long long)B * ((long long)width * page / 64 + 32) >= (1LL << 31))
    return EF_ERR_INVALID_SHAPE;
  if (!std::isfinite(scale)) return EF_ERR_INVALID_SCALE;
  if (T == 0 || B == 0) return EF_OK;
  if (uneven(starts, T, B) || (starts == nullptr && max_queries < T / B))
    return EF_ERR_INVALID_SHAPE;
  if (p.heads == 0) return EF_OK;  // no row of a sequence is asked for
  if (q == nullptr || o == nullptr || lengths == nullptr) return EF_ERR_NULL_POINTER;
  if (misaligned(q) || misaligned(o) || misaligned4(lengths) || misaligned4(starts))
    return EF_ERR_MISALIGNED;
  ef::PagedParams a{};
  st = set_pages(a.c, k_cache, v_cache, k_scale, v_scale, table, pages, page, width, format);
  if (st != EF_OK) return st;
  if (workspace == nullptr || workspace_bytes < p.bytes) return EF_ERR_WORKSPACE_TOO_SMALL;
  if (misaligned(workspace)) return EF_ERR_MISALIGNED;
  char* const ws = static_cast<char*>(workspace);
  a.q = static_cast<const uint16_t*>(q);
  a.o = static_cast<uint16_t*>(o);
  a.lengths = lengths;
  a.starts = starts;
  a.parts = reinterpret_cast<int2*>(ws + p.parts_off);
  a.counters = p.fused ? reinterpret_cast<unsigned*>(ws) : nullptr;
  // Counters lie as far apart as there is room for.
  a.counter_stride = p.heads * p.W <= ef::kCounterSlots ? ef::kCounterStride : 16;
  a.ws_m = reinterpret_cast<float*>(ws + p.m_off);
  a.ws_l = reinterpret_cast<float*>(ws + p.l_off);
  a.ws_acc = reinterpret_cast<float*>(ws + p.acc_off);
  a.T = T; a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.D = D;
  a.G = Hq / Hkv;
  a.even = T / B;
  a.max_queries = max_queries;
  a.rt = p.rt;
  a.mtiles = p.mtiles;
  a.rows = p.rows;
  a.heads = p.heads;
  a.W = p.W;
  // The floor keeps a zero scale well defined (every visible key gets weight 1).
  a.c_abs = std::fmax(std::fabs(scale) * ef::kLog2e, 1e-30f);
  a.qflip = scale < 0.f ? 0x80008000u : 0u;
  return from_hip(ef::launch_attention_paged(a, format == EF_CACHE_E4M3,
                                             static_cast<hipStream_t>(stream)));
}

size_t ef_attention_packed_workspace_size(int T, int Tk, int B, int Hq, int Hkv, int D) {
  PackedPlan p{};
  if (packed_plan(p, T, Tk, B, Hq, Hkv, D) != EF_OK || T == 0 || B == 0) return 0;
  return p.bytes;
}

ef_status ef_attention_packed(const void* q, const void* k, const void* v, const int* starts,
                              const int* k_starts, void* o, int T, int Tk, int B, int Hq, int Hkv,
                              int D, float scale, int causal, void* workspace,
                              size_t workspace_bytes, void* stream) {
  PackedPlan p{};
  const ef_status st = packed_plan(p, T, Tk, B, Hq, Hkv, D);
  if (st != EF_OK) return st;
  if (!std::isfinite(scale)) return EF_ERR_INVALID_SCALE;
  if (T == 0 || B == 0) return EF_OK;
  if (q == nullptr || o == nullptr || starts == nullptr || k_starts == nullptr ||
      (Tk > 0 && (k == nullptr || v == nullptr)))
    return EF_ERR_NULL_POINTER;
  if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(o) || misaligned4(starts) ||
      misaligned4(k_starts))
    return EF_ERR_MISALIGNED;
  ef::PackedParams a{};
  if (p.slots > 0) {
    if (workspace == nullptr || workspace_bytes < p.need) return EF_ERR_WORKSPACE_TOO_SMALL;
    if (misaligned(workspace)) return EF_ERR_MISALIGNED;
    char* const ws = static_cast<char*>(workspace);
    a.split = reinterpret_cast<int*>(ws + p.split_off);
    a.ws_m = reinterpret_cast<float*>(ws + p.m_off);
    a.ws_l = reinterpret_cast<float*>(ws + p.l_off);
    a.ws_acc = reinterpret_cast<float*>(ws + p.acc_off);
  }
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.starts = starts;
  a.k_starts = k_starts;
  a.o = static_cast<uint16_t*>(o);
  a.T = T; a.Tk = Tk; a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.D = D;
  a.G = Hq / Hkv;
  a.causal = causal ? 1 : 0;
  a.fill = p.fill;
  a.least = p.least;
  a.slots = p.slots;
  a.per_head = p.per_head;
  a.c_abs = std::fabs(scale) * ef::kLog2e;
  a.qflip = scale < 0.f ? 0x80008000u : 0u;
  return from_hip(ef::launch_attention_packed(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
