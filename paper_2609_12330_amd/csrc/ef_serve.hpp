// Kernel parameter blocks and launchers of the serving operators (rotary positions, a
// paged cache, packed sequences), and how they find their sequences.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ef {

// Workgroups of a launch: it holds fewer than 2^32 threads, and these stay well below.
constexpr long long kMaxGroups = (1LL << 31) / 256;

// A cache in pages: k, v [pages][Hkv][page][D], bf16 or e4m3 codes with a scale a row.
struct PagesParams {
  char* k;
  char* v;
  float* k_scale;  // [pages][Hkv][page], e4m3 only
  float* v_scale;
  const int* table;  // [B][width]
  int pages, width;
  int shift;  // log2 of the rows of a page
};

// Rows of new tokens: rotated, and written to out or to the cache (row_ops.hip).
struct RowsParams {
  const uint16_t* q;  // [T][Hq][D]; null: none
  uint16_t* q_out;
  const uint16_t* k;  // [T][Hkv][D]; null: no cache
  const uint16_t* v;
  const double* turns;   // [rot / 2]; null: nothing is rotated
  const int* positions;  // [T]; null: from lengths and starts
  const int* lengths;    // [B]
  const int* starts;     // [B + 1], or null: T / B tokens each
  PagesParams c;
  int T, B, Hq, Hkv, D;
  int rot, interleaved;
  double amplitude;
  int transpose;
  int per;     // tokens of a workgroup, 1 .. 16
  int blocks;  // workgroups that share the rows of these tokens
  int once;    // stores are non-temporal
};

struct CacheReadParams {
  PagesParams c;
  const int* starts;  // [B + 1]
  uint16_t* k_out;    // [T][Hkv][D]
  uint16_t* v_out;
  int T, B, Hkv, D;
  int per;   // tokens of a workgroup, 1 .. 16
  int once;  // stores are non-temporal
};

struct PagedParams {
  const uint16_t* q;  // [T][Hq][D]
  PagesParams c;
  const int* lengths;
  const int* starts;  // or null
  uint16_t* o;
  unsigned* counters;  // not null: the last workgroup of a sequence's rows combines them
  int2* parts;         // [B][heads]: first workgroup and number of the parts of its rows
  float* ws_m;         // [heads * W][2][rows]
  float* ws_l;
  float* ws_acc;       // [heads * W][2][rows][D]
  int T, B, Hq, Hkv, D, G;
  int even;  // rows of a sequence without starts
  int max_queries;
  int rt;       // row tiles of 16 of a workgroup: 1 or 2
  int mtiles;   // workgroup tiles of a kv head's rows
  int rows;     // most rows of a kv head: G max_queries
  int heads;    // Hkv * mtiles: what a launch deals out apart from each other
  int W;        // workgroups of each
  int counter_stride;
  float c_abs;     // |scale| * log2(e)
  uint32_t qflip;  // 0x80008000 for a negative scale, else 0
};

struct PackedParams {
  const uint16_t* q;  // [T][Hq][D]
  const uint16_t* k;  // [Tk][Hkv][D]
  const uint16_t* v;
  const int* starts;
  const int* k_starts;
  uint16_t* o;
  int* split;     // states of a kv head that the call makes
  float* ws_m;    // [Hkv][slots][128]
  float* ws_l;
  float* ws_acc;  // [Hkv][slots][128][D]
  int T, Tk, B, Hq, Hkv, D, G;
  int causal;
  int fill;      // workgroups of a kv head that fill its share of the chip
  int least;     // fewest key tiles of a part
  int slots;     // partial states of a kv head that the workspace holds; 0: nothing is split
  int per_head;  // workgroups of a kv head
  float c_abs;
  uint32_t qflip;
};

hipError_t launch_rows(const RowsParams& a, bool e4m3, hipStream_t stream);
hipError_t launch_cache_read(const CacheReadParams& a, bool e4m3, hipStream_t stream);
hipError_t launch_attention_paged(const PagedParams& a, bool e4m3, hipStream_t stream);
hipError_t launch_attention_packed(const PackedParams& a, hipStream_t stream);

#ifdef __HIPCC__
// Start of sequence b (b <= B): starts[b] clamped to the rows, or b * (T / B).
__device__ __forceinline__ int sequence_start(const int* starts, int b, int B, int T) {
  return starts == nullptr ? b * (T / B) : min(max(starts[b], 0), T);
}

// Sequence of packed row t: the number of starts[1 .. B] that are at most t, B where t lies behind
// the last one. -1 where it lies in front of the first. The wave's lanes make the call with the
// same t, and read 64 starts at a time.
__device__ __forceinline__ int find_sequence(const int* starts, int B, int T, int t) {
  if (starts == nullptr) return t / (T / B);
  const int lane = threadIdx.x & 63;
  int n = 0;
  for (int i = 0; i <= B; i += 64) {
    const bool below = i + lane <= B && starts[i + lane] <= t;
    const int c = __popcll(__builtin_amdgcn_ballot_w64(below));
    n += c;
    if (c < 64) break;
  }
  return n - 1;
}

// Inclusive sums over the wave's lanes: within rows of 16, then rows 0 and 2 into the next ones,
// then the first half into the second.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111 /* row_shr:1 */, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142 /* row_bcast:15 */, 0xa, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x143 /* row_bcast:31 */, 0xc, 0xf, false);
  return x;
}
#endif

}  // namespace ef
