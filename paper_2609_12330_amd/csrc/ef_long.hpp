// Kernel parameter blocks and launchers of the long-context operators: block
// summaries, block selection, attention over selected blocks, attention over a
// shared prefix.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ef {

// Most blocks of a key axis: a query's scores, one fp32 per block, stay in LDS.
constexpr int kMaxBlocks = 16000;
// Most blocks of a list: the exact choice at a list's border holds four per lane.
constexpr int kMaxTopk = 256;

// Valid keys of sequence b: lengths[b] clamped to the capacity, or all of them.
__device__ __forceinline__ int sequence_length(const int* lengths, int b, int capacity) {
  return lengths == nullptr ? capacity : min(max(lengths[b], 0), capacity);
}

struct SummaryParams {
  const uint16_t* k;   // [B][Hkv][Skv][D] bf16
  const int* lengths;  // [B] or null
  uint16_t* s;         // [B][Hkv][NB][D] bf16
  int B, Hkv, Skv, D;
  int NB;
  int block;     // keys per block
  int new_keys;  // > 0: only the blocks of each sequence's last new_keys keys
  int touched;   // blocks per (sequence, head) that the launch looks at
};

// Bytes of LDS for the scores of a selection workgroup of many rows: two to a compute
// unit. With few rows the launch sets the size, 64 KiB at most.
constexpr int kSelectLds = 66 * 1024;

struct SelectParams {
  const uint16_t* q;   // [B][Hq][Sq][D] bf16
  const uint16_t* s;   // [B][Hkv][NB][D] bf16
  const int* lengths;  // [B] or null
  int* out;            // [B][Hkv][Sq][K]
  int B, Hq, Hkv, Sq, Skv, D;
  int G;         // Hq / Hkv
  int NB;
  int shift;     // log2 of the keys per block
  int K, sinks, local;
  // Rows of the score product: a position takes gp rows (G rounded up to a power of
  // two, at most 16) of a 16-row tile, or `per` whole tiles when G > 16.
  int gp, per;
  int waves;     // waves per workgroup where its rows fill one tile: 4 or 8
  int pos;       // positions per workgroup
  int ptiles;    // workgroups per (sequence, head)
  int stride;    // floats of a position's score row in LDS
};

// Combine inside the launch that stores the states: states of a row, and elements of rows,
// that one round of its loads takes.
constexpr int kSharedParts = 8;
constexpr int kSharedElems = 512;

// Attention over selected blocks (matrix-core kernel). With P > 1 the workgroups of a
// row tile share its blocks and store partial states, m, l [rows][P] and
// acc [rows][P][D]; with P = 1 they write o.
struct BlocksParams {
  const uint16_t* q;   // [B][Hq][Sq][D] bf16
  const uint16_t* k;   // [B][Hkv][Skv][D] bf16
  const uint16_t* v;
  const int* blocks;   // [B][Hkv][Sq][K]
  const int* lengths;  // [B] or null
  uint16_t* o;         // [B][Hq][Sq][D] bf16
  float* ws_m;
  float* ws_l;
  float* ws_acc;
  unsigned* counters;  // not null: the last workgroup of a (sequence, kv head) to store
                       // its state combines (one row tile; see group_combine.hpp)
  int B, Hq, Hkv, Sq, Skv, D;
  int G, R;      // Hq / Hkv, rows of a kv head (G * Sq)
  int NB, shift, K;
  int P;         // workgroups per row tile
  int bm;        // rows per workgroup, 64 or 128
  int mtiles;    // row tiles per kv head
  float c_abs;     // |scale| * log2(e)
  uint32_t qflip;  // 0x80008000 for a negative scale (q is negated), else 0
};

// Attention over a shared prefix and each sequence's own keys (matrix-core kernel).
// The keys of sequence b are Lp prefix keys, then len_b own ones. Two kinds of
// workgroups in one launch:
//  - the first n_prefix hold rows of several sequences (all rows of a kv head, in
//    the order [b][sq][g]) and a part of the prefix;
//  - the others hold rows of one sequence and a part of its own keys, or of all its
//    keys (whole = 1, n_prefix = 0).
// Partial states go to slots 0 .. P1 - 1 (prefix) and P1 .. P - 1 (own keys) of
// m, l [rows][P] and acc [rows][P][D]; with P = 1 workgroups write o.
struct PrefixParams {
  const uint16_t* q;   // [B][Hq][Sq][D] bf16
  const uint16_t* kp;  // [Hkv][Lp][D] bf16
  const uint16_t* vp;
  const uint16_t* k;   // [B][Hkv][Skv][D] bf16
  const uint16_t* v;
  const int* lengths;  // [B] or null
  uint16_t* o;         // [B][Hq][Sq][D] bf16
  float* ws_m;
  float* ws_l;
  float* ws_acc;
  int B, Hq, Hkv, Sq, Skv, Lp, D;
  int G, R;         // Hq / Hkv, rows of a (sequence, kv head): G * Sq
  int causal;
  int whole;
  int P1, T1, mt1;  // prefix: partitions, their tiles of 64 keys, row tiles per kv head
  int P2, T2, mt2;  // own keys: the same, row tiles per (sequence, kv head)
  int P;            // P1 + P2, or 1
  unsigned n_prefix, n_own;  // workgroups
  float c_abs;
  uint32_t qflip;
};

// o[row] = sum_p e^(m_p - M) acc_p / sum_p e^(m_p - M) l_p in bf16, 0 where no state
// has a key (M = -inf).
struct StateCombineParams {
  const float* m;  // [rows][P], natural-log units
  const float* l;
  const float* acc;  // [rows][P][D]; not read where m is -inf
  uint16_t* o;       // [rows][D] bf16
  int rows, P, D;
};

hipError_t launch_attention_blocks(const BlocksParams& a, hipStream_t stream);
hipError_t launch_attention_prefix(const PrefixParams& a, hipStream_t stream);
hipError_t launch_state_combine(const StateCombineParams& a, hipStream_t stream);
hipError_t launch_block_summary(const SummaryParams& a, hipStream_t stream);
hipError_t launch_block_select(const SelectParams& a, hipStream_t stream);

}  // namespace ef
