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
  // Columns of the score product: a position takes gp columns (G rounded up to a
  // power of two, at most 16) of a 16-column tile, or `per` whole tiles when G > 16.
  int gp, per;
  int pos;       // positions per workgroup
  int ptiles;    // workgroups per (sequence, head)
  int stride;    // floats of a position's score row in LDS
};

hipError_t launch_block_summary(const SummaryParams& a, hipStream_t stream);
hipError_t launch_block_select(const SelectParams& a, hipStream_t stream);

}  // namespace ef
