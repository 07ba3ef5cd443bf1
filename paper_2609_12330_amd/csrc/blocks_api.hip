// Host side of the long-context entry points of include/ef_attention.h: argument
// validation, launch shapes and workspace arithmetic.
#include <algorithm>

#include "ef_attention.h"
#include "ef_blocks.hpp"
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

// Most bytes of LDS a selection workgroup keeps its scores in: two workgroups to
// a compute unit, and any list of EF_MAX_BLOCKS scores fits.
constexpr int kSelectLds = 64 * 1024 - 256;

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
  // Rows of four floats more than whole tiles: 16 positions' rows start in different banks.
  a.stride = (nb + 15) / 16 * 16 + 4;
  // Positions per workgroup: four column tiles where the scores fit and the grid
  // still fills the chip, else one tile, fewer positions where they do not fit.
  const long long heads = (long long)B * Hkv;
  const int fit = std::max(1, kSelectLds / (a.stride * 4));
  int pos = a.per > 1 ? 1 : 16 / a.gp;
  if (a.per == 1 && 4 * pos <= fit && heads * ((Sq + 4 * pos - 1) / (4 * pos)) >= 512) pos *= 4;
  a.pos = std::min(std::min(pos, fit), Sq);
  const long long ptiles = ((long long)Sq + a.pos - 1) / a.pos;
  if (heads * ptiles >= (1LL << 31)) return EF_ERR_INVALID_SHAPE;
  a.ptiles = (int)ptiles;
  return from_hip(ef::launch_block_select(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
