// Argument checks shared by the entry points of the C ABI (host side).
#pragma once

#include <cmath>
#include <cstdint>

#include "ef_attention.h"
#include "ef_kernels.hpp"

namespace ef {
namespace host {

constexpr int kMaxGridYZ = 65535;

struct Shape {
  int B, Hq, Hkv, Sq, Skv, D;
  long long rows() const { return (long long)B * Hq * Sq; }
};

inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

inline ef_status check_shape(const Shape& s) {
  if (s.B < 0 || s.Sq < 0 || s.Skv < 0 || s.Hq < 1 || s.Hkv < 1) return EF_ERR_INVALID_SHAPE;
  if (s.Hq % s.Hkv != 0) return EF_ERR_GQA_RATIO;
  if (s.D != 64 && s.D != 128) return EF_ERR_UNSUPPORTED_HEAD_DIM;
  // Per-head extents stay below 2^31 elements; batch*heads fits the grid.
  if ((long long)s.Sq * s.D >= (1LL << 31) || (long long)s.Skv * s.D >= (1LL << 31))
    return EF_ERR_INVALID_SHAPE;
  if ((long long)s.B * s.Hkv > kMaxGridYZ || (long long)(s.Hq / s.Hkv) * s.Sq >= (1LL << 31))
    return EF_ERR_INVALID_SHAPE;
  return EF_OK;
}

inline ef_status check_io(const Shape& s, const void* q, const void* k, const void* v,
                          const void* o, float scale) {
  if (!std::isfinite(scale)) return EF_ERR_INVALID_SCALE;
  if (s.rows() == 0) return EF_OK;
  if (q == nullptr || o == nullptr) return EF_ERR_NULL_POINTER;
  if (s.Skv > 0 && (k == nullptr || v == nullptr)) return EF_ERR_NULL_POINTER;
  if (misaligned(q) || misaligned(o) || misaligned(k) || misaligned(v)) return EF_ERR_MISALIGNED;
  return EF_OK;
}

inline ef_status from_hip(hipError_t e) { return e == hipSuccess ? EF_OK : EF_ERR_HIP; }

}  // namespace host
}  // namespace ef
