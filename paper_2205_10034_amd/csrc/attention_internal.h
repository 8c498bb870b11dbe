// What the attention half's translation units share (not part of the ABI).
#pragma once
#include "moesys_internal.h"
#include "kv_pages.h"

namespace moesys {

__device__ __forceinline__ float bf16_to_float(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }

// float -> bfloat16 bits, round to nearest even (NaN kept quiet).
__device__ __forceinline__ uint32_t float_to_bf16(float f) {
  const uint32_t u = __float_as_uint(f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return (u >> 16) | 0x40u;
  return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

inline bool rows_aligned(const moe_head_rows* r, size_t es) {
  return ((uintptr_t)r->data & 15) == 0 && (r->token_stride * (int64_t)es) % 16 == 0 && (r->head_stride * (int64_t)es) % 16 == 0;
}

}  // namespace moesys
