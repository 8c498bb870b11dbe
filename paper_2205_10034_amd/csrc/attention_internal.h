// What the attention half's translation units share (not part of the ABI).
#pragma once
#include "moesys_internal.h"
#include "kv_pages.h"

namespace moesys {

inline bool rows_aligned(const moe_head_rows* r, size_t es) {
  return ((uintptr_t)r->data & 15) == 0 && (r->token_stride * (int64_t)es) % 16 == 0 && (r->head_stride * (int64_t)es) % 16 == 0;
}

}  // namespace moesys
