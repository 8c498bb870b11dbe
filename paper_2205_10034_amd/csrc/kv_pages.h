// Places of a paged cache and which of them a new token attends to.  Plain C++ for the host as well: the CPU tests run it.
#pragma once
#include <stdint.h>

#ifdef __HIPCC__
#define MOESYS_HD __host__ __device__ __forceinline__
#else
#define MOESYS_HD inline
#endif

namespace moesys {

// Places of a sequence as attention takes them: a length outside what the table can hold is clamped to it.
MOESYS_HD int kept_length(int len, int capacity) { return len < 0 ? 0 : len > capacity ? capacity : len; }

// First place that a window leaves (0: no window).
MOESYS_HD int first_place(int len, int window) { return window > 0 && len > window ? len - window : 0; }

// Page that a table entry names, or -1: a page that is not there.
MOESYS_HD int valid_page(int entry, int64_t n_pages) { return entry >= 0 && entry < n_pages ? entry : -1; }

}  // namespace moesys
