// What the calls on a caller's paged cache share: its device view, and the checks of the host side.
#pragma once
#include <cstdint>
#include <string>

#include "tsd_internal.h"

namespace tsd {

// implemented in tsd_api.hip: records the message tsd_last_error(NULL) returns
int fail_no_handle(int code, const std::string& msg);

// The cache as kernels see it.  Offsets are in elements and 64 bits wide: a long cache passes 2^32.
struct PagedView {
  char* k;
  char* v;
  long page_stride, token_stride, head_stride;
  const int* table;
  int table_stride, cols, n_pages, pt_shift;
};

// Rows of heads, [B][T][heads][head_dim] with dense heads.
struct RowsView {
  char* p;
  long sb, st, sh;
};

inline RowsView rows_view(const tsd_rows& r) { return {static_cast<char*>(r.data_dev), (long)r.stride_b, (long)r.stride_t, (long)r.stride_h}; }

#if defined(__HIPCC__)
// Offset of cache row `slot` of a sequence whose table row is `table` (head 0), or -1 where the table has no page for it: beyond its columns,
// or an entry that names none of the pool's pages.  Such a slot is a hole: nothing is read or written there.
// In two halves, so that the entry can be on its way before it is known whether it counts.
__device__ __forceinline__ int paged_entry(const PagedView& c, const int* table, int slot) {
  return table[min(max(slot, 0) >> c.pt_shift, c.cols - 1)];
}
__device__ __forceinline__ long paged_row(const PagedView& c, int entry, int slot) {
  if (slot < 0 || slot >> c.pt_shift >= c.cols || (unsigned)entry >= (unsigned)c.n_pages) return -1;
  return entry * c.page_stride + (slot & ((1 << c.pt_shift) - 1)) * c.token_stride;
}
#endif

constexpr int kTreeNodes = 256;  // most nodes of a tree of drafts

// A launch has fewer than 2^32 lanes.
constexpr int64_t max_workgroups(int lanes) { return 0xFFFFFFFFll / lanes; }

inline int type_bytes(int dtype) { return dtype == TSD_BF16 ? 2 : 4; }

// 16-byte loads: rows start on 16 bytes, whatever the strides.
inline bool rows_aligned(const tsd_rows& r, int es) {
  return !(reinterpret_cast<uintptr_t>(r.data_dev) & 15) && !(r.stride_b * es & 15) && !(r.stride_t * es & 15) && !(r.stride_h * es & 15);
}

int check_cache(const tsd_paged_cache* c);                                        // TSD_OK or a recorded failure
int check_rows(const tsd_rows* r, int es, const char* name);
PagedView cache_view(const tsd_paged_cache& c);

}  // namespace tsd
