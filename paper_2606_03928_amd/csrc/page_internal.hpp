// page_internal.hpp -- the paged cache: device view, row addresses and launch
// declarations shared by page_abi.hip, page_attn.hip and page_state.hip.
#pragma once

#include "vase_internal.hpp"
#include "vase_page.h"

namespace vase {

// Rows come in groups of 16, the unit of a page's size, so that 16 rows that begin at a
// multiple of 16 lie in one page.  group / (page / 16) is a product and a shift: with
// n < 2^26 groups and D <= 2^12, floor(n m / 2^(26 + b)) for b = ceil(log2 D) and
// m = ceil(2^(26 + b) / D) is exact, as n (m D - 2^(26 + b)) < 2^26 D <= 2^(26 + b) D.
struct PageDiv {
  uint32_t mul, shift, groups;   // m, 26 + b, D
};
inline PageDiv page_div(int page) {
  const uint32_t D = (uint32_t)page / 16;
  uint32_t b = 0;
  while ((1u << b) < D) ++b;
  const uint32_t shift = 26 + b;
  return PageDiv{(uint32_t)((((uint64_t)1 << shift) + D - 1) / D), shift, D};
}
__host__ __device__ __forceinline__ int page_of_group(const PageDiv& v, int group) {
  return (int)(((uint64_t)(uint32_t)group * v.mul) >> v.shift);
}

// The cache as kernels take it: pools in 16-byte pieces.
struct PageView {
  uint4 *k, *v;
  int32_t *ref, *table, *len;
  int64_t page_u4;      // pieces from a page to the next
  int64_t head_u4;      // pieces of a head in a page
  PageDiv div;
  int n_pages, H, page, S, M;
};
inline PageView page_view(const vase_pages& c) {
  const int per = 16 / (c.dtype == VASE_BF16 ? 2 : 4);   // elements in 16 bytes
  return PageView{static_cast<uint4*>(c.k), static_cast<uint4*>(c.v), c.ref, c.table, c.len,
                  c.page_stride / per, (int64_t)c.page * c.d / per, page_div(c.page),
                  c.n_pages, c.H, c.page, c.S, c.M};
}

__device__ __forceinline__ bool valid_page(const PageView& c, int p) {
  return (unsigned)p < (unsigned)c.n_pages;
}
// a slot's rows, forced into what its table can hold
__device__ __forceinline__ int slot_len(const PageView& c, int s) {
  return min(max(c.len[s], 0), c.M * c.page);
}
__device__ __forceinline__ int pages_for(const PageView& c, int rows) {
  return page_of_group(c.div, (rows + 15) / 16 + (int)c.div.groups - 1);
}

// The slot of token t: the last s with f(s) <= t, for a function f with f(0) = 0 that does
// not decrease, 64 of its values at a time.  Every lane of the wave gets it; t is
// the same in all of them.  In [0, S) whatever f gives.
template <typename F>
__device__ __forceinline__ int find_slot(int S, int t, F f) {
  const int lane = threadIdx.x % kWave;
  int lo = 0, n = S;
  while (n > 1) {
    const int step = (n + kWave - 1) / kWave;
    const bool le = lane * step < n && f(lo + lane * step) <= t;
    const int c = max(__popcll(__ballot(le)), 1) - 1;
    lo += c * step;
    n = min(step, n - c * step);
  }
  return lo;
}

// page_attn.hip
struct PageAttnPlan {
  bool few;                // row tiles of 16 rows
  bool by_slot;            // and a slot has one at most (max_new * G <= 16)
  bool once;               // V rows are read once, more of them than the caches keep
  int n_tile;              // row tiles of the batch, at most
  int n_split, keys;       // few: key ranges and their length
  int shares;              // else: workgroups among which the work is shared out, or 0
  // workspace: partial outputs, their maxima and sums, the sums of the row tiles' key tiles
  size_t off_ml, off_sums, bytes;
};
PageAttnPlan page_attn_plan(const vase_pages& c, int T, int G, int max_new, int max_len);
hipError_t launch_page_attn(const vase_pages& c, const void* q, int64_t q_stride, const int32_t* cu,
                            int T, int G, int causal, void* out, float* lse, void* ws,
                            const PageAttnPlan& plan, uint32_t* status, hipStream_t stream);

// page_state.hip
hipError_t launch_page_write(const vase_pages& c, const void* k_new, const void* v_new,
                             int64_t new_stride, const int32_t* cu, int T, uint32_t* status,
                             hipStream_t stream);
size_t page_resize_bytes(const vase_pages& c);
hipError_t launch_page_resize(const vase_pages& c, const int32_t* new_len, void* ws, uint32_t* status,
                              hipStream_t stream);
hipError_t launch_page_fork(const vase_pages& c, const int32_t* parent, uint32_t* status,
                            hipStream_t stream);
size_t page_compact_bytes(const vase_pages& c);
hipError_t launch_page_compact(const vase_pages& c, const int32_t* map, const int32_t* src, int n_map,
                               int K, void* ws, uint32_t* status, hipStream_t stream);

}  // namespace vase
