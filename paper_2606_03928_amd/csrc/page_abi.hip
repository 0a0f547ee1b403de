// page_abi.hip -- the extern "C" entry points of the paged cache: host-side validation and
// dispatch.  Every argument is checked before the first HIP call.
#include "page_internal.hpp"

namespace {

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

constexpr int kMaxHeads = 65536, kMaxSlots = 65536, kMaxPage = 65536, kMaxTokens = 1 << 24;

constexpr int64_t kMaxBlocks = (1 << 24) - 1;   // of 256 threads: a launch has less than 2^32

// strides in elements: whole 16-byte pieces
bool whole_pieces(int64_t stride, int dtype) { return stride % (dtype == VASE_BF16 ? 8 : 4) == 0; }

int check_cache(const vase_pages* c) {
  if (!c || !c->k || !c->v || !c->ref || !c->table || !c->len) return VASE_ERR_INVALID_ARG;
  if (c->dtype != VASE_BF16 && c->dtype != VASE_F32) return VASE_ERR_DTYPE;
  if (c->d != 64 && c->d != 128) return VASE_ERR_INVALID_ARG;
  if (c->n_pages < 1 || c->H < 1 || c->H > kMaxHeads || c->S < 1 || c->S > kMaxSlots || c->M < 1)
    return VASE_ERR_INVALID_ARG;
  if (c->page < 16 || c->page > kMaxPage || c->page % 16 != 0) return VASE_ERR_INVALID_ARG;
  if ((int64_t)c->M * c->page > (1 << 29)) return VASE_ERR_INVALID_ARG;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->ref, 4) || !aligned(c->table, 4) ||
      !aligned(c->len, 4))
    return VASE_ERR_INVALID_ARG;
  // pools of up to 2^62 bytes, so that offsets stay in 64 bits
  if (c->page_stride < (int64_t)c->H * c->page * c->d || !whole_pieces(c->page_stride, c->dtype) ||
      c->page_stride > ((int64_t)1 << 60) / c->n_pages)
    return VASE_ERR_INVALID_ARG;
  return VASE_OK;
}

bool valid_attn_sizes(const vase_pages& c, int T, int G, int max_new, int max_len) {
  return T >= 1 && T <= kMaxTokens && G >= 1 && G <= 16 && max_new >= 1 && max_new <= T &&
         max_len >= 1 && max_len <= c.M * c.page;
}

// token strides, of up to 2^60 elements over the batch
bool valid_stride(int64_t stride, int64_t least, int T, int dtype) {
  return stride >= least && whole_pieces(stride, dtype) && stride <= ((int64_t)1 << 60) / T;
}

int hip_status(hipError_t e) { return e == hipSuccess ? VASE_OK : VASE_ERR_HIP; }

uint32_t* word(int32_t* s) { return reinterpret_cast<uint32_t*>(s); }

}  // namespace

extern "C" {

size_t vase_page_workspace_bytes(int op, const vase_pages* c, int T, int G, int max_new,
                                 int max_len) {
  if (check_cache(c) != VASE_OK) return 0;
  switch (op) {
    case VASE_OP_PAGE_ATTN:
      if (!valid_attn_sizes(*c, T, G, max_new, max_len)) return 0;
      return vase::page_attn_plan(*c, T, G, max_new, max_len).bytes;
    case VASE_OP_PAGE_RESIZE:
      return vase::page_resize_bytes(*c);
    case VASE_OP_PAGE_COMPACT:
      return vase::page_compact_bytes(*c);
    default:
      return 0;
  }
}

int vase_page_attn(const vase_pages* c, const void* q, int64_t q_stride, const int32_t* cu, int T,
                   int G, int max_new, int max_len, int causal, void* out, float* lse, void* ws,
                   size_t ws_bytes, int32_t* dev_status, void* stream) {
  const int st = check_cache(c);
  if (st != VASE_OK) return st;
  if (!aligned(dev_status, 4) || T < 0) return VASE_ERR_INVALID_ARG;
  if (T == 0) return VASE_OK;
  if (!q || !cu || !out || !valid_attn_sizes(*c, T, G, max_new, max_len)) return VASE_ERR_INVALID_ARG;
  if (!valid_stride(q_stride, (int64_t)c->H * G * c->d, T, c->dtype)) return VASE_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4) || !aligned(cu, 4))
    return VASE_ERR_INVALID_ARG;
  const vase::PageAttnPlan plan = vase::page_attn_plan(*c, T, G, max_new, max_len);
  const int64_t rows = (int64_t)T * c->H * G;
  if ((int64_t)plan.n_tile * c->H > kMaxBlocks / plan.n_split || rows > 0x7fffffffLL)
    return VASE_ERR_UNSUPPORTED;
  // the launch that joins ranges has a wave to each row, padding too
  if (plan.n_split > 1 && rows > 4 * kMaxBlocks) return VASE_ERR_UNSUPPORTED;
  if (plan.bytes > 0 && (!ws || ws_bytes < plan.bytes || !aligned(ws, 16))) return VASE_ERR_WORKSPACE;
  return hip_status(vase::launch_page_attn(*c, q, q_stride, cu, T, G, causal, out, lse, ws, plan,
                                           word(dev_status), static_cast<hipStream_t>(stream)));
}

int vase_page_write(const vase_pages* c, const void* k_new, const void* v_new, int64_t new_stride,
                    const int32_t* cu, int T, int32_t* dev_status, void* stream) {
  const int st = check_cache(c);
  if (st != VASE_OK) return st;
  if (!aligned(dev_status, 4) || T < 0 || T > kMaxTokens) return VASE_ERR_INVALID_ARG;
  if (T == 0) return VASE_OK;
  if (!k_new || !v_new || !cu || !valid_stride(new_stride, (int64_t)c->H * c->d, T, c->dtype))
    return VASE_ERR_INVALID_ARG;
  if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(cu, 4)) return VASE_ERR_INVALID_ARG;
  return hip_status(vase::launch_page_write(*c, k_new, v_new, new_stride, cu, T, word(dev_status),
                                            static_cast<hipStream_t>(stream)));
}

int vase_page_resize(const vase_pages* c, const int32_t* new_len, void* ws, size_t ws_bytes,
                     int32_t* dev_status, void* stream) {
  const int st = check_cache(c);
  if (st != VASE_OK) return st;
  if (!new_len || !aligned(new_len, 4) || !aligned(dev_status, 4)) return VASE_ERR_INVALID_ARG;
  if (!ws || ws_bytes < vase::page_resize_bytes(*c) || !aligned(ws, 16)) return VASE_ERR_WORKSPACE;
  return hip_status(vase::launch_page_resize(*c, new_len, ws, word(dev_status),
                                             static_cast<hipStream_t>(stream)));
}

int vase_page_fork(const vase_pages* c, const int32_t* parent, int32_t* dev_status, void* stream) {
  const int st = check_cache(c);
  if (st != VASE_OK) return st;
  if (!parent || !aligned(parent, 4) || !aligned(dev_status, 4)) return VASE_ERR_INVALID_ARG;
  return hip_status(vase::launch_page_fork(*c, parent, word(dev_status),
                                           static_cast<hipStream_t>(stream)));
}

int vase_page_compact(const vase_pages* c, const int32_t* map, const int32_t* src, int n_map, int K,
                      void* ws, size_t ws_bytes, int32_t* dev_status, void* stream) {
  const int st = check_cache(c);
  if (st != VASE_OK) return st;
  if (!map || !src || n_map < 1 || n_map > (1 << 20) || K < 1 || K > c->M * c->page)
    return VASE_ERR_INVALID_ARG;
  if (!aligned(map, 4) || !aligned(src, 4) || !aligned(dev_status, 4)) return VASE_ERR_INVALID_ARG;
  if (!ws || ws_bytes < vase::page_compact_bytes(*c) || !aligned(ws, 16)) return VASE_ERR_WORKSPACE;
  return hip_status(vase::launch_page_compact(*c, map, src, n_map, K, ws, word(dev_status),
                                              static_cast<hipStream_t>(stream)));
}

}  // extern "C"
