/*
 * vase_page.h -- C ABI of the paged KV cache of libvase (gfx950).
 *
 * The static cache of vase.h holds N = K + B slots for every head instance, used or
 * not.  A paged cache holds the K and V rows of S sequence slots in a pool of pages,
 * so that a sequence takes the memory of the rows it has, prompts of any length go in
 * chunk by chunk, and sequences that begin alike share their pages:
 *
 *   vase_page_attn      attention of each slot's newest rows (one token of decoding, a
 *                       chunk of a prompt) over all rows of the slot (Eq. 1)
 *   vase_page_write     the new rows of a step into the last rows of their slots
 *   vase_page_resize    slots truncated and grown: pages freed, taken, and copied where
 *                       a slot grows within a page that it shares
 *   vase_page_fork      slots that begin as another slot's rows, on the same pages
 *   vase_page_compact   the survivors of an eviction round (vase_select's map) to the
 *                       front of their slot's pages, the pages behind them freed
 *
 * The cache (vase_pages), all of it the caller's device memory:
 *   k, v    pools: page p, head h, row r is at p * page_stride + (h * page + r) * d
 *           elements, H heads.  A head is any (layer, KV head); attention and writes may
 *           be called on some of the heads (k and v moved to the first of them, H their
 *           number, the same page_stride), the other calls take all of them at once.
 *   table   [S][M] int32: table[s][j] is the page of rows [j * page, (j + 1) * page) of
 *           slot s.  Entries behind a slot's last page are not read by any call.
 *   len     [S] int32: the slot's rows.  0: the slot is free.
 *   ref     [n_pages] int32: how many table entries name the page.  0: the page is free.
 * A new cache has len and ref zero.  With page = K + B and one page per slot, the pools
 * are static caches of n_pages * H instances as vase.h's calls take them.
 *
 * Conventions are those of vase.h: nothing is allocated, calls only enqueue work, results
 * are bitwise reproducible, arguments are checked on the host before any HIP call.
 * The stream's device must be the current one.  What is known on the device alone (len, table,
 * ref, cu and the other int32 arrays) is checked there: a call that meets a bad value sets a
 * VASE_STATUS_PAGE_* bit in the nullable dev_status, and nothing outside the
 * caller's buffers is accessed whatever the arrays hold.  Calls that share a
 * workspace or a cache must be ordered by the caller.
 */
#ifndef VASE_PAGE_H_
#define VASE_PAGE_H_

#include "vase.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bits of dev_status, beside vase.h's */
#define VASE_STATUS_PAGE_FULL 16  /* more pages asked for than are free: the call did nothing */
#define VASE_STATUS_PAGE_BAD 32   /* a page number, length, offset or slot number out of range:
                                     see each call for what is left undone */

/* operation ids for vase_page_workspace_bytes */
#define VASE_OP_PAGE_ATTN 0
#define VASE_OP_PAGE_RESIZE 1
#define VASE_OP_PAGE_COMPACT 2

typedef struct {
  void *k, *v;           /* pools, 16-byte aligned */
  int32_t *ref;          /* [n_pages] */
  int32_t *table;        /* [S][M] */
  int32_t *len;          /* [S] */
  int64_t page_stride;   /* elements from a page to the next in k and in v: >= H * page * d,
                            a multiple of 16 bytes */
  int32_t dtype;         /* VASE_BF16 or VASE_F32 */
  int32_t n_pages;       /* >= 1 */
  int32_t H;             /* heads, 1 .. 65536 */
  int32_t page;          /* rows of a page: a multiple of 16, 16 .. 65536 */
  int32_t d;             /* 64 or 128 */
  int32_t S;             /* slots, 1 .. 65536 */
  int32_t M;             /* table entries of a slot; M * page <= 2^29 */
} vase_pages;

/*
 * Workspace in bytes that a call of `op` needs (0 if none, and for invalid arguments).
 * T, G, max_new and max_len are vase_page_attn's; the other operations ignore them.
 */
size_t vase_page_workspace_bytes(int op, const vase_pages* c, int T, int G, int max_new,
                                 int max_len);

/*
 * Attention of the newest rows of every slot over the slot's pages.  cu[s] .. cu[s+1] are
 * slot s's tokens of the batch, n_s = cu[s+1] - cu[s] (0: none): token i of them is
 * the slot's row len[s] - n_s + i, already written.  For each query head a = h * G + g:
 *
 *   out[t][a] = sum_j softmax_j(q[t][a] . k_j / sqrt(d)) v_j
 *   lse[t][a] = ln sum_j exp(q[t][a] . k_j / sqrt(d))
 *
 * over the rows j of head h with j < len[s] and, if causal, j <= len[s] - n_s + i.  A token
 * that sees no row (len[s] < n_s), or only scores of -inf, has out = 0 and lse = -inf; one that
 * sees a score of +inf or NaN has out = NaN, and lse as the formula gives it.  Values of V that
 * are infinite or NaN and seen make an output infinite or NaN as the formula does (where
 * their probability is 0 in fp32, which of both is unspecified).  What rows hold that a
 * token does not see (rows behind len[s], later tokens' rows) does not reach its output, be it
 * infinite or NaN.  Sums and the softmax are in fp32; bf16 caches round the
 * probabilities to bf16 for the product with V.
 *
 *  q         in   [T][H * G][d] device, the cache's dtype; q_stride elements from a token to
 *                 the next (>= H * G * d, a multiple of 16 bytes)
 *  cu        in   [S + 1] int32, cu[0] = 0, not decreasing, cu[S] <= T.  Tokens from
 *                 cu[S] on belong to no slot: their out and lse are left as they were
 *  T         0 .. 2^24; 0: the call does nothing
 *  max_new   no slot has more new tokens than this (1 .. T): a slot that has more
 *            may be left out (VASE_STATUS_PAGE_BAD)
 *  max_len   the longest slot's rows, for the split of the work (1 .. M * page); slots may
 *            be longer, at some loss of speed
 *  G         query heads per head, 1 .. 16
 *  out       out  [T][H * G][d] device, the cache's dtype
 *  lse       out  nullable; [T][H * G] device fp32
 *  ws        >= vase_page_workspace_bytes(VASE_OP_PAGE_ATTN, ...) bytes, 16-byte aligned
 * The order of the sums goes by the sizes that the call is given (T, S, H, G, max_new,
 * max_len): the same call gives the same bits.
 * VASE_STATUS_PAGE_BAD: a page number out of range (the outputs of the slot are
 * unspecified), len[s] outside [0, M * page] (taken as the nearest of both), or max_new
 * exceeded.
 * Errors: VASE_ERR_INVALID_ARG (null or unaligned pointer, sizes out of range),
 *         VASE_ERR_DTYPE, VASE_ERR_WORKSPACE, VASE_ERR_UNSUPPORTED (2^24 or more
 *         workgroups, or 2^31 or more query rows), VASE_ERR_HIP.
 */
int vase_page_attn(const vase_pages* c, const void* q, int64_t q_stride, const int32_t* cu, int T,
                   int G, int max_new, int max_len, int causal, void* out, float* lse, void* ws,
                   size_t ws_bytes, int32_t* dev_status, void* stream);

/*
 * The rows of a step's tokens: token i of slot s (cu as above) becomes row
 * len[s] - n_s + i of its H heads.  No two slots may share the pages written to (vase_page_resize
 * sees to that).  Other rows are left as they were.
 *
 *  k_new, v_new  in  [T][H][d] device, the cache's dtype; new_stride elements from a token
 *                    to the next in both (>= H * d, a multiple of 16 bytes)
 * VASE_STATUS_PAGE_BAD: a token whose row or page is out of range is not written.
 * Errors: as vase_page_attn, without VASE_ERR_WORKSPACE.
 */
int vase_page_write(const vase_pages* c, const void* k_new, const void* v_new, int64_t new_stride,
                    const int32_t* cu, int T, int32_t* dev_status, void* stream);

/*
 * New lengths.  A slot that shrinks (new_len[s] < len[s]) gives up the pages behind its
 * new last row; one that grows takes free pages, the lowest numbers first, slot by
 * slot and row by row.  Where a slot grows within its last page and shares that page
 * (ref > 1), it takes a page of its own for it and copies its rows, of all H heads.  The new
 * rows' contents are whatever their pages held.  new_len[s] < 0 leaves slot s alone.
 * Pages count as free or shared as they are when the call begins: what a call
 * gives up can be taken by the next one.  The entries given up become -1.
 *
 *  new_len   in  [S] device int32, at most M * page
 *  ws        >= vase_page_workspace_bytes(VASE_OP_PAGE_RESIZE, ...) bytes, 16-byte aligned
 * VASE_STATUS_PAGE_FULL (too few free pages) and VASE_STATUS_PAGE_BAD (a length above
 * M * page, the len of a slot that is not left alone or the page it grows in out of
 * range): nothing is changed.  An entry given up that names no page sets
 * VASE_STATUS_PAGE_BAD and becomes -1 like the others.
 * Errors: as vase_page_attn.
 */
int vase_page_resize(const vase_pages* c, const int32_t* new_len, void* ws, size_t ws_bytes,
                     int32_t* dev_status, void* stream);

/*
 * Slots that begin as another's: where parent[s] >= 0, slot s takes the rows and the length
 * of slot parent[s] by sharing its pages.  No row is copied.
 *
 *  parent    in  [S] device int32; negative: slot s is left alone
 * VASE_STATUS_PAGE_BAD, and slot s is left alone: parent[s] >= S, len[s] is not 0,
 * the parent is forked in the same call, or a length or page of the parent out of range.
 * Errors: as vase_page_attn, without VASE_ERR_WORKSPACE.
 */
int vase_page_fork(const vase_pages* c, const int32_t* parent, int32_t* dev_status, void* stream);

/*
 * Compaction (Sec. 2) of the slots with map[s] >= 0: for every head h and j < K
 *
 *   k[s][h][j] <- k[s][h][src[map[s]][h][j]]   and v likewise,   len[s] <- K
 *
 * with src strictly increasing in j and below len[s], as vase_select's survivor maps are
 * (K <= len[s]).  A page that the slot has alone is compacted in place, rows behind K left
 * as they were; for a shared one (ref > 1 when the call begins) the slot takes a free
 * page (the lowest numbers first, slot by slot, row by row), so that the slots it was
 * shared with keep theirs.  The pages behind the K rows are given up (entries -1).
 *
 *  map       in  [S] device int32: which of the n_map maps; negative: slot s is left alone.
 *                Slots may have the same map
 *  src       in  [n_map][H][K] device int32
 *  ws        >= vase_page_workspace_bytes(VASE_OP_PAGE_COMPACT, ...) bytes, 16-byte aligned
 * VASE_STATUS_PAGE_FULL (too few free pages) and VASE_STATUS_PAGE_BAD (map[s] >= n_map, K
 * above a slot's len, a len or a page out of range): nothing is changed.  A src that breaks its
 * contract gives unspecified rows (its entries are clamped to the slot).
 * Errors: as vase_page_attn, plus VASE_ERR_INVALID_ARG for K < 1, n_map < 1.
 */
int vase_page_compact(const vase_pages* c, const int32_t* map, const int32_t* src, int n_map, int K,
                      void* ws, size_t ws_bytes, int32_t* dev_status, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* VASE_PAGE_H_ */
