// page_state.hip -- the paged cache's state: rows written, slots resized, forked and
// compacted.  Page numbers are whole numbers and the lowest free ones are taken in slot
// order, so every result is fixed by the inputs (the counts' atomics are on integers).
#include "page_internal.hpp"

namespace vase {
namespace {

constexpr int kBlock = 256;
constexpr int kPlanBlock = 1024;
constexpr int kPlanWaves = kPlanBlock / kWave;

__device__ __forceinline__ void raise(uint32_t* status, uint32_t bit) {
  if (status) atomicOr(status, bit);
}

// rows that are not read again soon: past the caches (compact of 2304 heads of 4096 rows:
// 1936 us with plain accesses, 1896 so)
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load_once(const uint4* p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)));
}
__device__ __forceinline__ void store_once(uint4* p, const uint4& x) {
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4, x), reinterpret_cast<u32x4*>(p));
}

// ---------------------------------------------------------------------------
// write: one wave per token and group of heads, K and V.  Bound by HBM (each row read
// once, written once); the token's slot is found by the wave's lanes together.  fp32, 8 heads of
// 128, 9 slots of 1000 tokens: 28 us, 5.3 TB/s; a token to each of 64 slots: 3.4 us, latency.
// ---------------------------------------------------------------------------
constexpr int kWritePieces = 512;   // of a token, per wave and pool

template <int PPR>
__global__ __launch_bounds__(kBlock) void page_write_kernel(PageView c, const uint4* __restrict__ kn,
                                                            const uint4* __restrict__ vn,
                                                            int64_t token_u4,
                                                            const int32_t* __restrict__ cu, int T,
                                                            uint32_t* status) {
  const int lane = threadIdx.x % kWave;
  const int t = __builtin_amdgcn_readfirstlane(blockIdx.x * (kBlock / kWave) + threadIdx.x / kWave);
  if (t >= T || t >= cu[c.S]) return;
  const int s = find_slot(c.S, t, [&](int i) { return cu[i]; });
  const int64_t at = (int64_t)c.len[s] - ((int64_t)cu[s + 1] - t);   // of any len: in range or not
  const int row = at < 0 || at >= c.M * c.page ? -1 : (int)at;
  const int q = row < 0 ? 0 : page_of_group(c.div, row / 16);
  // offsets that fall may give a slot that the token is not of
  const int p = row < 0 || t < cu[s] || t >= cu[s + 1] ? -1 : c.table[(int64_t)s * c.M + q];
  if (!valid_page(c, p)) {
    if (lane == 0) raise(status, VASE_STATUS_PAGE_BAD);
    return;
  }
  const int64_t to = p * c.page_u4 + (int64_t)(row - q * c.page) * PPR;
  const int64_t from = t * token_u4;
  const int n = c.H * PPR;
  const int i1 = min(n, (int)(blockIdx.y + 1) * kWritePieces);
  for (int i = blockIdx.y * kWritePieces + lane; i < i1; i += 4 * kWave) {
    uint4 a[4], b[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int x = min(i + u * kWave, i1 - 1);
      a[u] = kn[from + x];
      b[u] = vn[from + x];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int x = i + u * kWave;
      if (x < i1) {
        c.k[to + (x / PPR) * c.head_u4 + x % PPR] = a[u];
        c.v[to + (x / PPR) * c.head_u4 + x % PPR] = b[u];
      }
    }
  }
}

// ---------------------------------------------------------------------------
// The plan of a resize or a compaction: one workgroup counts what each slot needs, lists the
// lowest free pages and decides whether the call goes through; the launch behind it
// changes the state, all of it or nothing.  One workgroup and a launch are a chain of
// latencies (256 slots: 6.6 us, and 3.0 for the entries), and shorter than a plan among
// workgroups that wait for each other would be.
// ---------------------------------------------------------------------------
// exclusive sums over the workgroup, and the total
__device__ __forceinline__ long long block_scan(long long x, long long* s_wave, long long& total) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  long long y = x;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const long long z = __shfl_up(y, o, kWave);
    if (lane >= o) y += z;
  }
  if (lane == kWave - 1) s_wave[wave] = y;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    before += w < wave ? s_wave[w] : 0;
    all += s_wave[w];
  }
  __syncthreads();
  total = all;
  return before + y - x;
}

// The counts of the pages from `base` on that a thread looks at in one pass of the search
// (behind the last page: its own count).
constexpr int kLook = 8;
struct Look {
  int r[kLook];
};
__device__ __forceinline__ Look look(const int32_t* __restrict__ ref, int n_pages, int64_t base) {
  Look l;
#pragma unroll
  for (int u = 0; u < kLook; ++u) {
    const int64_t p = base + u * kPlanBlock + threadIdx.x;
    l.r[u] = ref[p < n_pages ? p : n_pages - 1];
  }
  return l;
}

// The lowest `want` pages without a count into list, in order; how many there are of them.
// l: the first pass's counts, which do not wait for `want`.
__device__ int list_free(const int32_t* __restrict__ ref, int n_pages, int want, Look l, int32_t* list,
                         int* s_count /* [kLook * kPlanWaves] */) {
  constexpr int U = kLook;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int found = 0;
  for (int64_t base = 0; base < n_pages && found < want; base += U * kPlanBlock) {
    uint64_t m[U];
    if (base > 0) l = look(ref, n_pages, base);
#pragma unroll
    for (int u = 0; u < U; ++u)
      m[u] = __ballot(base + u * kPlanBlock + threadIdx.x < n_pages && l.r[u] == 0);
    if (lane < U) {
      uint64_t mine = 0;
#pragma unroll
      for (int u = 0; u < U; ++u) mine = lane == u ? m[u] : mine;
      s_count[lane * kPlanWaves + wave] = __popcll(mine);
    }
    __syncthreads();
    // sums over the U * kPlanWaves = 128 counts, two of them to a lane
    const int a = s_count[2 * lane], b = s_count[2 * lane + 1];
    int y = a + b;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int z = __shfl_up(y, o, kWave);
      if (lane >= o) y += z;
    }
    const int all = __shfl(y, kWave - 1, kWave);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = u * kPlanWaves + wave;                 // this wave's count of pass u
      const int upto = __shfl(y, e / 2, kWave);            // through the lane that holds it
      const int ea = __shfl(a, e / 2, kWave), eb = __shfl(b, e / 2, kWave);
      const int before = found + upto - (e % 2 == 0 ? ea + eb : eb);
      const int at = before + __popcll(m[u] & ((1ull << lane) - 1));
      const int64_t p = base + u * kPlanBlock + threadIdx.x;
      if ((m[u] >> lane & 1) && at < want) list[at] = (int32_t)p;
    }
    found += all;
    __syncthreads();
  }
  return min(found, want);
}

// workspace head: the call goes through; number of listed slots
constexpr int kHead = 16;

constexpr int kCopyBlocks = 512;   // of a resize: most calls copy little or nothing

struct ResizePlan {   // in the workspace, int32 each
  int32_t *head, *begin, *off, *cow_slot, *cow_page, *cow_rows, *free;
};
ResizePlan resize_plan(void* ws, int S) {
  int32_t* p = static_cast<int32_t*>(ws);
  return ResizePlan{p, p + kHead, p + kHead + S, p + kHead + 2 * S, p + kHead + 3 * S,
                    p + kHead + 4 * S, p + kHead + 5 * S};
}

__global__ __launch_bounds__(kPlanBlock) void page_resize_plan_kernel(PageView c,
                                                                      const int32_t* __restrict__ new_len,
                                                                      ResizePlan w, uint32_t* status) {
  __shared__ long long s_wave[kPlanWaves];
  __shared__ int s_count[kLook * kPlanWaves];
  constexpr int kCow = 48;   // sums of two numbers in one: pages below bit 48, copies above
  const int cap = c.M * c.page;
  const Look first_look = look(c.ref, c.n_pages, 0);
  bool bad = false;
  long long need_all = 0;
  int n_cow = 0;
  for (int base = 0; base < c.S; base += kPlanBlock) {
    const int s = base + threadIdx.x;
    int need = 0, rows = 0, last = 0;
    bool cow = false;
    if (s < c.S) {
      const int L = c.len[s], t = new_len[s];
      int first = 0;
      if (t >= 0) {
        if (t > cap || L < 0 || L > cap) {
          bad = true;
        } else if (t > L) {
          const int old = pages_for(c, L);
          first = old;
          const int full = page_of_group(c.div, L / 16);   // whole pages
          rows = L - full * c.page;
          if (rows > 0) {
            last = c.table[(int64_t)s * c.M + old - 1];
            if (!valid_page(c, last)) {
              bad = true;
            } else if (c.ref[last] > 1) {
              cow = true;
              first = old - 1;
            }
          }
          need = pages_for(c, t) - first;
        }
      }
      w.begin[s] = first;
    }
    long long all;
    const long long x = block_scan((long long)need | (long long)cow << kCow, s_wave, all);
    constexpr long long kLow = (1ll << kCow) - 1;
    if (s < c.S) {
      const long long off = need_all + (x & kLow);
      w.off[s] = (int)min(off, (long long)c.n_pages);
      if (cow) {
        const int i = n_cow + (int)(x >> kCow);
        w.cow_slot[i] = s;
        w.cow_page[i] = last;
        w.cow_rows[i] = rows;
      }
    }
    need_all += all & kLow;
    n_cow += (int)(all >> kCow);
  }
  bad = __syncthreads_or(bad);
  bool full = need_all > c.n_pages;
  if (!bad && !full && need_all > 0)
    full = list_free(c.ref, c.n_pages, (int)need_all, first_look, w.free, s_count) < need_all;
  if (threadIdx.x == 0) {
    w.head[0] = !bad && !full;
    w.head[1] = n_cow;
    if (bad) raise(status, VASE_STATUS_PAGE_BAD);
    else if (full) raise(status, VASE_STATUS_PAGE_FULL);
  }
}

// Workgroups below c.S: a slot's entries, counts and length.  The others: the rows of the
// pages that slots take for their own, a head of one page at a time (64 pages of 64 heads of
// 32 rows of 128, 47 MB: 9.3 us, 5 TB/s).
template <int PPR>
__global__ __launch_bounds__(kBlock) void page_resize_kernel(PageView c,
                                                             const int32_t* __restrict__ new_len,
                                                             ResizePlan w, uint32_t* status) {
  if ((int)blockIdx.x < c.S) {
    const int s = blockIdx.x;
    // every load that waits for no other; the plan writes begin and off of every slot
    const int go = w.head[0], L = c.len[s], t = new_len[s], first = w.begin[s], off = w.off[s];
    if (!go || t < 0 || t == L) return;
    __syncthreads();   // every thread has the old length
    int32_t* row = c.table + (int64_t)s * c.M;
    const int old = pages_for(c, L), now = pages_for(c, t);
    if (t > L) {
      for (int j = first + threadIdx.x; j < now; j += kBlock) {
        if (j < old) atomicSub(&c.ref[row[j]], 1);   // the shared page that it grows in
        const int p = w.free[off + j - first];
        row[j] = p;
        c.ref[p] = 1;
      }
    } else {
      for (int j = now + threadIdx.x; j < old; j += kBlock) {
        const int p = row[j];
        if (valid_page(c, p)) atomicSub(&c.ref[p], 1);
        else raise(status, VASE_STATUS_PAGE_BAD);
        row[j] = -1;
      }
    }
    if (threadIdx.x == 0) c.len[s] = t;
    return;
  }
  const int64_t items = w.head[0] ? (int64_t)w.head[1] * c.H : 0;
  for (int64_t i = blockIdx.x - c.S; i < items; i += gridDim.x - c.S) {
    const int e = (int)(i / c.H), h = (int)(i % c.H);
    const int64_t from = w.cow_page[e] * c.page_u4 + h * c.head_u4;
    const int64_t to = w.free[w.off[w.cow_slot[e]]] * c.page_u4 + h * c.head_u4;
    const int n = w.cow_rows[e] * PPR;
    for (int x = threadIdx.x; x < n; x += kBlock) {
      const uint4 a = c.k[from + x], b = c.v[from + x];
      c.k[to + x] = a;
      c.v[to + x] = b;
    }
  }
}

// ---------------------------------------------------------------------------
// fork: a workgroup per slot.  Bound by latency (16 slots: 3.5 us) and the counts' atomics
// (1024 slots of 500 to 8192 rows on pages of 16, three of four forked: 11 us).
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(kBlock) void page_fork_kernel(PageView c, const int32_t* __restrict__ parent,
                                                           uint32_t* status) {
  const int s = blockIdx.x;
  const int p = parent[s];
  if (p < 0) return;
  // a parent is no child of this call, so its length and entries stand
  bool bad = p >= c.S || parent[p < c.S ? p : 0] >= 0 || c.len[s] != 0;
  const int L = bad ? 0 : c.len[p];
  bad = bad || L < 0 || L > c.M * c.page;
  const int n = bad ? 0 : pages_for(c, L);
  const int32_t* from = c.table + (int64_t)(bad ? 0 : p) * c.M;
  for (int j = threadIdx.x; j < n; j += kBlock) bad |= !valid_page(c, from[j]);
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) raise(status, VASE_STATUS_PAGE_BAD);
    return;
  }
  for (int j = threadIdx.x; j < n; j += kBlock) {
    const int q = from[j];
    c.table[(int64_t)s * c.M + j] = q;
    atomicAdd(&c.ref[q], 1);
  }
  if (threadIdx.x == 0) c.len[s] = L;
}

// ---------------------------------------------------------------------------
// compact
// ---------------------------------------------------------------------------
// rows that a workgroup moves at once: 16 KB of K and V each, 8 KB of the shortest rows
constexpr int chunk_rows(int row_pieces) { return row_pieces == 32 ? 32 : 64; }
constexpr int kTicketGap = 32;      // counters of their own cache lines
constexpr int kFewItems = 512;     // (slot, head) pairs below which chunks go one by one

struct CompactState {   // in the workspace, int32 each
  int32_t *head;
  int32_t *slot, *len;  // [S]: the slots to compact and their lengths
  int32_t *old, *rank;  // [S][M] by list place: the entries, and which free page replaces each (-1: none)
  int32_t *free;        // [n_pages]
  int32_t *ticket;      // few (slot, head) pairs: the next chunk of each, kTicketGap apart
  int32_t *said;        // and [pair][chunk], 1: its rows are in registers
};
// fewer than kFewItems, whatever the slots
size_t few_pairs(const vase_pages& c) { return (size_t)c.S * c.H < kFewItems ? (size_t)c.S * c.H : kFewItems; }
CompactState compact_state(void* ws, const vase_pages& c) {
  int32_t* p = static_cast<int32_t*>(ws) + kHead;
  const size_t S = c.S, sm = S * c.M;
  return CompactState{static_cast<int32_t*>(ws), p, p + S, p + 2 * S, p + 2 * S + sm, p + 2 * S + 2 * sm,
                      p + 2 * S + 2 * sm + c.n_pages,
                      p + 2 * S + 2 * sm + c.n_pages + few_pairs(c) * kTicketGap};
}

__global__ __launch_bounds__(kPlanBlock) void page_compact_plan_kernel(PageView c,
                                                                       const int32_t* __restrict__ map,
                                                                       int n_map, int K, int chunk, CompactState w,
                                                                       uint32_t* status) {
  __shared__ long long s_wave[kPlanWaves];
  __shared__ int s_count[kLook * kPlanWaves];
  __shared__ int s_most;
  const Look first_look = look(c.ref, c.n_pages, 0);
  if (threadIdx.x == 0) s_most = 0;
  __syncthreads();
  bool bad = false;
  int n = 0;
  for (int base = 0; base < c.S; base += kPlanBlock) {
    const int s = base + threadIdx.x;
    const int m = s < c.S ? map[s] : -1, L = s < c.S ? c.len[s] : 0;
    const bool ok = m >= 0 && m < n_map && L >= K && L <= c.M * c.page;
    bad |= m >= 0 && !ok;
    long long all;
    const long long x = block_scan(ok, s_wave, all);
    if (ok) {
      w.slot[n + (int)x] = s;
      w.len[n + (int)x] = L;
      atomicMax(&s_most, pages_for(c, L));
    }
    n += (int)all;
  }
  bad = __syncthreads_or(bad);   // also: the lists and s_most are written
  const int64_t items = (int64_t)n * c.H;
  if (items < kFewItems) {
    for (int i = threadIdx.x; i < items; i += kPlanBlock) w.ticket[i * kTicketGap] = 0;
    for (int64_t i = threadIdx.x; i < items * ((K + chunk - 1) / chunk); i += kPlanBlock) w.said[i] = 0;
  }
  const int most = max(s_most, 1), kept = pages_for(c, K);
  const int64_t pairs = bad ? 0 : (int64_t)n * most;
  long long need = 0;
  int e = threadIdx.x / most, j = threadIdx.x % most;   // of pair i
  const int e_step = kPlanBlock / most, j_step = kPlanBlock % most;
  for (int64_t base = 0; base < pairs; base += kPlanBlock, e += e_step, j += j_step) {
    const int64_t i = base + threadIdx.x;
    if (j >= most) {
      j -= most;
      ++e;
    }
    bool shared = false;
    if (i < pairs && j < pages_for(c, w.len[e])) {
      const int p = c.table[(int64_t)w.slot[e] * c.M + j];
      bad |= !valid_page(c, p);
      shared = j < kept && valid_page(c, p) && c.ref[p] > 1;
      w.old[(int64_t)e * c.M + j] = p;
    }
    long long all;
    const long long x = block_scan(shared, s_wave, all);
    if (i < pairs && j < kept)
      w.rank[(int64_t)e * c.M + j] = shared ? (int)min(need + x, (long long)c.n_pages) : -1;
    need += all;
  }
  bad = __syncthreads_or(bad);
  bool full = need > c.n_pages;
  if (!bad && !full && need > 0) full = list_free(c.ref, c.n_pages, (int)need, first_look, w.free, s_count) < need;
  if (threadIdx.x == 0) {
    w.head[0] = !bad && !full;
    w.head[1] = n;
    if (bad) raise(status, VASE_STATUS_PAGE_BAD);
    else if (full) raise(status, VASE_STATUS_PAGE_FULL);
  }
}

// Where row j of a (slot, head) comes from and goes to, in pieces from the pools' first; `to`
// is -1 for a row that stays where it is, and for rows from K on.
struct RowMove {
  int64_t from, to;
};
template <int PPR>
__device__ __forceinline__ RowMove row_move(const PageView& c, const CompactState& w, int e, int64_t head,
                                            int K, int j, int src) {
  const int32_t* old = w.old + (int64_t)e * c.M;
  const int jj = min(j, K - 1);
  const int f = min(max(src, 0), w.len[e] - 1);
  const int qf = page_of_group(c.div, f / 16), qt = page_of_group(c.div, jj / 16);
  const int rt = w.rank[(int64_t)e * c.M + qt];
  const int pt = rt < 0 ? old[qt] : w.free[rt];
  RowMove m;
  m.from = old[qf] * c.page_u4 + head + (int64_t)(f - qf * c.page) * PPR;
  m.to = j < K && (f != j || rt >= 0) ? pt * c.page_u4 + head + (int64_t)(jj - qt * c.page) * PPR : -1;
  return m;
}

// Workgroups below n_state: entries, counts and lengths of the listed slots.  The others move
// rows, K and V of a (slot, head) together, a chunk at a time.  As src[j] >= j and src
// increases, a row that a chunk overwrites is read by that chunk and earlier ones only.
//
// Many (slot, head) pairs: a workgroup takes whole ones, its chunks in ascending order; a
// chunk's stores wait for its own loads (and a barrier, for the other waves'), while the next
// chunk's loads are under way.  Few: workgroups take single chunks of a pair, by ticket;
// a chunk's rows are all in registers before it says so, and its stores wait until the chunks
// before it whose sources reach into it have said so.  They have lower tickets, so they
// are with running workgroups, which wait for nothing before they speak: every wait
// ends.  Bound by HBM: each row is read once and written once.  2304 pairs of 4096 rows of 128
// (bf16): 1.9 ms, 5.1 TB/s (a copy kernel reaches 6.2); 32 pairs of 2048 rows: 15 us, 4.4 TB/s.
template <int PPR>
__global__ __launch_bounds__(kBlock) void page_compact_kernel(PageView c, const int32_t* __restrict__ map,
                                                              const int32_t* __restrict__ src, int K,
                                                              CompactState w, int n_state) {
  constexpr int kChunk = chunk_rows(PPR);
  constexpr int kRows = kBlock / PPR;        // rows of one load by the workgroup
  constexpr int U = kChunk / kRows;
  __shared__ RowMove s_move[4][kChunk];
  __shared__ int s_ticket;
  if (!w.head[0]) return;
  const int n = w.head[1], kept = pages_for(c, K);
  if ((int)blockIdx.x < n_state) {
    for (int e = blockIdx.x; e < n; e += n_state) {
      const int s = w.slot[e], old = pages_for(c, w.len[e]);
      int32_t* row = c.table + (int64_t)s * c.M;
      for (int j = threadIdx.x; j < old; j += kBlock) {
        const int p = w.old[(int64_t)e * c.M + j];
        const int r = j < kept ? w.rank[(int64_t)e * c.M + j] : 0;
        if (j < kept && r < 0) continue;
        atomicSub(&c.ref[p], 1);
        const int q = j < kept ? w.free[r] : -1;
        row[j] = q;
        if (q >= 0) c.ref[q] = 1;
      }
      if (threadIdx.x == 0) c.len[s] = K;
    }
    return;
  }
  const int tid = threadIdx.x, col = tid % PPR, r0 = tid / PPR;
  const int64_t items = (int64_t)n * c.H;
  const int chunks = (K + kChunk - 1) / kChunk;
  auto head_of = [&](int64_t i, int& e) {
    e = (int)(i / c.H);
    return src + ((int64_t)map[w.slot[e]] * c.H + i % c.H) * K;
  };
  uint4 a[2][U], b[2][U];
  auto load = [&](const RowMove* mv, uint4 (&x)[U], uint4 (&y)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = mv[r0 + u * kRows].from + col;
      x[u] = load_once(c.k + at);
      y[u] = load_once(c.v + at);
    }
  };
  auto arrived = [&](uint4 (&x)[U], uint4 (&y)[U]) {   // waits for the wave's loads
#pragma unroll
    for (int u = 0; u < U; ++u) {
      asm volatile("" : "+v"(x[u].x), "+v"(x[u].y), "+v"(x[u].z), "+v"(x[u].w));
      asm volatile("" : "+v"(y[u].x), "+v"(y[u].y), "+v"(y[u].z), "+v"(y[u].w));
    }
  };
  auto store = [&](const RowMove* mv, const uint4 (&x)[U], const uint4 (&y)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = mv[r0 + u * kRows].to;
      if (at >= 0) {
        store_once(c.k + at + col, x[u]);
        store_once(c.v + at + col, y[u]);
      }
    }
  };

  if (items == 0) return;
  if (items < kFewItems) {
    // one counter to a pair: on a single one the workgroups' atomics queued (60 us for 32 pairs
    // of 32 chunks)
    const int n_block = (int)(gridDim.x - n_state), per = n_block / (int)items;
    const int i = (int)(blockIdx.x - n_state) % (int)items;
    if ((int)(blockIdx.x - n_state) >= per * (int)items) return;
    int e;
    const int32_t* sr = head_of(i, e);
    int32_t* said = w.said + (int64_t)i * chunks;
    for (int taken = 0; taken < chunks; taken += per) {
      __syncthreads();   // the chunk before is stored
      if (tid == 0) s_ticket = atomicAdd(&w.ticket[i * kTicketGap], 1);
      __syncthreads();
      const int ch = s_ticket;
      if (ch >= chunks) return;
      if (tid < kChunk) {
        const int j = ch * kChunk + tid;
        s_move[0][tid] = row_move<PPR>(c, w, e, (i % c.H) * c.head_u4, K, j, sr[min(j, K - 1)]);
      }
      __syncthreads();
      load(s_move[0], a[0], b[0]);
      arrived(a[0], b[0]);
      __syncthreads();   // every wave's
      if (tid == 0) __hip_atomic_store(&said[ch], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      // the chunks before, nearest first, as long as their last source is in this chunk's rows
      if (tid < kWave) {
        for (int p = ch - 1 - tid;; p -= kWave) {
          const bool reaches = p >= 0 && sr[(p + 1) * kChunk - 1] >= ch * kChunk;
          if (reaches)
            while (__hip_atomic_load(&said[p], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == 0)
              __builtin_amdgcn_s_sleep(1);
          if (__ballot(!reaches)) break;
        }
      }
      __syncthreads();
      store(s_move[0], a[0], b[0]);
    }
    return;
  }

  for (int64_t i = blockIdx.x - n_state; i < items; i += gridDim.x - n_state) {
    int e;
    const int32_t* sr = head_of(i, e);
    const int64_t head = (i % c.H) * c.head_u4;
    // the moves of chunk x into its place of four; their sources read a chunk earlier
    int ahead = tid < kChunk ? sr[min(tid, K - 1)] : 0;
    auto moves = [&](int x) {
      if (tid < kChunk) {
        const int j = x * kChunk + tid;
        s_move[x % 4][tid] = row_move<PPR>(c, w, e, head, K, j, ahead);
        ahead = sr[min(j + kChunk, K - 1)];
      }
    };
    __syncthreads();   // the item before has read its moves
    moves(0);
    moves(1);
    __syncthreads();
    load(s_move[0], a[0], b[0]);
    for (int x = 0; x < chunks; x += 2) {
#pragma unroll
      for (int o = 0; o < 2; ++o) {
        const int y = x + o;
        if (y >= chunks) break;
        moves(y + 2);   // ahead of the loads, whose end its own look-ups would wait for
        if (y + 1 < chunks) load(s_move[(y + 1) % 4], a[1 - o], b[1 - o]);
        arrived(a[o], b[o]);
        __syncthreads();
        store(s_move[y % 4], a[o], b[o]);
      }
    }
  }
}

int row_pieces(const vase_pages& c) { return c.d * (c.dtype == VASE_BF16 ? 2 : 4) / 16; }

template <typename F>
hipError_t by_row(const vase_pages& c, F f) {   // 16-byte pieces of a row
  const int ppr = row_pieces(c);
  if (ppr == 8) f(std::integral_constant<int, 8>());
  else if (ppr == 16) f(std::integral_constant<int, 16>());
  else f(std::integral_constant<int, 32>());
  return hipGetLastError();
}

}  // namespace

hipError_t launch_page_write(const vase_pages& c, const void* k_new, const void* v_new,
                             int64_t new_stride, const int32_t* cu, int T, uint32_t* status,
                             hipStream_t stream) {
  const PageView w = page_view(c);
  return by_row(c, [&](auto ppr) {
    constexpr int P = decltype(ppr)::value;
    const dim3 grid((T + kBlock / kWave - 1) / (kBlock / kWave), (c.H * P + kWritePieces - 1) / kWritePieces);
    hipLaunchKernelGGL((page_write_kernel<P>), grid, dim3(kBlock), 0, stream, w,
                       static_cast<const uint4*>(k_new), static_cast<const uint4*>(v_new),
                       new_stride / (c.dtype == VASE_BF16 ? 8 : 4), cu, T, status);
  });
}

size_t page_resize_bytes(const vase_pages& c) {
  return sizeof(int32_t) * (kHead + 5 * (size_t)c.S + (size_t)c.n_pages);
}

hipError_t launch_page_resize(const vase_pages& c, const int32_t* new_len, void* ws, uint32_t* status,
                              hipStream_t stream) {
  const PageView v = page_view(c);
  const ResizePlan w = resize_plan(ws, c.S);
  hipLaunchKernelGGL(page_resize_plan_kernel, dim3(1), dim3(kPlanBlock), 0, stream, v, new_len, w, status);
  const int64_t copies = (int64_t)c.S * c.H;
  return by_row(c, [&](auto ppr) {
    constexpr int P = decltype(ppr)::value;
    hipLaunchKernelGGL((page_resize_kernel<P>), dim3((unsigned)(c.S + (copies < kCopyBlocks ? copies : kCopyBlocks))),
                       dim3(kBlock), 0, stream, v, new_len, w, status);
  });
}

hipError_t launch_page_fork(const vase_pages& c, const int32_t* parent, uint32_t* status,
                            hipStream_t stream) {
  hipLaunchKernelGGL(page_fork_kernel, dim3(c.S), dim3(kBlock), 0, stream, page_view(c), parent, status);
  return hipGetLastError();
}

size_t page_compact_bytes(const vase_pages& c) {
  const int chunk = chunk_rows(row_pieces(c));
  const size_t chunks = ((size_t)c.M * c.page + chunk - 1) / chunk;
  return sizeof(int32_t) * (kHead + 2 * (size_t)c.S + 2 * (size_t)c.S * c.M + (size_t)c.n_pages +
                            few_pairs(c) * (kTicketGap + chunks));
}

hipError_t launch_page_compact(const vase_pages& c, const int32_t* map, const int32_t* src, int n_map,
                               int K, void* ws, uint32_t* status, hipStream_t stream) {
  const PageView v = page_view(c);
  const CompactState w = compact_state(ws, c);
  const int chunk = chunk_rows(row_pieces(c));
  hipLaunchKernelGGL(page_compact_plan_kernel, dim3(1), dim3(kPlanBlock), 0, stream, v, map, n_map, K,
                     chunk, w, status);
  const int n_state = c.S < 1024 ? c.S : 1024;
  // one workgroup per pair, or per chunk where pairs are few, up to a chip's fill of them
  const int64_t pairs = (int64_t)c.S * c.H;
  int64_t movers = pairs < kFewItems ? pairs * ((K + chunk - 1) / chunk) : pairs;
  const int64_t most = pairs < kFewItems ? 2048 : 8192;
  if (movers > most) movers = most;
  return by_row(c, [&](auto ppr) {
    constexpr int P = decltype(ppr)::value;
    hipLaunchKernelGGL((page_compact_kernel<P>), dim3((unsigned)(n_state + movers)),
                       dim3(kBlock), 0, stream, v, map, src, K, w, n_state);
  });
}

}  // namespace vase
