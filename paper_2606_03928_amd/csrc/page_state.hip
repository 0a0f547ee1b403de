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

// ---------------------------------------------------------------------------
// write: one wave per token and group of heads, K and V.  Bound by HBM (each row read
// once, written once); the token's slot is found by the wave's lanes together.
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
  const int row = slot_len(c, s) - (cu[s + 1] - t);
  const int q = row < 0 ? 0 : page_of_group(c.div, row / 16);
  const int p = row < 0 || t < cu[s] || q >= c.M ? -1 : c.table[(int64_t)s * c.M + q];
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
// changes the state, all of it or nothing.
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

// the lowest `want` pages without a count into list, in order; how many there are of them
__device__ int list_free(const int32_t* __restrict__ ref, int n_pages, int want, int32_t* list,
                         int* s_count /* [8 * kPlanWaves] */) {
  constexpr int U = 8;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int found = 0;
  for (int64_t base = 0; base < n_pages && found < want; base += U * kPlanBlock) {
    uint64_t m[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t p = base + u * kPlanBlock + threadIdx.x;
      const int r = ref[p < n_pages ? p : n_pages - 1];
      m[u] = __ballot(p < n_pages && r == 0);
    }
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
  __shared__ int s_count[8 * kPlanWaves];
  constexpr int kCow = 48;   // sums of two numbers in one: pages below bit 48, copies above
  const int cap = c.M * c.page;
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
    full = list_free(c.ref, c.n_pages, (int)need_all, w.free, s_count) < need_all;
  if (threadIdx.x == 0) {
    w.head[0] = !bad && !full;
    w.head[1] = n_cow;
    if (bad) raise(status, VASE_STATUS_PAGE_BAD);
    else if (full) raise(status, VASE_STATUS_PAGE_FULL);
  }
}

// Workgroups below c.S: a slot's entries, counts and length.  The others: the rows of the
// pages that slots take for their own, a head of one page at a time.
template <int PPR>
__global__ __launch_bounds__(kBlock) void page_resize_kernel(PageView c,
                                                             const int32_t* __restrict__ new_len,
                                                             ResizePlan w, uint32_t* status) {
  if (!w.head[0]) return;
  if ((int)blockIdx.x < c.S) {
    const int s = blockIdx.x;
    const int L = c.len[s], t = new_len[s];
    if (t < 0 || t == L) return;
    __syncthreads();   // every thread has the old length
    int32_t* row = c.table + (int64_t)s * c.M;
    const int old = pages_for(c, L), now = pages_for(c, t);
    if (t > L) {
      const int first = w.begin[s], off = w.off[s];
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
  const int64_t items = (int64_t)w.head[1] * c.H;
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
// fork: a workgroup per slot
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
struct CompactState {   // in the workspace, int32 each
  int32_t *head;
  int32_t *slot, *len;  // [S]: the slots to compact and their lengths
  int32_t *old, *rank;  // [S][M] by list place: the entries, and which free page replaces each (-1: none)
  int32_t *free;        // [n_pages]
};
CompactState compact_state(void* ws, int S, int M) {
  int32_t* p = static_cast<int32_t*>(ws) + kHead;
  const size_t sm = (size_t)S * M;
  return CompactState{static_cast<int32_t*>(ws), p, p + S, p + 2 * S, p + 2 * S + sm, p + 2 * S + 2 * sm};
}

__global__ __launch_bounds__(kPlanBlock) void page_compact_plan_kernel(PageView c,
                                                                       const int32_t* __restrict__ map,
                                                                       int n_map, int K, CompactState w,
                                                                       uint32_t* status) {
  __shared__ long long s_wave[kPlanWaves];
  __shared__ int s_count[8 * kPlanWaves];
  __shared__ int s_most;
  if (threadIdx.x == 0) s_most = 0;
  __syncthreads();
  bool bad = false;
  int n = 0;
  for (int base = 0; base < c.S; base += kPlanBlock) {
    const int s = base + threadIdx.x;
    const int m = s < c.S ? map[s] : -1;
    const int L = m >= 0 ? c.len[s] : 0;
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
  const int most = s_most, kept = pages_for(c, K);
  const int64_t pairs = bad ? 0 : (int64_t)n * most;
  long long need = 0;
  for (int64_t base = 0; base < pairs; base += kPlanBlock) {
    const int64_t i = base + threadIdx.x;
    const int e = (int)(i / most), j = (int)(i % most);
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
  if (!bad && !full && need > 0) full = list_free(c.ref, c.n_pages, (int)need, w.free, s_count) < need;
  if (threadIdx.x == 0) {
    w.head[0] = !bad && !full;
    w.head[1] = n;
    if (bad) raise(status, VASE_STATUS_PAGE_BAD);
    else if (full) raise(status, VASE_STATUS_PAGE_FULL);
  }
}

// Workgroups below n_state: entries, counts and lengths of listed slots.  The others move
// rows, one (slot, head, pool) at a time, in ascending chunks.  As src[j] >= j and src
// increases, a row that a chunk overwrites is read by that chunk or an earlier one only,
// so a chunk's stores wait for its own loads (and a barrier, for the other waves'), and
// the next chunk's loads need not wait for them.
template <int PPR>
__global__ __launch_bounds__(kBlock) void page_compact_kernel(PageView c, const int32_t* __restrict__ map,
                                                              const int32_t* __restrict__ src, int K,
                                                              CompactState w, int n_state) {
  constexpr int U = 8;
  constexpr int kRows = kBlock / PPR;        // rows of one load by the workgroup
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
  const int col = threadIdx.x % PPR, r0 = threadIdx.x / PPR;
  const int64_t items = (int64_t)n * c.H * 2;
  for (int64_t i = blockIdx.x - n_state; i < items; i += gridDim.x - n_state) {
    const int e = (int)(i / (2 * c.H)), h = (int)(i % (2 * c.H)) / 2;
    uint4* pool = i % 2 ? c.v : c.k;
    const int s = w.slot[e], L = w.len[e];
    const int32_t* sr = src + ((int64_t)map[s] * c.H + h) * K;
    const int32_t* old = w.old + (int64_t)e * c.M;
    const int32_t* rank = w.rank + (int64_t)e * c.M;
    const int64_t head = h * c.head_u4 + col;
    for (int c0 = 0; c0 < K; c0 += U * kRows) {
      uint4 x[U];
      int64_t to[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int j = c0 + r0 + u * kRows;
        const int jj = min(j, K - 1);
        const int f = min(max(sr[jj], 0), L - 1);
        const int qf = page_of_group(c.div, f / 16), qt = page_of_group(c.div, jj / 16);
        const int pf = old[qf], rt = rank[qt];
        const int pt = rt < 0 ? old[qt] : w.free[rt];
        x[u] = pool[pf * c.page_u4 + head + (int64_t)(f - qf * c.page) * PPR];
        to[u] = j < K && (f != j || rt >= 0)
                    ? pt * c.page_u4 + head + (int64_t)(jj - qt * c.page) * PPR
                    : -1;
      }
#pragma unroll
      for (int u = 0; u < U; ++u)   // the loads are done before the barrier
        asm volatile("" : "+v"(x[u].x), "+v"(x[u].y), "+v"(x[u].z), "+v"(x[u].w));
      __syncthreads();
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (to[u] >= 0) pool[to[u]] = x[u];
    }
  }
}

template <typename F>
hipError_t by_row(const vase_pages& c, F f) {   // 16-byte pieces of a row
  const int ppr = c.d * (c.dtype == VASE_BF16 ? 2 : 4) / 16;
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
    hipLaunchKernelGGL((page_resize_kernel<P>), dim3((unsigned)(c.S + (copies < 1024 ? copies : 1024))),
                       dim3(kBlock), 0, stream, v, new_len, w, status);
  });
}

hipError_t launch_page_fork(const vase_pages& c, const int32_t* parent, uint32_t* status,
                            hipStream_t stream) {
  hipLaunchKernelGGL(page_fork_kernel, dim3(c.S), dim3(kBlock), 0, stream, page_view(c), parent, status);
  return hipGetLastError();
}

size_t page_compact_bytes(const vase_pages& c) {
  return sizeof(int32_t) * (kHead + 2 * (size_t)c.S + 2 * (size_t)c.S * c.M + (size_t)c.n_pages);
}

hipError_t launch_page_compact(const vase_pages& c, const int32_t* map, const int32_t* src, int n_map,
                               int K, void* ws, uint32_t* status, hipStream_t stream) {
  const PageView v = page_view(c);
  const CompactState w = compact_state(ws, c.S, c.M);
  hipLaunchKernelGGL(page_compact_plan_kernel, dim3(1), dim3(kPlanBlock), 0, stream, v, map, n_map, K, w,
                     status);
  const int n_state = c.S < 1024 ? c.S : 1024;
  const int64_t items = (int64_t)c.S * c.H * 2;
  return by_row(c, [&](auto ppr) {
    constexpr int P = decltype(ppr)::value;
    hipLaunchKernelGGL((page_compact_kernel<P>), dim3((unsigned)(n_state + (items < 8192 ? items : 8192))),
                       dim3(kBlock), 0, stream, v, map, src, K, w, n_state);
  });
}

}  // namespace vase
