// page_attn.hip -- attention of new rows over a paged cache (Eq. 1), gfx950.
//
// Of one slot and one KV head, the n new tokens' G query heads are n * G query rows that read
// the same K and V rows; row r is head r % G of token r / G.  Scores are taken
// transposed, S^T = K Q^T, so that an MFMA result holds one query row per lane column: a
// lane keeps its row's running maximum and sum, and the probabilities it holds are, as they
// stand, the B operand of O^T = V^T P^T, whose A operand reads V^T out of row-major LDS
// (bf16: ds_read_b64_tr_b16) in the same order of keys.  No probability moves
// between lanes or through LDS.
//
// Many rows are bound by MFMAs and exponentials: page_wide_kernel takes 256 (bf16) and
// page_tile_kernel 128 (fp32) to a workgroup.  Few (tokens of decoding) are bound by the K
// and V rows that they read: page_few_kernel takes 16.  Where workgroups would be too few or too
// uneven to fill the chip, the keys are split, and partial (m, l, O) are joined in the order
// of their keys by a launch behind: ranges of one length (few), equal shares of all tiles.
//
// Masked keys take p = 0 by a select on the score, and V rows behind the slot's end are
// zeroed where they are staged.  A later token's V row may hold an infinity or a NaN, which
// p = 0 would not keep out of a product: in tiles whose keys not every row sees, V rows are
// looked through as they are staged, such values go in as 0, and each output column
// keeps the first key that had one of either sign (a NaN counts as both); rows that see that
// key have the infinity, or of both signs NaN, added at the end.
#include "page_internal.hpp"

#include <type_traits>
#include <utility>

namespace vase {
namespace {

typedef __bf16 pbf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 pbf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 pbf16x2 __attribute__((ext_vector_type(2)));
typedef short ps16x4 __attribute__((ext_vector_type(4)));
typedef unsigned short pu16x2 __attribute__((ext_vector_type(2)));
typedef float pf32x8 __attribute__((ext_vector_type(8)));
typedef float pf32x16 __attribute__((ext_vector_type(16)));
typedef float pf32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));   // 16 bytes of a row
typedef __attribute__((address_space(3))) ps16x4 lds_s16x4;

#define INLINE __attribute__((always_inline))   // of lambdas: what they capture stays in registers

constexpr int kBlock = 256;
constexpr int kWaves = kBlock / kWave;
constexpr int kTileRows = 32 * kWaves;   // query rows of a tile workgroup
constexpr int kFewRows = 16;             // query rows of a few-row workgroup
constexpr int kMaxSplit = 64;
constexpr float kLn2 = 0.69314718055994531f;

struct AttnArgs {
  PageView c;
  const u4* q;
  int64_t q_u4;            // pieces from a token's queries to the next one's
  const int32_t* cu;
  int T, G, HG;
  int causal;
  void* out;
  float* lse;
  // partials.  few: [range][T][HG] of D and of 2; tile: [workgroup][2][its rows] likewise
  float *part_o, *part_ml;
  int32_t* sums;           // tile, shares: [n_tile + 1], the sums of the row tiles' triples
  int n_tile;              // row tiles, at most
  int n_split, keys;       // few: key ranges
  int by_slot;             // few: a slot's rows are one row tile
  int shares;              // tile: workgroups that share the work (0: one to a row tile and head)
  float scale_log2;
  uint32_t* status;
};

// x, the same in all lanes, kept for the wave as a whole (what comes out of LDS is not by itself)
__device__ __forceinline__ int of_wave(int x) { return __builtin_amdgcn_readfirstlane(x); }

// A slot's share of the batch, read as it stands but kept inside the caller's arrays.
struct Span {
  int s, c0, n, L;   // slot, first token, tokens, rows
  __device__ __forceinline__ Span(const AttnArgs& a, const int32_t* cu, int slot) : s(slot) {
    c0 = min(max(cu[s], 0), a.T);
    n = min(max(cu[s + 1], c0), a.T) - c0;
    L = slot_len(a.c, s);
  }
  __device__ __forceinline__ Span(const AttnArgs& a, int slot) : Span(a, a.cu, slot) {}
  __device__ __forceinline__ Span of_all() const {   // where all lanes have the same
    Span x = *this;
    x.s = of_wave(s);
    x.c0 = of_wave(c0);
    x.n = of_wave(n);
    x.L = of_wave(L);
    return x;
  }
  // for a workgroup that has rows of the slot: a length that was out of range
  __device__ __forceinline__ void check(const AttnArgs& a) const {
    if (threadIdx.x == 0 && a.status && a.c.len[s] != L) atomicOr(a.status, VASE_STATUS_PAGE_BAD);
  }
  // rows that token i sees
  __device__ __forceinline__ int sees(const AttnArgs& a, int i) const {
    return a.causal ? max(L - n + i + 1, 0) : L;
  }
};

// Row tiles of R rows: those of slot s begin at number floor(cu[s] G / R) + min(s, cu[s]).  No more
// than min(s, cu[s]) slots before it have tokens, so there is room for a last tile of each, a
// tile's slot is found in cu alone, and slots without tokens behind the last add no tiles.
template <int R>
__device__ __forceinline__ int first_tile(const AttnArgs& a, const int32_t* cu, int s) {
  const int c = min(max(cu[s], 0), a.T);
  return (int)((int64_t)c * a.G / R) + min(s, c);
}
template <int R>
__device__ __forceinline__ int first_tile(const AttnArgs& a, int s) {
  return first_tile<R>(a, a.cu, s);
}

// Where the 16-row groups of a slot lie: lane l holds the address of group g0 + l of head h in
// the K pool, 64 groups at a time.
template <int PPR>
struct GroupBases {
  uint32_t lo, hi;
  int g0;
  __device__ __forceinline__ void fill(const AttnArgs& a, const Span& sp, int h, int g) {
    const int lane = threadIdx.x % kWave;
    const int gl = min(g + lane, max(sp.L - 1, 0) / 16);   // groups behind the last read the last
    const int q = page_of_group(a.c.div, gl);
    int p = a.c.table[(int64_t)sp.s * a.c.M + q];
    if (!valid_page(a.c, p)) {
      if (a.status) atomicOr(a.status, VASE_STATUS_PAGE_BAD);
      p = 0;
    }
    const uint64_t at = reinterpret_cast<uint64_t>(
        a.c.k + (p * a.c.page_u4 + h * a.c.head_u4 + (int64_t)(gl * 16 - q * a.c.page) * PPR));
    lo = (uint32_t)at;
    hi = (uint32_t)(at >> 32);
    g0 = g;
  }
  // for at() of groups [first, last]; at most 64 of them
  __device__ __forceinline__ void reach(const AttnArgs& a, const Span& sp, int h, int first, int last) {
    if (last >= g0 + kWave) fill(a, sp, h, first);
  }
  __device__ __forceinline__ uint64_t at(int g) const {
    const uint32_t x = __builtin_amdgcn_readlane(lo, g - g0), y = __builtin_amdgcn_readlane(hi, g - g0);
    return (uint64_t)y << 32 | x;
  }
};
// 16 bytes at a uniform address and a lane's offset
__device__ __forceinline__ u4 load_at(uint64_t address, uint32_t offset) {
  return *reinterpret_cast<const u4*>(reinterpret_cast<const char*>(address) + offset);
}
// the same of what is not read again soon
__device__ __forceinline__ u4 load_once_at(uint64_t address, uint32_t offset) {
  return __builtin_nontemporal_load(reinterpret_cast<const u4*>(reinterpret_cast<const char*>(address) + offset));
}
// from an address in the K pool to the same row's in the V pool
__device__ __forceinline__ uint64_t to_v(const PageView& c) {
  return reinterpret_cast<uint64_t>(c.v) - reinterpret_cast<uint64_t>(c.k);
}

// f(0) .. f(N - 1), the number a constant in each
template <int... I, typename F>
__device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F f) {
  (f(std::integral_constant<int, I>()), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F f) {
  each_of(std::make_integer_sequence<int, N>(), f);
}

// x, for code that only some iterations run: what is computed from it is computed there, and
// takes no register in the others
__device__ __forceinline__ int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// the lane's number, computed anew: no register holds it from one use to the next
__device__ __forceinline__ int lane_here() {
  int x;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=&v"(x));
  return x;
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// exp2((x - top) scale) for x <= top, also where both are infinite: 1
__device__ __forceinline__ float weight(float x, float top, float scale = 1.f) {
  return x == top ? 1.f : exp2_((x - top) * scale);
}
// what is taken from scores whose maximum is m, in log2 units: finite, so that a score of +inf
// stays one and the sum with it, and scores of -inf alone count as none
__device__ __forceinline__ float reference(float m, float scale) {
  return __builtin_amdgcn_fmed3f(m * scale, -3.4028234663852886e38f, 3.4028234663852886e38f);
}
// ln of the sum l of probabilities over 2^m
__device__ __forceinline__ float lse_of(float m, float l) {
  return l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;   // NaN stays
}

// Four outputs of a row from d0 on: the result, or (part: the row's place) a partial.
template <typename T>
__device__ __forceinline__ void store4(const AttnArgs& a, float* part, int64_t at, const float (&o)[4]) {
  if (part) {
    *reinterpret_cast<float4*>(part) = make_float4(o[0], o[1], o[2], o[3]);
  } else if constexpr (std::is_same<T, float>::value) {
    *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = make_float4(o[0], o[1], o[2], o[3]);
  } else {
    ushort4 w;
    w.x = f32_to_bf16_bits(o[0]);
    w.y = f32_to_bf16_bits(o[1]);
    w.z = f32_to_bf16_bits(o[2]);
    w.w = f32_to_bf16_bits(o[3]);
    *reinterpret_cast<ushort4*>(static_cast<uint16_t*>(a.out) + at) = w;
  }
}
// its maximum (in scaled log2 units) and sum
__device__ __forceinline__ void store_ml(const AttnArgs& a, float* part, int64_t row, float m, float l) {
  if (part) *reinterpret_cast<float2*>(part) = make_float2(m, l);
  else if (a.lse) a.lse[row] = lse_of(m, l);
}

// ---------------------------------------------------------------------------
// Values of V that no product with 0 keeps out: taken out of a piece of key `key`'s row
// (columns col on), the first key of each column and sign noted in bad.
// ---------------------------------------------------------------------------
constexpr int kNoKey = 0x7fffffff;
template <int D>
struct BadKeys {
  int pos[D], neg[D];
  __device__ __forceinline__ void clear(int tid) {
    if (tid < D) pos[tid] = neg[tid] = kNoKey;
  }
  __device__ __forceinline__ void note(int col, int key, uint32_t fp32) {
    const bool nan = (fp32 & 0x7fffffffu) > 0x7f800000u;
    if (nan || !(fp32 >> 31)) atomicMin(&pos[col], key);
    if (nan || fp32 >> 31) atomicMin(&neg[col], key);
  }
  // is there one among the keys below end, in any column; the same in all lanes
  __device__ __forceinline__ bool any(int end) const {
    const int lane = threadIdx.x % kWave;
    int first = min(pos[lane], neg[lane]);
    if constexpr (D > kWave) first = min(first, min(pos[lane + D - kWave], neg[lane + D - kWave]));
    return __ballot(first < end) != 0;
  }
  // what those below end add to an output: -0, which leaves any output as it is, for none
  __device__ __forceinline__ float sum(int col, int end) const {
    return (pos[col] < end ? INFINITY : -0.f) + (neg[col] < end ? -INFINITY : -0.f);
  }
};
__device__ __forceinline__ bool is_bad(uint32_t fp32) { return (fp32 & 0x7fffffffu) >= 0x7f800000u; }
template <typename T, int D>
__device__ __forceinline__ void scrub(u4& w, int key, int col, BadKeys<D>& bad) {
  if constexpr (std::is_same<T, float>::value) {
    if (is_bad(w.x) || is_bad(w.y) || is_bad(w.z) || is_bad(w.w)) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (is_bad(w[i])) {
          bad.note(col + i, key, w[i]);
          w[i] = 0;
        }
    }
  } else {
    // the largest exponent and fraction of the low and of the high halves
    pu16x2 most = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      most = __builtin_elementwise_max(most, __builtin_bit_cast(pu16x2, w[i] & 0x7fff7fffu));
    if (most.x >= 0x7f80 || most.y >= 0x7f80) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (is_bad(w[i] << 16)) {
          bad.note(col + 2 * i, key, w[i] << 16);
          w[i] &= 0xffff0000u;
        }
        if (is_bad(w[i])) {
          bad.note(col + 2 * i + 1, key, w[i] & 0xffff0000u);
          w[i] &= 0xffffu;
        }
      }
    }
  }
}

// V^T operand: two transposed reads (4 keys each) of row-major LDS
__device__ __forceinline__ pbf16x8 read_vt(const u4* base, int byte0, int byte1) {
  const char* p = reinterpret_cast<const char*>(base);
  const ps16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + byte0));
  const ps16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + byte1));
  return __builtin_bit_cast(pbf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
}

// ---------------------------------------------------------------------------
// The tile kernel (fp32).  A wave keeps 32 query rows (one per lane column) and their O^T in
// registers; K and V tiles of 32 keys pass through two LDS buffers, the next tile's
// rows on their way to registers while this one is used.  8 slots of 192 tokens over 2100 rows, 4
// heads to each of 8 KV heads of 128: 690 us, 73 TFLOP/s of the 153 that a large fp32 product reaches.
// An operand of K or V is read from LDS, waited for and used by 4 MFMAs, one after the other, and
// a wave has its SIMD to itself (d 128), so that nothing hides LDS's latency.
// ---------------------------------------------------------------------------
template <typename T, int D>
struct Tile {
  static constexpr bool kBf16 = std::is_same<T, bf16_t>::value;
  static constexpr int BN = kBf16 ? 64 : 32;          // keys
  static constexpr int PPR = D * (kBf16 ? 2 : 4) / 16;
  static constexpr int kPieces = BN * PPR;
  static constexpr int NP = kPieces / kBlock;         // of each, per thread
  static constexpr int KS = PPR / 2;                  // pairs of pieces (one to a half wave)
  static constexpr int NB = D / 32;                   // O^T blocks of 32 outputs
  // LDS place of piece p of row r: pieces of a 256-byte line are permuted by the line, so
  // that 16 rows' piece p (K), or the parts of 4 rows that one transposed read takes
  // (V; fp32: a piece of rows r and r + 4), lie in different banks
  __device__ static __forceinline__ int k_at(int r, int p) {
    if constexpr (PPR == 8) return r / 2 * 16 + (((r % 2) * 8 + p) ^ ((r / 2) & 15));
    else return r * PPR + (p ^ (r & 15));
  }
  __device__ static __forceinline__ int v_at(int r, int p) {
    if constexpr (!kBf16) return r * PPR + (p ^ (8 * ((r >> 2) & 1)));
    else if constexpr (PPR == 8) return r / 2 * 16 + (((r % 2) * 8 + p) ^ (4 * ((r >> 1) & 1)));
    else return r * PPR + (p ^ (4 * (r & 3)));
  }
};

// Shares: the (head, row tile, key tile) triples in that order, cut into equal parts for at most
// a.shares workgroups and none below kLeastShare triples.  A row tile's beginning and end (Q, the
// first loads, its output: 11 us, where a key tile takes 1.9) count as kSetup triples before
// its first: with none a fresh prompt's short tiles made some parts twice as long as others
// (3200 tokens: 202 us, with 6 under 120).  The number is bf16's: us with 2, 6 and 12, a mixed
// step of 16 slots over 600 to 4224 rows 114, 104 and 107 (d 64: 80, 74, 78), two fresh prompts of
// 1600 tokens 66, 57 and 61 (50, 43, 47).  fp32, whose tiles of 32 keys take longer, would have a
// smaller one: 432, 452 and 481 (189, 194, 205), two of 1100 tokens 80, 94 and 107 (50, 52, 58).
// What a workgroup cannot finish of a row tile (its first and last at most) it leaves as a partial.
constexpr int kMaxTiles = 1023;    // row tiles whose sums a workgroup keeps
constexpr int kLeastShare = 4;
constexpr int kSetup = 6;
struct Shares {
  int64_t total;   // triples
  int n;           // parts
  __device__ __forceinline__ Shares(const AttnArgs& a, int per_head) : total((int64_t)per_head * a.c.H) {
    n = (int)min((int64_t)a.shares, max(total / kLeastShare, (int64_t)1));
  }
  __device__ __forceinline__ int64_t begin(int i) const { return total * i / n; }
  // the part that triple x is in
  __device__ __forceinline__ int of(int64_t x) const { return (int)((x * n + n - 1) / total); }
};

// cu, in which a slot is searched for often: S <= kMaxTiles
__device__ __forceinline__ void keep_cu(const AttnArgs& a, int32_t* s_cu) {
  for (int x = threadIdx.x; x <= a.c.S; x += kBlock) s_cu[x] = a.cu[x];
}

// A row tile's triples: 0 of a number that no rows have, otherwise one key tile at least.
template <int BN, int R>
__device__ __forceinline__ int key_tiles(const AttnArgs& a, const int32_t* s_cu, int tile) {
  int lo = 0, hi = a.c.S;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (first_tile<R>(a, s_cu, mid) <= tile) lo = mid;
    else hi = mid;
  }
  const Span sp(a, s_cu, lo);
  const int rows = sp.n * a.G, r0 = (tile - first_tile<R>(a, s_cu, lo)) * R;
  if (r0 < 0 || r0 >= rows) return 0;
  return kSetup + max((sp.sees(a, (min(r0 + R, rows) - 1) / a.G) + BN - 1) / BN, 1);
}

// cu into s_cu, the sums of the row tiles' triples into s_sum (those before tile x at x), and
// this workgroup's triples; false: it has none.
template <int BN, int R>
__device__ __forceinline__ bool share_out(const AttnArgs& a, uint32_t id, int32_t* s_cu, int* s_sum, int* s_wave,
                                          int64_t& next, int64_t& end) {
  constexpr int E = (kMaxTiles + 1) / kBlock;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  keep_cu(a, s_cu);
  __syncthreads();
  for (int x = threadIdx.x; x <= kMaxTiles; x += kBlock) s_sum[x] = x < a.n_tile ? key_tiles<BN, R>(a, s_cu, x) : 0;
  __syncthreads();
  int mine[E], sum = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    mine[e] = sum;
    sum += s_sum[threadIdx.x * E + e];
  }
  int upto = sum;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int z = __shfl_up(upto, o, kWave);
    if (lane >= o) upto += z;
  }
  if (lane == kWave - 1) s_wave[wave] = upto;
  __syncthreads();
  int before = upto - sum;
  for (int w = 0; w < wave; ++w) before += s_wave[w];
#pragma unroll
  for (int e = 0; e < E; ++e) s_sum[threadIdx.x * E + e] = before + mine[e];
  __syncthreads();
  if (id == 0)
    for (int x = threadIdx.x; x <= a.n_tile; x += kBlock) a.sums[x] = s_sum[x];
  const Shares sh(a, of_wave(s_sum[a.n_tile]));
  if (sh.total == 0 || (int)id >= sh.n) return false;
  auto begin = [&](int i) {
    const int64_t x = sh.begin(i);
    return (int64_t)of_wave((int)(x >> 32)) << 32 | (uint32_t)of_wave((int)x);
  };
  next = begin(id);
  end = begin(id + 1);
  return true;
}

// The key tiles [kt0, kt1) of a row tile and head; whole: all that there are.
struct Segment {
  int tile, h, kt0, kt1;
  bool whole;
};
__device__ __forceinline__ Segment next_segment(const AttnArgs& a, const int* s_sum, int64_t& next, int64_t end) {
  Segment g;
  const int per_head = of_wave(s_sum[a.n_tile]);
  g.h = of_wave((int)(next / per_head));
  const int at = (int)(next - (int64_t)g.h * per_head);
  int lo = 0, hi = a.n_tile;     // the last tile that begins at or before it, and is not empty
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (of_wave(s_sum[mid]) <= at) lo = mid;
    else hi = mid;
  }
  g.tile = lo;
  const int sum = of_wave(s_sum[lo]), first = at - sum, all = of_wave(s_sum[lo + 1]) - sum;
  const int upto = (int)min((int64_t)all, first + (end - next));
  g.kt0 = max(first - kSetup, 0);
  g.kt1 = max(upto - kSetup, 0);   // none: another workgroup's
  g.whole = g.kt0 == 0 && upto == all;
  next += upto - first;
  return g;
}

// Workgroups that a CU holds (waves per SIMD).  Rows of 128 take more than half of the registers,
// Q alone 64, and fp32 MFMAs, 8 times as long as bf16's, need no second wave.
constexpr int tile_waves(int d) { return d == 64 ? 2 : 1; }

template <int D, bool SHARES>
__global__ __launch_bounds__(kBlock, tile_waves(D)) void page_tile_kernel(AttnArgs a) {
  using S = Tile<float, D>;
  constexpr int BN = S::BN, PPR = S::PPR, NP = S::NP, KS = S::KS, NB = S::NB;
  static_assert(BN == 32, "one MFMA result of keys");
  __shared__ u4 s_k[2][S::kPieces], s_v[2][S::kPieces];
  __shared__ BadKeys<D> s_bad;
  __shared__ int s_sum[SHARES ? kMaxTiles + 1 : 1];
  __shared__ int32_t s_cu[SHARES ? kMaxTiles + 1 : 1];
  __shared__ int s_wave[kWaves];

  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int l32 = lane % 32, half = lane / 32;
  // workgroups of one head side by side, on one XCD: they share its K and V
  const uint32_t id = xcd_logical_block(blockIdx.x, gridDim.x);
  const int32_t* cu = SHARES ? s_cu : a.cu;
  int64_t next = 0, end = 1;    // of this workgroup's triples
  if constexpr (SHARES) {
    if (!share_out<BN, kTileRows>(a, id, s_cu, s_sum, s_wave, next, end)) return;
  }

  for (int seg = 0; next < end; ++seg) {
    Segment sg;
    if constexpr (SHARES) {
      sg = next_segment(a, s_sum, next, end);
      if (sg.kt1 == 0) break;
      if (seg) __syncthreads();      // the tile before is done with s_bad
    } else {
      sg = Segment{a.n_tile - 1 - (int)(id % a.n_tile), (int)(id / a.n_tile), 0, 0x7fffffff, true};   // long ones first
      next = end;
    }
    const int tile = sg.tile, h = sg.h;
    const bool whole = sg.whole;
    const Span sp = Span(a, cu, find_slot(a.c.S, tile, [&](int s) { return first_tile<kTileRows>(a, cu, s); })).of_all();
    const int rows = sp.n * a.G, r0 = (tile - of_wave(first_tile<kTileRows>(a, cu, sp.s))) * kTileRows;
    if (r0 < 0 || r0 >= rows) return;   // none; r0 < 0: cu that falls
    sp.check(a);

    // the keys that this lane's row sees
    const int lim = sp.sees(a, min(r0 + 32 * wave + l32, rows - 1) / a.G);
    const int wave_lo = __builtin_amdgcn_readfirstlane(lim);              // the wave's first row's
    const int wave_hi = __builtin_amdgcn_readlane(lim, 31);               // and its last row's
    const bool has_rows = r0 + 32 * wave < rows;
    const int kb = sg.kt0 * BN;
    const int ke = (int)min((int64_t)sp.sees(a, (min(r0 + kTileRows, rows) - 1) / a.G), (int64_t)sg.kt1 * BN);
    const int least = sp.sees(a, r0 / a.G);   // keys that all rows see
    s_bad.clear(threadIdx.x);
    __syncthreads();

    u4 qf[KS];
    {
      const int row = min(r0 + 32 * wave + l32, rows - 1), tok = row / a.G;
      const u4* qp = a.q + (int64_t)(sp.c0 + tok) * a.q_u4 + (int64_t)(h * a.G + row - tok * a.G) * PPR + half;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qf[ks] = qp[2 * ks];
    }
    pf32x16 o[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[b][i] = 0.f;
    float m = -INFINITY, l = 0.f;   // in score units (before 1/sqrt(d)), over this lane's keys

    GroupBases<PPR> bases;
    u4 rk[NP], rv[NP];
    auto load = [&](int j0, uint64_t pool, u4 (&to)[NP]) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int x = i * kBlock + wave * kWave;    // the wave's first piece of this load
        to[i] = load_at(bases.at(j0 / 16 + x / (16 * PPR)) + pool, (x % (16 * PPR) + lane) * 16);
      }
    };
    auto stage = [&](int b, int j0) {
      if (j0 + BN > least) {
        const int tid = wave * kWave + lane_here();
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int x = i * kBlock + tid, key = j0 + x / PPR;
          rv[i] = key < sp.L ? rv[i] : u4{0, 0, 0, 0};
          scrub<float>(rv[i], key, x % PPR * (D / PPR), s_bad);
        }
      }
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int x = i * kBlock + threadIdx.x;
        s_k[b][S::k_at(x / PPR, x % PPR)] = rk[i];
        s_v[b][S::v_at(x / PPR, x % PPR)] = rv[i];
      }
    };

    if (kb < ke) {
      bases.fill(a, sp, h, kb / 16);
      load(kb, 0, rk);
      load(kb, to_v(a.c), rv);
      stage(0, kb);
    }
    int buf = 0;
    for (int j0 = kb; j0 < ke; j0 += BN, buf ^= 1) {
      __syncthreads();
      const bool more = j0 + BN < ke;
      if (more) {
        bases.reach(a, sp, h, (j0 + BN) / 16, (j0 + BN) / 16 + BN / 16 - 1);
        load(j0 + BN, 0, rk);
        load(j0 + BN, to_v(a.c), rv);
      }
      if (has_rows && j0 < wave_hi) {
        const u4* tk = s_k[buf];
        pf32x16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          if (ks % 4 == 0) __builtin_amdgcn_sched_barrier(0);   // not every operand at once in registers
          const u4 w = tk[S::k_at(l32, 2 * ks + half)];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(w[i]), __uint_as_float(qf[ks][i]), s, 0, 0, 0);
        }
        if (j0 + BN > wave_lo) {
          const int left = here(lim) - j0 - 4 * half;
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = 8 * (i / 4) + i % 4 < left ? s[i] : -INFINITY;
        }
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        if (__ballot(top > m)) {
          const float now = fmaxf(m, top);
          const float alpha = weight(m, now, a.scale_log2);
          m = now;
          l *= alpha;
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[b][i] *= alpha;
        }
        const float mc = reference(m, a.scale_log2);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[i] = exp2_(__builtin_fmaf(s[i], a.scale_log2, -mc));
          l += s[i];
        }
        const float* tv = reinterpret_cast<const float*>(s_v[buf]);
        auto vt = [&](int i, int b) {   // key of result element i, output 32 b + l32
          const int r = 8 * (i / 4) + 4 * half + i % 4;
          return tv[S::v_at(r, 8 * b + l32 / 4) * 4 + l32 % 4];
        };
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int b = 0; b < NB; ++b) o[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(vt(i, b), s[i], o[b], 0, 0, 0);
        }
      }
      if (more) stage(buf ^ 1, j0 + BN);
    }

    __syncthreads();   // s_bad
    if (has_rows) {
      l += __shfl_xor(l, 32, kWave);
      const int lane = lane_here(), half = lane / 32, r = 32 * wave + lane % 32;
      const int row = r0 + r, tok = row / a.G;
      const int64_t at = (int64_t)(sp.c0 + tok) * a.HG + h * a.G + row - tok * a.G;
      // a partial's place: a workgroup's first row tile, or its last
      const int64_t slot = ((int64_t)id * 2 + (seg > 0)) * kTileRows + r;
      const float mul = !whole ? 1.f : l > 0.f ? 1.f / l : l;   // no key: 0; NaN stays
      if (half == 0 && row < rows) store_ml(a, whole ? nullptr : a.part_ml + slot * 2, at, m * a.scale_log2, l);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4 && row < rows; ++i) {
          const int d0 = 32 * b + 8 * i + 4 * half;
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = o[b][4 * i + e] * mul + s_bad.sum(d0 + e, min(lim, ke));
          store4<float>(a, whole ? nullptr : a.part_o + slot * D + d0, at * D + d0, x);
        }
    }
  }
}

// ---------------------------------------------------------------------------
// The wide tile kernel (bf16).  A wave keeps 64 query rows (two to a lane), so that every K and
// V operand read from LDS feeds two MFMAs: with 32 rows LDS was as busy as the MFMAs.  MFMAs
// and the softmax's VALU work hardly overlap between waves of a SIMD on this part, but
// they do within one, so a wave has its SIMD to itself and its steps of 32 keys overlap:
// step t's exponentials run beside the scores of step t + 1 and the V product of step t - 1.
// Maxima that grow by less than 2^8 leave the reference alone (a probability is then at most
// 2^8, its rounding to bf16 relative as before).  4 slots of 2048 tokens over 4096 to 8448 rows, 5
// heads to each of 8 KV heads of 128: 960 to 1110 us by the card's clock, 1.07 to 0.93
// PFLOP/s, where a product of 8192^3 reaches 1.15; with 128 rows to a workgroup and two to a
// CU 1200 to 1390; rows of 64 645 us, 0.80 PFLOP/s (half of the MFMAs to an exponential).  The
// clock falls to 1.9 GHz under the power limit, and pool loads are waited for with LDS's.
// ---------------------------------------------------------------------------
constexpr int kWideRows = 64 * kWaves;

template <int D, bool SHARES>
__global__ __launch_bounds__(kBlock, 1) void page_wide_kernel(AttnArgs a) {
  using S = Tile<bf16_t, D>;
  constexpr int BN = S::BN, PPR = S::PPR, NP = S::NP, KS = S::KS, NB = S::NB;
  static_assert(BN == 64, "two steps of 32 keys");
  __shared__ u4 s_k[3][S::kPieces], s_v[3][S::kPieces];
  __shared__ BadKeys<D> s_bad;
  __shared__ int s_sum[SHARES ? kMaxTiles + 1 : 1];
  __shared__ int32_t s_cu[SHARES ? kMaxTiles + 1 : 1];
  __shared__ int s_wave[kWaves];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint32_t id = xcd_logical_block(blockIdx.x, gridDim.x);
  const int32_t* cu = SHARES ? s_cu : a.cu;
  int64_t next = 0, end = 1;
  if constexpr (SHARES) {
    if (!share_out<BN, kWideRows>(a, id, s_cu, s_sum, s_wave, next, end)) return;
  }

  for (int seg = 0; next < end; ++seg) {
    const int lane = lane_here(), l32 = lane % 32, half = lane / 32, tid = wave * kWave + lane;
    Segment sg;
    if constexpr (SHARES) {
      sg = next_segment(a, s_sum, next, end);
      if (sg.kt1 == 0) break;
      if (seg) __syncthreads();      // the tile before is done with LDS
    } else {
      sg = Segment{a.n_tile - 1 - (int)(id % a.n_tile), (int)(id / a.n_tile), 0, 0x7fffffff, true};
      next = end;
    }
    const int h = sg.h;
    const Span sp = Span(a, cu, find_slot(a.c.S, sg.tile, [&](int s) { return first_tile<kWideRows>(a, cu, s); })).of_all();
    const int rows = sp.n * a.G, r0 = (sg.tile - of_wave(first_tile<kWideRows>(a, cu, sp.s))) * kWideRows;
    if (r0 < 0 || r0 >= rows) return;   // none; r0 < 0: cu that falls
    sp.check(a);

    // the keys that this lane's two rows see; computed anew where they matter
    auto lim = [&](int c) INLINE {
      return sp.sees(a, min(r0 + 64 * wave + 32 * c + lane_here() % 32, rows - 1) / a.G);
    };
    const int wave_lo = sp.sees(a, min(r0 + 64 * wave, rows - 1) / a.G);   // the wave's first row's
    const int kb = sg.kt0 * BN;
    const int ke = (int)min((int64_t)sp.sees(a, (min(r0 + kWideRows, rows) - 1) / a.G), (int64_t)sg.kt1 * BN);
    const int least = sp.sees(a, r0 / a.G);   // keys that all rows see
    const int steps = max((ke - kb + BN - 1) / BN, 0) * 2;   // whole tiles: what lies behind is masked
    s_bad.clear(tid);
    __syncthreads();

    u4 qf[2][KS];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int row = min(r0 + 64 * wave + 32 * c + l32, rows - 1), tok = row / a.G;
      const u4* qp = a.q + (int64_t)(sp.c0 + tok) * a.q_u4 + (int64_t)(h * a.G + row - tok * a.G) * PPR + half;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qf[c][ks] = qp[2 * ks];
    }
    pf32x16 o[NB][2];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][c][i] = 0.f;
    // a row's reference m (in score units), mc (in log2 units), and the sum l over this lane's
    // keys; a score must pass m by more than slack for m to follow
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, alpha[2] = {1.f, 1.f};
    float mc[2] = {0.f, 0.f};
    const float slack = 8.f / a.scale_log2;
    bool grown = false;   // m has changed for the step in hand: O follows behind its V product

    GroupBases<PPR> bases;
    constexpr int kGroups = BN / 16;
    u4 rk[NP], rv[NP];
    uint64_t at_k[NP], at_v[NP];   // a tile's addresses: K's loads find them, V's follow a tile later
    const uint64_t kv = to_v(a.c);
    const uint32_t offset = (wave * kWave % (16 * PPR) + lane) * 16;
    auto reach = [&](int j0) INLINE { bases.reach(a, sp, h, j0 / 16, j0 / 16 + kGroups - 1); };
    auto load_k = [&](int j0, int i) INLINE {   // behind reach()
      at_v[i] = at_k[i] + kv;
      at_k[i] = bases.at(j0 / 16 + (i * kBlock + wave * kWave) / (16 * PPR));
      rk[i] = load_at(at_k[i], offset);
    };
    auto load_v = [&](int i) INLINE { rv[i] = load_at(at_v[i], offset); };
    auto put_k = [&](int b, int i) INLINE {
      const int x = i * kBlock + tid;
      s_k[b][S::k_at(x / PPR, x % PPR)] = rk[i];
    };
    auto put_v = [&](int b, int i) INLINE {
      const int x = i * kBlock + tid;
      s_v[b][S::v_at(x / PPR, x % PPR)] = rv[i];
    };
    auto clean_v = [&](int j0) INLINE {
      if (j0 + BN > least) {
        const int tid = wave * kWave + lane_here();
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int x = i * kBlock + tid, key = j0 + x / PPR;
          rv[i] = key < sp.L ? rv[i] : u4{0, 0, 0, 0};
          scrub<bf16_t>(rv[i], key, x % PPR * (D / PPR), s_bad);
        }
      }
    };
    // V^T operand of keys 32 x + 16 kk on, outputs 32 b on
    const int kr = 4 * half + lane % 16 / 4, pc = 2 * (lane / 16 % 2) + lane % 4 / 2, by = lane % 2 * 8;
    auto vt = [&](const u4* tv, int x, int kk, int b) INLINE {
      return read_vt(tv, S::v_at(32 * x + 16 * kk + kr, 4 * b + pc) * 16 + by,
                     S::v_at(32 * x + 16 * kk + 8 + kr, 4 * b + pc) * 16 + by);
    };
    // O stays in AGPRs, which leaves the other registers to what the VALU works on.  The compiler
    // does not see these as MFMAs: o_ready() keeps O's readers behind them.
    auto add_product = [&](const pbf16x8& v, const pbf16x8& p, pf32x16& x) INLINE {
      asm("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(x) : "v"(v), "v"(p));
    };
    auto o_ready = [&]() INLINE {   // 32 wait states (19 needed behind the last MFMA)
#pragma unroll
      for (int b = 0; b < NB; ++b) asm volatile("s_nop 15\n\ts_nop 15" : "+a"(o[b][0]), "+a"(o[b][1]));
    };
    float top[2] = {0.f, 0.f};
    u4 kf[KS];   // K operands of the next step
    auto k_operand = [&](const u4* tk, int x, int ks) INLINE { kf[ks] = tk[S::k_at(32 * x + l32, 2 * ks + half)]; };
    // a step's scores masked, and its reference: keys from j on
    auto settle = [&](pf32x16 (&s)[2], int j, bool first = false) INLINE {
      if (first || j + 32 > min(wave_lo, ke)) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int left = min(lim(c), ke) - j - 4 * half;
#pragma unroll
          for (int i = 0; i < 16; ++i) s[c][i] = 8 * (i / 4) + i % 4 < left ? s[c][i] : -INFINITY;
          top[c] = s[c][0];
#pragma unroll
          for (int i = 1; i < 16; ++i) top[c] = __builtin_elementwise_maximum(top[c], s[c][i]);
        }
      }
      grown = __ballot(top[0] > m[0] + slack || top[1] > m[1] + slack) != 0;
      if (grown) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          // a row whose own maximum has not passed stays as it is: no row's result hangs on another's
          const float both = fmaxf(top[c], __shfl_xor(top[c], 32, kWave));
          const float now = both > m[c] + slack ? both : m[c];
          alpha[c] = weight(m[c], now, a.scale_log2);
          m[c] = now;
          mc[c] = reference(now, a.scale_log2);
          l[c] *= alpha[c];
        }
      }
    };
    // One step: scores of the next 32 keys (kf) into `next`, the probabilities of the scores in
    // `cur` (pn), the V product of those before (pp), and the K operands of the step after it
    // (rows 32 kx on of tk).  Written out MFMA by MFMA, with what fits beside each: an MFMA takes
    // the pipe for 32 cycles, in which the wave can issue 7 other instructions.  A lane's element
    // goes through three of these places (argument, exponential, rounding), so that none of its
    // parts waits for the one before.  Probabilities are rounded to bf16 (to nearest, 2^-8 of each
    // at most); their sum is taken before, in fp32.
    auto step = [&](const u4* tk, int kx, const u4* tv, int vx, pf32x16 (&cur)[2], pf32x16 (&next)[2],
                    const u4 (&pp)[2][2], u4 (&pn)[2][2], int j, auto behind, auto beside) INLINE {
      constexpr int Q = 2 * KS, V = 4 * NB, E = 32;      // MFMAs of each kind, elements of a lane
      constexpr int per = E / (Q + V);                   // elements beside an MFMA
      pbf16x8 vf[2][NB];
      auto part0 = [&](auto e) INLINE {
        if constexpr (e < E) cur[e / 16][e % 16] = __builtin_fmaf(cur[e / 16][e % 16], a.scale_log2, -mc[e / 16]);
      };
      auto part1 = [&](auto e) INLINE {
        if constexpr (e < E) cur[e / 16][e % 16] = exp2_(cur[e / 16][e % 16]);
      };
      auto part2 = [&](auto e) INLINE {
        constexpr int c = e / 16, i = e % 16;
        l[c] += cur[c][i];
        asm volatile("" : "+v"(l[c]));   // here, not behind the step
        if constexpr (i % 2 == 1) {
          typedef float f2 __attribute__((ext_vector_type(2)));
          const pbf16x2 y = __builtin_convertvector(f2{cur[c][i - 1], cur[c][i]}, pbf16x2);
          pn[i / 8][c][i % 8 / 2] = __builtin_bit_cast(uint32_t, y);
        }
      };
      auto elements = [&](auto n) INLINE {
        each<per>([&](auto y) INLINE {
          part2(std::integral_constant<int, per * n + y>());
          part1(std::integral_constant<int, per * n + y + per>());
          part0(std::integral_constant<int, per * n + y + 2 * per>());
        });
      };
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) next[c][i] = 0.f;
      __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): the K operands, all in one wait
      __builtin_amdgcn_sched_barrier(0);
      each<Q>([&](auto n) INLINE {
        constexpr int ks = n / 2, c = n % 2, x = n - Q / 2;
        if constexpr (n == 2) {   // behind the first MFMAs: what would leave the pipe empty before them
          behind();
          settle(cur, j);
          each<2 * per>([&](auto e) INLINE { part0(e); });
          each<per>([&](auto e) INLINE { part1(e); });
        }
        next[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(pbf16x8, kf[ks]),
                                                          __builtin_bit_cast(pbf16x8, qf[c][ks]), next[c], 0, 0, 0);
        if constexpr (x >= 0 && x < 2 * NB) vf[x / NB][x % NB] = vt(tv, vx, x / NB, x % NB);
        if constexpr (n == 2 || n == 3) {
          beside(std::integral_constant<int, n - 2>());
          elements(std::integral_constant<int, 2 * n - 4>());
          elements(std::integral_constant<int, 2 * n - 3>());
        }
        if constexpr (x < 0 && n >= 2) beside(n);
        if constexpr (n >= 4) elements(n);
        __builtin_amdgcn_sched_barrier(0);
      });
      each<V>([&](auto n) INLINE {
        constexpr int kk = n / (2 * NB), b = n / 2 % NB, c = n % 2;
        add_product(vf[kk][b], __builtin_bit_cast(pbf16x8, pp[kk][c]), o[b][c]);
        if constexpr (n % 2 == 0 && n / 2 < KS) k_operand(tk, kx, n / 2);
        elements(std::integral_constant<int, Q + decltype(n)::value>());
        // the highest of the next scores, from behind their last MFMA on
        if constexpr (n >= 2) {
          constexpr int most = ((E + V - 3) / (V - 2) + 1) / 2 * 2;
          constexpr int e0 = (n - 2) * most, e1 = (n - 1) * most < E ? (n - 1) * most : E;
          each<(e1 > e0 ? e1 - e0 : 0)>([&](auto y) INLINE {
            constexpr int e = e0 + y;
            top[e / 16] = e % 16 ? __builtin_elementwise_maximum(top[e / 16], next[e / 16][e % 16]) : next[e / 16][0];
          });
          asm volatile("" : "+v"(top[0]), "+v"(top[1]));   // here, not behind the step
        }
        __builtin_amdgcn_sched_barrier(0);
      });
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) asm volatile("" : "+v"(pn[kk][c]));
    };
    auto follow = [&]() INLINE {
      if (grown) {
        o_ready();
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
#pragma unroll
            for (int i = 0; i < 16; ++i) o[b][c][i] *= alpha[c];
            asm volatile("s_nop 7" : "+a"(o[b][c]));
          }
      }
    };

    if (steps > 0) {
      bases.fill(a, sp, h, kb / 16);
#pragma unroll
      for (int i = 0; i < NP; ++i) at_k[i] = 0;
      auto load_tile = [&](int j0) INLINE {
        reach(j0);
#pragma unroll
        for (int i = 0; i < NP; ++i) load_k(j0, i);
      };
      u4 rk1[NP];
      load_tile(kb + BN);           // behind the last key: the last group again
#pragma unroll
      for (int i = 0; i < NP; ++i) rk1[i] = rk[i];
      load_tile(kb);
#pragma unroll
      for (int i = 0; i < NP; ++i) rv[i] = load_at(at_k[i] + kv, offset);
      // Q stays in AGPRs
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+a"(qf[c][ks]));
      clean_v(kb);
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        put_k(0, i);
        put_v(0, i);
        const int x = i * kBlock + tid;   // step 0's product, with probabilities of 0: rows of 0, as
        s_v[2][S::v_at(x / PPR, x % PPR)] = u4{0, 0, 0, 0};   // an infinity would leave NaN
        rk[i] = rk1[i];
        put_k(1, i);
        at_k[i] = bases.at((kb + BN) / 16 + (i * kBlock + wave * kWave) / (16 * PPR));
      }
      load_tile(kb + 2 * BN);
#pragma unroll
      for (int i = 0; i < NP; ++i) load_v(i);
      __syncthreads();
      pf32x16 s0[2], s1[2];
      u4 p0[2][2], p1[2][2];
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int c = 0; c < 2; ++c) p1[kk][c] = u4{0, 0, 0, 0};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) k_operand(s_k[0], 0, ks);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s0[c][i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
          s0[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(pbf16x8, kf[ks]),
                                                          __builtin_bit_cast(pbf16x8, qf[c][ks]), s0[c], 0, 0, 0);
      }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) k_operand(s_k[0], 1, ks);
      settle(s0, kb, true);
      // 64 keys.  Of K, tile b and the next are read and the one behind it written; of V, the
      // tile before, tile b, and the next: three buffers of each, one barrier.
      auto stage = [&](auto buffer, int j0) INLINE {
        constexpr int b = decltype(buffer)::value, b1 = (b + 1) % 3, b2 = (b + 2) % 3;
        step(s_k[b1], 0, s_v[b2], 1, s0, s1, p1, p0, j0,
             [&]() INLINE {
               __syncthreads();
               reach(j0 + 3 * BN);
             },
             // a tile's loads right behind the stores of the one before, nearly two steps ahead of
             // their use. They are flat loads, which the counter of LDS counts too, so that the waits
             // for LDS in between wait for them as well
             [&](auto n) INLINE {
               if constexpr (n < NP) put_k(b2, n);
               else if constexpr (n < 2 * NP) load_k(j0 + 3 * BN, n - NP);
             });
        follow();
        step(s_k[b1], 1, s_v[b], 0, s1, s0, p0, p1, j0 + 32, [&]() INLINE { clean_v(j0 + BN); },
             [&](auto n) INLINE {
               if constexpr (n < NP) put_v(b1, n);
               else if constexpr (n < 2 * NP) load_v(n - NP);
             });
        follow();
      };
      for (int t = 0; t < steps; t += 6) {
        stage(std::integral_constant<int, 0>(), kb + 32 * t);
        if (t + 2 >= steps) break;
        stage(std::integral_constant<int, 1>(), kb + 32 * t + 64);
        if (t + 4 >= steps) break;
        stage(std::integral_constant<int, 2>(), kb + 32 * t + 128);
      }
      const u4* tv = s_v[(steps / 2 - 1) % 3];   // the last step's product
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const pbf16x8 w = vt(tv, 1, kk, b);
#pragma unroll
          for (int c = 0; c < 2; ++c) add_product(w, __builtin_bit_cast(pbf16x8, p1[kk][c]), o[b][c]);
        }
      o_ready();
    }

    __syncthreads();   // s_bad; and K and V are read
    // Out by way of LDS, 32 rows at a time: a lane's 4 outputs of each block make stores of whole
    // lines there: 4 us, where straight from registers took 8.
    {
      const int lane = lane_here(), l32 = lane % 32, half = lane / 32;
      u4* room = (wave < 2 ? s_k[0] : s_v[0]) + wave % 2 * (32 * D / 4);   // of this wave
      if (s_bad.any(ke)) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int sees = min(lim(c), ke);
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[b][c][i] += s_bad.sum(32 * b + 8 * (i / 4) + 4 * half + i % 4, sees);
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        l[c] += __shfl_xor(l[c], 32, kWave);
        const int r = 64 * wave + 32 * c, left = rows - r0 - r;   // rows from r on
        const int row = r0 + r + l32, tok = row / a.G;
        const int at = (sp.c0 + tok) * a.HG + h * a.G + row - tok * a.G;   // T H G fits
        // a partial's place: a workgroup's first row tile, or its last
        const int64_t slot = ((int64_t)id * 2 + (seg > 0)) * kWideRows + r;
        const float mul = !sg.whole ? 1.f : l[c] > 0.f ? 1.f / l[c] : l[c];   // no key: 0; NaN stays
        if (half == 0 && l32 < left)
          store_ml(a, sg.whole ? nullptr : a.part_ml + (slot + l32) * 2, at, m[c] * a.scale_log2, l[c]);
        auto put = [&](auto f) INLINE {
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              pf32x4 x;
#pragma unroll
              for (int e = 0; e < 4; ++e) x[e] = o[b][c][4 * i + e] * mul;
              f(4 * b + i, x);
            }
          __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        };
        // rows of P pieces, permuted so that 16 rows' writes and a row's reads take all banks
        auto place = [&](int r, int p, int P) INLINE { return r * P + (p ^ (r & (P < 16 ? P - 1 : 15))); };
        if (sg.whole) {
          put([&](int q, pf32x4 x) INLINE {
            const pbf16x4 y = __builtin_convertvector(x, pbf16x4);
            reinterpret_cast<uint64_t*>(room + place(l32, q, PPR))[half] = __builtin_bit_cast(uint64_t, y);
          });
#pragma unroll
          for (int i = 0; i < 32 * PPR / kWave; ++i) {
            const int r = (i * kWave + lane) / PPR, q = lane % PPR;
            const int64_t to = __shfl(at, r, kWave);
            if (r < left) static_cast<u4*>(a.out)[to * PPR + q] = room[place(r, q, PPR)];
          }
        } else {
          constexpr int P = D / 4;
          put([&](int q, pf32x4 x) INLINE { room[place(l32, 2 * q + half, P)] = __builtin_bit_cast(u4, x); });
#pragma unroll
          for (int i = 0; i < 32 * P / kWave; ++i) {
            const int r = (i * kWave + lane) / P, q = lane % P;
            if (r < left) reinterpret_cast<u4*>(a.part_o)[(slot + r) * P + q] = room[place(r, q, P)];
          }
        }
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");   // read before the next rows
      }
    }
  }
}

// Behind shares: the rows of each (row tile, head) joined in the order of the keys, if several
// shares have some of them.  A thread takes 4 outputs of one row, so that a call of few rows
// still has many workgroups: it is a chain of memory latencies.
template <typename T, int D, int R>
__global__ __launch_bounds__(kBlock) void page_join_kernel(AttnArgs a) {
  constexpr int TPR = D / 4, RPB = kBlock / TPR, kPer = R / RPB;   // threads of a row, ...
  constexpr int U = 4;                                                    // partials in flight
  const int tile = (int)(blockIdx.x / kPer) % a.n_tile, h = (int)(blockIdx.x / kPer) / a.n_tile;
  const int per_head = a.sums[a.n_tile], sum0 = a.sums[tile], sum1 = a.sums[tile + 1];
  const Span sp(a, find_slot(a.c.S, tile, [&](int s) { return first_tile<R>(a, s); }));   // while those come
  if (sum1 <= sum0) return;
  const Shares sh(a, per_head);
  const int64_t x0 = (int64_t)h * per_head + sum0, x1 = (int64_t)h * per_head + sum1;
  const int first = sh.of(x0 + kSetup), last = sh.of(x1 - 1);
  if (first == last) return;   // whole: already written
  // the first part's partial is that of its last row tile if it began before this one; the others
  // begin in it
  const int64_t place0 = ((int64_t)first * 2 + (sh.begin(first) < x0)) * R;
  const int r0 = (tile - first_tile<R>(a, sp.s)) * R;
  const int d0 = threadIdx.x % TPR * 4, r = (int)(blockIdx.x % kPer) * RPB + threadIdx.x / TPR;
  if (r0 < 0 || r0 + r >= sp.n * a.G) return;
  auto place = [&](int i) { return (i == first ? place0 : (int64_t)i * 2 * R) + r; };
  float top = -INFINITY, l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
  for (int i = first; i <= last; i += U) {
    float2 y[U];
    float4 z[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = place(min(i + u, last));
      y[u] = *reinterpret_cast<const float2*>(a.part_ml + at * 2);
      z[u] = *reinterpret_cast<const float4*>(a.part_o + at * D + d0);
    }
    float now = top;
#pragma unroll
    for (int u = 0; u < U; ++u) now = fmaxf(now, y[u].x);
    const float old = weight(top, now);
    top = now;
    l *= old;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] *= old;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u > last) break;
      const float f = weight(y[u].x, top);
      l += y[u].y * f;
      x[0] += z[u].x * f;
      x[1] += z[u].y * f;
      x[2] += z[u].z * f;
      x[3] += z[u].w * f;
    }
  }
  const float mul = l > 0.f ? 1.f / l : l;
  const int tok = (r0 + r) / a.G;
  const int64_t at = (int64_t)(sp.c0 + tok) * a.HG + h * a.G + r0 + r - tok * a.G;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] *= mul;
  store4<T>(a, nullptr, at * D + d0, x);
  if (d0 == 0) store_ml(a, nullptr, at, top, l);
}

// ---------------------------------------------------------------------------
// The few-row kernel: a workgroup takes one (range, head, row tile of 16), its waves every
// fourth tile of 32 keys (fp32: 16).  K rows go from memory into A operands as they are, V rows
// through a piece of LDS that the wave has alone; the waves' states are joined at the
// end.  The next tile's rows are loaded as soon as this one's have left their registers.
// 64 slots of 2000 to 8320 rows, one token, 8 heads to each of 8 KV heads of 128: 234 us, 5.8
// TB/s (a large copy reaches 5 to 6).
// ---------------------------------------------------------------------------
template <typename T, int D>
struct Few {
  static constexpr bool kBf16 = std::is_same<T, bf16_t>::value;
  static constexpr int NS = kBf16 ? 2 : 1;            // MFMA results of 16 keys
  static constexpr int BN = 16 * NS;
  static constexpr int PPR = D * (kBf16 ? 2 : 4) / 16;
  static constexpr int NP = BN * PPR / kWave;         // V pieces per lane
  static constexpr int KS = PPR / 4;                  // groups of 4 pieces, one to a quarter wave
  static constexpr int NB = D / 16;
  // see Tile: here one transposed read of half a wave takes 2 pieces of 8 rows, and one
  // fp32 read 16 floats of rows r, r + 4, r + 8, r + 12
  __device__ static __forceinline__ int v_at(int r, int p) {
    if constexpr (!kBf16) return r * PPR + (p ^ (4 * ((r >> 2) & 3)));
    else if constexpr (PPR == 8) return r / 2 * 16 + (((r % 2) * 8 + p) ^ (2 * ((r >> 1) & 3)));
    else return r * PPR + (p ^ (2 * (r & 7)));
  }
};

template <typename T, int D, bool ONCE>
__global__ __launch_bounds__(kBlock) void page_few_kernel(AttnArgs a) {
  using S = Few<T, D>;
  constexpr int BN = S::BN, NS = S::NS, PPR = S::PPR, NP = S::NP, KS = S::KS, NB = S::NB;
  static_assert(BN * PPR * 16 == kFewRows * D * 4, "a wave's V rows and its O take the same room");
  __shared__ u4 s_v[kWaves][BN * PPR];
  __shared__ float s_ml[kWaves][kFewRows][2];
  __shared__ BadKeys<D> s_bad;

  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int l16 = lane % 16, quad = lane / 16;
  const uint32_t id = xcd_logical_block(blockIdx.x, gridDim.x);
  const int split = (int)(id % a.n_split), h = (int)(id / a.n_split) % a.c.H;
  const int tile = (int)(id / a.n_split) / a.c.H;
  const Span sp(a, a.by_slot ? tile : find_slot(a.c.S, tile, [&](int s) { return first_tile<kFewRows>(a, s); }));
  const int r0 = a.by_slot ? 0 : (tile - first_tile<kFewRows>(a, sp.s)) * kFewRows;
  if (a.by_slot && sp.n * a.G > kFewRows) {   // more tokens than max_new said
    if (threadIdx.x == 0 && a.status) atomicOr(a.status, VASE_STATUS_PAGE_BAD);
    return;
  }
  const int rows = min(sp.n * a.G - r0, kFewRows);   // of this tile
  if (r0 < 0 || rows <= 0) return;   // none; r0 < 0: cu that falls
  sp.check(a);
  const int row = r0 + min(l16, rows - 1);
  const int tok = row / a.G, g = row - tok * a.G;
  const int lim = sp.sees(a, tok);
  const int least = sp.sees(a, r0 / a.G);   // keys that all rows see
  const int kb = split * a.keys;
  int ke = sp.sees(a, (r0 + rows - 1) / a.G);
  if (split < a.n_split - 1) ke = min(ke, kb + a.keys);
  if (kb >= ke && a.n_split > 1) return;   // combine takes no partial of this range
  s_bad.clear(threadIdx.x);
  __syncthreads();

  u4 qf[KS];
  {
    const u4* qp = a.q + (int64_t)(sp.c0 + tok) * a.q_u4 + (int64_t)(h * a.G + g) * PPR + quad;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = qp[4 * ks];
  }
  pf32x4 o[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) o[b] = pf32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  GroupBases<PPR> bases;
  u4 rk[NS][KS], rv[NP];
  auto load = [&](int j0) {
    bases.reach(a, sp, h, j0 / 16, j0 / 16 + NS - 1);
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const uint64_t at = bases.at(j0 / 16 + n);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) rk[n][ks] = load_at(at, (l16 * PPR + 4 * ks + quad) * 16);
#pragma unroll
      for (int i = 0; i < NP / NS; ++i) {
        const uint64_t av = at + to_v(a.c);
        const uint32_t offset = (i * kWave + lane) * 16;
        rv[n * (NP / NS) + i] = ONCE ? load_once_at(av, offset) : load_at(av, offset);
      }
    }
  };
  u4* tv = s_v[wave];
  const int j_first = kb + wave * BN;
  if (j_first < ke) {
    bases.fill(a, sp, h, j_first / 16);
    load(j_first);
  }
  for (int j0 = j_first; j0 < ke; j0 += kWaves * BN) {
    if (j0 + BN > least) {
      const int at = lane_here();
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int x = i * kWave + at, key = j0 + x / PPR;
        rv[i] = key < sp.L ? rv[i] : u4{0, 0, 0, 0};
        scrub<T>(rv[i], key, x % PPR * (D / PPR), s_bad);
      }
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) tv[S::v_at((i * kWave + lane) / PPR, (i * kWave + lane) % PPR)] = rv[i];
    pf32x4 s[NS];
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      s[n] = pf32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const u4 w = rk[n][ks];
        if constexpr (S::kBf16) {
          s[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pbf16x8, w),
                                                         __builtin_bit_cast(pbf16x8, qf[ks]), s[n], 0, 0, 0);
        } else {
          s[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w.x), __uint_as_float(qf[ks].x), s[n], 0, 0, 0);
          s[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w.y), __uint_as_float(qf[ks].y), s[n], 0, 0, 0);
          s[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w.z), __uint_as_float(qf[ks].z), s[n], 0, 0, 0);
          s[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w.w), __uint_as_float(qf[ks].w), s[n], 0, 0, 0);
        }
      }
    }
    if (j0 + kWaves * BN < ke) load(j0 + kWaves * BN);
    const bool masked = j0 + BN > least;
    if (masked) {
#pragma unroll
      for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][i] = j0 + 16 * n + 4 * quad + i < lim ? s[n][i] : -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int n = 0; n < NS; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, s[n][i]);
    top = fmaxf(top, __shfl_xor(top, 16, kWave));
    top = fmaxf(top, __shfl_xor(top, 32, kWave));
    if (__ballot(top > m)) {
      const float now = fmaxf(m, top);
      const float alpha = weight(m, now, a.scale_log2);
      m = now;
      l *= alpha;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[b][i] *= alpha;
    }
    const float mc = reference(m, a.scale_log2);
#pragma unroll
    for (int n = 0; n < NS; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[n][i] = exp2_(__builtin_fmaf(s[n][i], a.scale_log2, -mc));
        l += s[n][i];
      }
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");   // the V rows are in LDS
    if constexpr (S::kBf16) {
      const int kr = 4 * quad + l16 / 4, pc = l16 % 4 / 2, by = l16 % 2 * 8;
      auto vt = [&](int b) {
        return read_vt(tv, S::v_at(kr, 2 * b + pc) * 16 + by, S::v_at(16 + kr, 2 * b + pc) * 16 + by);
      };
      pf32x8 x;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = s[i / 4][i % 4];
      const pbf16x8 pb = __builtin_convertvector(x, pbf16x8);   // rounded as in the wide kernel
#pragma unroll
      for (int b = 0; b < NB; ++b) o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt(b), pb, o[b], 0, 0, 0);
    } else {
      const float* tf = reinterpret_cast<const float*>(tv);
      auto vt = [&](int i, int b) { return tf[S::v_at(4 * quad + i, 4 * b + l16 / 4) * 4 + l16 % 4]; };
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int b = 0; b < NB; ++b)
          o[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(vt(i, b), s[0][i], o[b], 0, 0, 0);
    }
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");   // read before the next rows
  }

  // join the waves: O rows into the wave's own room, [row][D]
  l += __shfl_xor(l, 16, kWave);
  l += __shfl_xor(l, 32, kWave);
  float* so = reinterpret_cast<float*>(tv);
#pragma unroll
  for (int b = 0; b < NB; ++b)
    *reinterpret_cast<float4*>(so + l16 * D + 16 * b + 4 * quad) = make_float4(o[b][0], o[b][1], o[b][2], o[b][3]);
  if (quad == 0) {
    s_ml[wave][l16][0] = m;
    s_ml[wave][l16][1] = l;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < rows * (D / 4); e += kBlock) {
    const int r = e / (D / 4), d0 = e % (D / 4) * 4;
    float mm = s_ml[0][r][0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) mm = fmaxf(mm, s_ml[w][r][0]);
    float ll = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float mw = s_ml[w][r][0];
      const float f = weight(mw, mm, a.scale_log2);
      ll += s_ml[w][r][1] * f;
      const float4 y = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(s_v[w]) + r * D + d0);
      x[0] += y.x * f;
      x[1] += y.y * f;
      x[2] += y.z * f;
      x[3] += y.w * f;
    }
    const int ti = (r0 + r) / a.G;
    const int64_t at = (int64_t)(sp.c0 + ti) * a.HG + h * a.G + r0 + r - ti * a.G;
    const int64_t part = (int64_t)split * a.T * a.HG + at;
    const bool whole = a.n_split == 1;
    const float mul = !whole ? 1.f : ll > 0.f ? 1.f / ll : ll;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = x[i] * mul + s_bad.sum(d0 + i, min(sp.sees(a, ti), ke));
    store4<T>(a, whole ? nullptr : a.part_o + part * D + d0, at * D + d0, x);
    if (d0 == 0) store_ml(a, whole ? nullptr : a.part_ml + part * 2, at, mm * a.scale_log2, ll);
  }
}

// ---------------------------------------------------------------------------
// Behind the few-row kernel's ranges: a wave per (token, query head), those that hold a key the
// token sees joined in order.
// ---------------------------------------------------------------------------
template <typename T, int D>
__global__ __launch_bounds__(kBlock) void page_combine_kernel(AttnArgs a) {
  constexpr int E = D / kWave;
  const int lane = threadIdx.x % kWave;
  const int64_t at = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int t = (int)(at / a.HG);
  if (t >= a.T || t >= a.cu[a.c.S]) return;
  const Span sp(a, find_slot(a.c.S, t, [&](int i) { return a.cu[i]; }));
  if (t < sp.c0 || t >= sp.c0 + sp.n) return;
  if (a.by_slot && sp.n * a.G > kFewRows) return;   // left out
  const int sees = sp.sees(a, t - sp.c0);
  const int n = min(a.n_split, (sees + a.keys - 1) / a.keys);
  const int64_t row = (int64_t)a.T * a.HG;     // rows of a range's partials
  float m = -INFINITY, l = 0.f;
  if (lane < n) {
    const float2 x = *reinterpret_cast<const float2*>(a.part_ml + (lane * row + at) * 2);
    m = x.x;
    l = x.y;
  }
  float top = m;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
  const float f = weight(m, top);
  float sum = l * f;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) sum += __shfl_xor(sum, o, kWave);
  float x[E] = {};
  for (int s = 0; s < n; ++s) {
    const float fs = __shfl(f, s, kWave);
    const float* p = a.part_o + (s * row + at) * D + E * lane;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] += p[e] * fs;
  }
  const float mul = sum > 0.f ? 1.f / sum : sum;
#pragma unroll
  for (int e = 0; e < E; ++e) store_out<T>(static_cast<T*>(a.out) + at * D + E * lane + e, x[e] * mul);
  if (a.lse && lane == 0) a.lse[at] = lse_of(top, sum);
}

template <typename T, int D>
hipError_t launch_td(const AttnArgs& a, const PageAttnPlan& pl, hipStream_t stream) {
  constexpr bool kWide = std::is_same<T, bf16_t>::value;
  constexpr int R = kWide ? kWideRows : kTileRows;
  const dim3 block(kBlock);
  if (pl.few) {
    const dim3 grid((unsigned)(a.n_tile * a.c.H * a.n_split));
    if (pl.once) hipLaunchKernelGGL((page_few_kernel<T, D, true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((page_few_kernel<T, D, false>), grid, block, 0, stream, a);
    // a wave per row
    if (a.n_split > 1)
      hipLaunchKernelGGL((page_combine_kernel<T, D>), dim3((unsigned)(((int64_t)a.T * a.HG + kWaves - 1) / kWaves)),
                         block, 0, stream, a);
    return hipGetLastError();
  }
  const dim3 grid(a.shares ? a.shares : (unsigned)(a.n_tile * a.c.H));
  if constexpr (kWide) {
    if (a.shares) hipLaunchKernelGGL((page_wide_kernel<D, true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((page_wide_kernel<D, false>), grid, block, 0, stream, a);
  } else {
    if (a.shares) hipLaunchKernelGGL((page_tile_kernel<D, true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((page_tile_kernel<D, false>), grid, block, 0, stream, a);
  }
  if (a.shares)
    hipLaunchKernelGGL((page_join_kernel<T, D, R>), dim3((unsigned)(a.n_tile * a.c.H * (R * D / 4 / kBlock))), block, 0,
                       stream, a);
  return hipGetLastError();
}

}  // namespace

PageAttnPlan page_attn_plan(const vase_pages& c, int T, int G, int max_new, int max_len) {
  PageAttnPlan p{};
  const bool wide = c.dtype == VASE_BF16;
  const int slots = std::min(c.S, T);          // that can have tokens
  const int64_t most = (int64_t)max_new * G;   // rows of a slot
  const double reads = (double)((int64_t)T * G / kFewRows + slots) * c.H * max_len * c.d;   // of K by 16-row tiles
  // 16-row tiles read K and V once each, larger ones begin late (13 us, with shares 25) and work
  // on rows that are not there.  8 slots over 4200 rows, 8 KV heads of 128, us of 16-row tiles and of
  // larger: 32 rows to a slot 53 and 59, 64 rows 88 and 60; fp32 32 rows 104 and 217, 64 rows 178
  // and 221, 128 rows (more) and 236.  Small calls: 1 slot over 4224 rows, 64 query rows (22 M
  // elements read) 26 and 34, 128 (39 M) 36 and 36; 256 over 1000 rows (17 M) 19 and 36.
  p.by_slot = most <= kFewRows && c.S <= T;
  p.few = most <= (wide ? 32 : 64) || reads <= 1 << 25;
  p.n_split = 1;
  p.keys = max_len;
  if (p.few) {
    const size_t rows = (size_t)T * c.H * G;
    p.n_tile = p.by_slot ? c.S : (int)((int64_t)T * G / kFewRows) + slots;
    // V rows past the caches where each is read once, from 2^17 of them on (bf16, d 128: 32 MB): us
    // with plain loads and so, 64 slots of 2000 to 8320 rows 251 and 234, 256 of 500 to 4224 441 and
    // 419; one of 4224, which stays in the caches, 8.3 and 9.3.  The other rows, slots of 4000 to 4200
    // over 8 heads: fp32, d 128, 1 slot 21 and 19, 4 (2^17 rows) 36 and 37, 16 108 and 90, 64 382 and
    // 346; bf16, d 64, 1 slot 10.5 and 10.9, 4 14.6 and 14.8, 16 30 and 30, 64 110 and 87; fp32, d 64, 1
    // slot 13 and 14, 4 22 and 21, 16 52 and 52, 64 199 and 181.
    // Not K rows: an operand load takes 64 bytes of each, half of a line (256 slots 492).
    p.once = p.by_slot && (int64_t)slots * c.H * max_len >= 1 << 17;
    // 8 workgroups to a CU, at least 256 keys to a range (512 and 1024 took as long), up to
    // kMaxSplit ranges
    const int64_t wgs = (p.by_slot ? slots : (int64_t)T * G / kFewRows + 1) * c.H;
    int64_t s = 2048 / wgs + 1;
    if (s > kMaxSplit) s = kMaxSplit;
    if (s > max_len / 256) s = max_len / 256;
    if (s < 1) s = 1;
    p.keys = (int)(((max_len + s - 1) / s + 127) / 128 * 128);
    p.n_split = (max_len + p.keys - 1) / p.keys;
    if (p.n_split > 1) {
      p.off_ml = p.n_split * rows * c.d * sizeof(float);
      p.bytes = p.off_ml + p.n_split * rows * 2 * sizeof(float);
    }
    return p;
  }
  const int R = wide ? kWideRows : kTileRows;
  p.n_tile = (int)((int64_t)T * G / R) + slots;
  const int shares = 256 * (wide ? 1 : tile_waves(c.d));   // workgroups that run at once
  const int64_t tiles = ((int64_t)T * G / R + 1) * c.H, most_tiles = max_new <= max_len / 2 ? shares * 3 / 2 : shares;
  // Where a second round of workgroups would run half empty or there is no full first one: us
  // shared (with the launch behind) and not, row tiles of about as many keys (8 slots, histories of
  // 3000 to 8000 rows): 328 row tiles 168 and 183, 264 and 320; 392 191 and 188, 311 and 329; 456 220
  // and 198, 358 and 375.  A fresh prompt's run from long to short and fill the gaps: 208
  // row tiles 62 and 54, 300 94 and 78, but 144 50 and 63.
  // The sums of 32-key tiles stay in 32 bits.
  if (tiles <= most_tiles && p.n_tile <= kMaxTiles && c.S <= kMaxTiles && max_len > 1024 &&
      (int64_t)p.n_tile * (c.M * c.page / 32 + 1 + kSetup) <= 0x7fffffff) {
    p.shares = shares;
    const size_t part = (size_t)p.shares * 2 * R;
    p.off_ml = part * c.d * sizeof(float);
    p.off_sums = p.off_ml + part * 2 * sizeof(float);
    p.bytes = p.off_sums + (kMaxTiles + 1) * sizeof(int32_t);
  }
  return p;
}

hipError_t launch_page_attn(const vase_pages& c, const void* q, int64_t q_stride, const int32_t* cu,
                            int T, int G, int causal, void* out, float* lse, void* ws,
                            const PageAttnPlan& plan, uint32_t* status, hipStream_t stream) {
  AttnArgs a{};
  a.c = page_view(c);
  a.q = static_cast<const u4*>(q);
  a.q_u4 = q_stride / (c.dtype == VASE_BF16 ? 8 : 4);
  a.cu = cu;
  a.T = T;
  a.G = G;
  a.HG = c.H * G;
  a.causal = causal != 0;
  a.out = out;
  a.lse = lse;
  a.part_o = static_cast<float*>(ws);
  a.part_ml = reinterpret_cast<float*>(static_cast<char*>(ws) + plan.off_ml);
  a.sums = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + plan.off_sums);
  a.n_tile = plan.n_tile;
  a.n_split = plan.n_split;
  a.keys = plan.keys;
  a.by_slot = plan.by_slot;
  a.shares = plan.shares;
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)c.d);
  a.status = status;
  if (c.dtype == VASE_BF16)
    return c.d == 128 ? launch_td<bf16_t, 128>(a, plan, stream) : launch_td<bf16_t, 64>(a, plan, stream);
  return c.d == 128 ? launch_td<float, 128>(a, plan, stream) : launch_td<float, 64>(a, plan, stream);
}

}  // namespace vase
