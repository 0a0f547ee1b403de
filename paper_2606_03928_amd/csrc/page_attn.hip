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
// Two kernels: page_tile_kernel takes 128 query rows to a workgroup and is bound by its
// MFMAs and exponentials; page_few_kernel takes up to 16 (a token of decoding) and is
// bound by the K and V rows it reads.  Both may split the keys into ranges, whose
// partial (m, l, O) page_combine_kernel joins in range order.
//
// Masked keys take p = 0 by a select on the score, and V rows behind the slot's end are
// zeroed where they are staged.  A later token's V row may hold an infinity or a NaN, which
// p = 0 would not keep out of a product: in tiles whose keys not every row sees, V rows are
// looked through as they are staged, such values go in as 0, and each output column
// keeps the first key that had one; rows that see that key end with NaN there.
#include "page_internal.hpp"

#include <type_traits>

namespace vase {
namespace {

typedef __bf16 pbf16x8 __attribute__((ext_vector_type(8)));
typedef short ps16x4 __attribute__((ext_vector_type(4)));
typedef unsigned short pu16x2 __attribute__((ext_vector_type(2)));
typedef float pf32x8 __attribute__((ext_vector_type(8)));
typedef float pf32x16 __attribute__((ext_vector_type(16)));
typedef float pf32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));   // 16 bytes of a row
typedef __attribute__((address_space(3))) ps16x4 lds_s16x4;

constexpr int kBlock = 256;
constexpr int kWaves = kBlock / kWave;
constexpr int kTileRows = 32 * kWaves;   // query rows of a tile workgroup
constexpr int kFewRows = 16;             // most query rows of a few-row workgroup
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
  float *part_o, *part_ml; // [split][T][HG][D], [split][T][HG][2]
  int n_tile, n_split, keys;
  int few_split, few_keys; // combine: those of the few-row kernel
  int split_rows;          // slots of up to so many rows are the other kernel's (tile: 0 none)
  float scale_log2;
  uint32_t* status;
};

// A slot's share of the batch, read as it stands but kept inside the caller's arrays.
struct Span {
  int s, c0, n, L;   // slot, first token, tokens, rows
  __device__ __forceinline__ Span(const AttnArgs& a, int slot) : s(slot) {
    c0 = min(max(a.cu[s], 0), a.T);
    n = min(max(a.cu[s + 1], c0), a.T) - c0;
    L = slot_len(a.c, s);
  }
  // rows that token i sees
  __device__ __forceinline__ int sees(const AttnArgs& a, int i) const {
    return a.causal ? max(L - n + i + 1, 0) : L;
  }
};

// Where the 16-row groups of a slot lie: lane l holds the offset (in pieces, from the pool's
// first) of group g0 + l of head h, 64 groups at a time.
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
    const uint64_t at = (uint64_t)(p * a.c.page_u4 + h * a.c.head_u4 + (int64_t)(gl * 16 - q * a.c.page) * PPR);
    lo = (uint32_t)at;
    hi = (uint32_t)(at >> 32);
    g0 = g;
  }
  // for at() of groups [first, last]; at most 64 of them
  __device__ __forceinline__ void reach(const AttnArgs& a, const Span& sp, int h, int first, int last) {
    if (last >= g0 + kWave) fill(a, sp, h, first);
  }
  __device__ __forceinline__ int64_t at(int g) const {
    const uint32_t x = __builtin_amdgcn_readlane(lo, g - g0), y = __builtin_amdgcn_readlane(hi, g - g0);
    return (int64_t)((uint64_t)y << 32 | x);
  }
};

// x, for code that only some iterations run: what is computed from it is computed there, and
// takes no register in the others
__device__ __forceinline__ int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// One output row (d values from d0 on, 4 of them): the result, or a range's partial.
template <typename T, int D>
__device__ __forceinline__ void store4(const AttnArgs& a, int split, int t, int hq, int d0, const float (&o)[4]) {
  if (a.n_split > 1) {
    *reinterpret_cast<float4*>(a.part_o + (((int64_t)split * a.T + t) * a.HG + hq) * D + d0) =
        make_float4(o[0], o[1], o[2], o[3]);
  } else if constexpr (std::is_same<T, float>::value) {
    *reinterpret_cast<float4*>(static_cast<float*>(a.out) + ((int64_t)t * a.HG + hq) * D + d0) =
        make_float4(o[0], o[1], o[2], o[3]);
  } else {
    ushort4 w;
    w.x = f32_to_bf16_bits(o[0]);
    w.y = f32_to_bf16_bits(o[1]);
    w.z = f32_to_bf16_bits(o[2]);
    w.w = f32_to_bf16_bits(o[3]);
    *reinterpret_cast<ushort4*>(static_cast<uint16_t*>(a.out) + ((int64_t)t * a.HG + hq) * D + d0) = w;
  }
}
// its maximum (in scaled log2 units) and sum
__device__ __forceinline__ void store_ml(const AttnArgs& a, int split, int t, int hq, float m, float l) {
  if (a.n_split > 1) {
    *reinterpret_cast<float2*>(a.part_ml + (((int64_t)split * a.T + t) * a.HG + hq) * 2) = make_float2(m, l);
  } else if (a.lse) {
    a.lse[(int64_t)t * a.HG + hq] = l > 0.f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
  }
}

// ---------------------------------------------------------------------------
// Values of V that no product with 0 keeps out: taken out of a piece of key `key`'s row
// (columns col on), the first key of each column noted in first_bad[D].
// ---------------------------------------------------------------------------
__device__ __forceinline__ bool is_bad(uint32_t fp32) { return (fp32 & 0x7fffffffu) >= 0x7f800000u; }
template <typename T>
__device__ __forceinline__ void scrub(u4& w, int key, int col, int* first_bad) {
  if constexpr (std::is_same<T, float>::value) {
    if (is_bad(w.x) || is_bad(w.y) || is_bad(w.z) || is_bad(w.w)) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (is_bad(w[i])) {
          atomicMin(&first_bad[col + i], key);
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
          atomicMin(&first_bad[col + 2 * i], key);
          w[i] &= 0xffff0000u;
        }
        if (is_bad(w[i])) {
          atomicMin(&first_bad[col + 2 * i + 1], key);
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
__device__ __forceinline__ pbf16x8 to_bf16x8(const pf32x8& x) { return __builtin_convertvector(x, pbf16x8); }

// ---------------------------------------------------------------------------
// The tile kernel.  A wave keeps 32 query rows (one per lane column) and their O^T in
// registers; K and V tiles of BN keys pass through two LDS buffers, the next tile's
// rows on their way to registers while this one is used.
// ---------------------------------------------------------------------------
template <typename T, int D>
struct Tile {
  static constexpr bool kBf16 = std::is_same<T, bf16_t>::value;
  static constexpr int BN = kBf16 ? 64 : 32;          // keys
  static constexpr int NS = BN / 32;                  // MFMA results of 32 keys
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

template <typename T, int D>
__global__ __launch_bounds__(kBlock, 2) void page_tile_kernel(AttnArgs a) {
  using S = Tile<T, D>;
  constexpr int BN = S::BN, NS = S::NS, PPR = S::PPR, NP = S::NP, KS = S::KS, NB = S::NB;
  __shared__ u4 s_k[2][S::kPieces], s_v[2][S::kPieces];
  __shared__ int s_bad[D];

  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int l32 = lane % 32, half = lane / 32;
  // workgroups of one head and range side by side, on one XCD: they share its K and V
  const uint32_t id = xcd_logical_block(blockIdx.x, gridDim.x);
  const int tile = a.n_tile - 1 - (int)(id % a.n_tile);
  const int h = (int)(id / a.n_tile) % a.c.H, split = (int)(id / a.n_tile) / a.c.H;

  // tiles of slot s begin at number floor(cu[s] G / 128) + s: room for all of its rows
  auto first_tile = [&](int s) { return (int)((int64_t)min(max(a.cu[s], 0), a.T) * a.G / kTileRows) + s; };
  const Span sp(a, find_slot(a.c.S, tile, first_tile));
  const int rows = sp.n * a.G, r0 = (tile - first_tile(sp.s)) * kTileRows;
  if (r0 >= rows || rows <= a.split_rows) return;

  // this lane's row, and the keys that it sees
  const int row = min(r0 + 32 * wave + l32, rows - 1);
  const int tok = row / a.G, g = row - tok * a.G;
  const int lim = sp.sees(a, tok);
  const int wave_lo = __builtin_amdgcn_readfirstlane(lim);              // the wave's first row's
  const int wave_hi = __builtin_amdgcn_readlane(lim, 31);               // and its last row's
  const bool has_rows = r0 + 32 * wave < rows;
  const int kb = split * a.keys;
  int ke = sp.sees(a, (min(r0 + kTileRows, rows) - 1) / a.G);
  if (split < a.n_split - 1) ke = min(ke, kb + a.keys);
  if (kb >= ke && a.n_split > 1) return;   // combine takes no partial of this range
  const int least = sp.sees(a, r0 / a.G);   // keys that all rows see
  if (threadIdx.x < D) s_bad[threadIdx.x] = 0x7fffffff;
  __syncthreads();

  u4 qf[KS];
  {
    const u4* qp = a.q + (int64_t)(sp.c0 + tok) * a.q_u4 + (int64_t)(h * a.G + g) * PPR + half;
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
  auto load = [&](int j0, const uint4* pool, u4 (&to)[NP]) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int r = (i * kBlock + wave * kWave) / PPR;    // the wave's first row of this load
      to[i] = reinterpret_cast<const u4*>(pool)[bases.at((j0 + r) / 16) +
                                                ((i * kBlock + wave * kWave) % (16 * PPR) + lane)];
    }
  };
  auto stage = [&](int b, int j0) {
    if (j0 + BN > least) {
      const int tid = here(threadIdx.x);
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int x = i * kBlock + tid, key = j0 + x / PPR;
        rv[i] = key < sp.L ? rv[i] : u4{0, 0, 0, 0};
        scrub<T>(rv[i], key, x % PPR * (D / PPR), s_bad);
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
    load(kb, a.c.k, rk);
    load(kb, a.c.v, rv);
    stage(0, kb);
  }
  int buf = 0;
  for (int j0 = kb; j0 < ke; j0 += BN, buf ^= 1) {
    __syncthreads();
    const bool more = j0 + BN < ke;
    // fp32: V rows only behind the scores, whose operands take twice the registers
    if (more) {
      bases.reach(a, sp, h, (j0 + BN) / 16, (j0 + BN) / 16 + BN / 16 - 1);
      load(j0 + BN, a.c.k, rk);
      if (S::kBf16) load(j0 + BN, a.c.v, rv);
    }
    if (has_rows && j0 < wave_hi) {
      const u4* tk = s_k[buf];
      const u4* tv = s_v[buf];
      pf32x16 s[NS];
#pragma unroll
      for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n][i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if (ks % 4 == 0) __builtin_amdgcn_sched_barrier(0);   // not every operand at once in registers
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          const u4 w = tk[S::k_at(32 * n + l32, 2 * ks + half)];
          if constexpr (S::kBf16) {
            s[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(pbf16x8, w),
                                                           __builtin_bit_cast(pbf16x8, qf[ks]), s[n], 0, 0, 0);
          } else {
            s[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(w.x), __uint_as_float(qf[ks].x), s[n], 0, 0, 0);
            s[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(w.y), __uint_as_float(qf[ks].y), s[n], 0, 0, 0);
            s[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(w.z), __uint_as_float(qf[ks].z), s[n], 0, 0, 0);
            s[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(w.w), __uint_as_float(qf[ks].w), s[n], 0, 0, 0);
          }
        }
      }
      const bool masked = j0 + BN > wave_lo;
      if (masked) {
        const int left = here(lim) - j0 - 4 * half;
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[n][i] = 32 * n + 8 * (i / 4) + i % 4 < left ? s[n][i] : -INFINITY;
      }
      float top = s[0][0];
#pragma unroll
      for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[n][i]);
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      if (__ballot(top > m)) {
        const float now = fmaxf(m, top);
        const float alpha = m == -INFINITY ? 0.f : exp2_((m - now) * a.scale_log2);
        m = now;
        l *= alpha;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[b][i] *= alpha;
      }
      const float mc = m == -INFINITY ? 0.f : m * a.scale_log2;
#pragma unroll
      for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[n][i] = exp2_(__builtin_fmaf(s[n][i], a.scale_log2, -mc));
          l += s[n][i];
        }
      if constexpr (S::kBf16) {
        // the lane's part of the transposed reads: key 4 half + (lane % 16) / 4 of 8, 8 bytes
        // from output 16 (lane / 16 % 2) + 4 (lane % 4) on
        const int kr = 4 * half + lane % 16 / 4, pc = 2 * (lane / 16 % 2) + lane % 4 / 2, by = lane % 2 * 8;
        auto vt = [&](int kk, int b) {
          return read_vt(tv, S::v_at(16 * kk + kr, 4 * b + pc) * 16 + by,
                         S::v_at(16 * kk + 8 + kr, 4 * b + pc) * 16 + by);
        };
        // probabilities rounded to bf16 (to nearest, 2^-9 of each at most): their sum l is
        // taken before, in fp32
        pbf16x8 pb[2 * NS];
#pragma unroll
        for (int kk = 0; kk < 2 * NS; ++kk) {
          pf32x8 x;
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = s[kk / 2][8 * (kk % 2) + i];
          pb[kk] = to_bf16x8(x);
        }
#pragma unroll
        for (int kk = 0; kk < 2 * NS; ++kk)
#pragma unroll
          for (int b = 0; b < NB; ++b)
            o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vt(kk, b), pb[kk], o[b], 0, 0, 0);
      } else {
        const float* tf = reinterpret_cast<const float*>(tv);
        auto vt = [&](int i, int b) {   // key of result element i, output 32 b + l32
          const int r = 8 * (i / 4) + 4 * half + i % 4;
          return tf[S::v_at(r, 8 * b + l32 / 4) * 4 + l32 % 4];
        };
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int b = 0; b < NB; ++b)
            o[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(vt(i, b), s[0][i], o[b], 0, 0, 0);
        }
      }
    }
    if (more) {
      if (!S::kBf16) load(j0 + BN, a.c.v, rv);
      stage(buf ^ 1, j0 + BN);
    }
  }

  __syncthreads();   // s_bad
  if (!has_rows || r0 + 32 * wave + l32 >= rows) return;
  l += __shfl_xor(l, 32, kWave);
  const int t = sp.c0 + tok, hq = h * a.G + g;
  const float mul = a.n_split > 1 ? 1.f : l > 0.f ? 1.f / l : l;   // no key: 0; NaN stays
  if (half == 0) store_ml(a, split, t, hq, m * a.scale_log2, l);
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d0 = 32 * b + 8 * i + 4 * half;
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = s_bad[d0 + e] < lim ? __builtin_nanf("") : o[b][4 * i + e] * mul;
      store4<T, D>(a, split, t, hq, d0, x);
    }
}

// ---------------------------------------------------------------------------
// The few-row kernel: a workgroup takes one (range, head, slot), its waves every fourth tile
// of 32 keys (fp32: 16).  K rows go from memory into A operands as they are, V rows
// through a piece of LDS that the wave has alone; the waves' states are joined at the
// end.  The next tile's rows are loaded as soon as this one's have left their registers.
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

template <typename T, int D>
__global__ __launch_bounds__(kBlock) void page_few_kernel(AttnArgs a) {
  using S = Few<T, D>;
  constexpr int BN = S::BN, NS = S::NS, PPR = S::PPR, NP = S::NP, KS = S::KS, NB = S::NB;
  static_assert(BN * PPR * 16 == kFewRows * D * 4, "a wave's V rows and its O take the same room");
  __shared__ u4 s_v[kWaves][BN * PPR];
  __shared__ float s_ml[kWaves][kFewRows][2];
  __shared__ int s_bad[D];

  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int l16 = lane % 16, quad = lane / 16;
  const uint32_t id = xcd_logical_block(blockIdx.x, gridDim.x);
  const int split = (int)(id % a.n_split), h = (int)(id / a.n_split) % a.c.H;
  const Span sp(a, (int)(id / a.n_split) / a.c.H);
  const int rows = sp.n * a.G;
  if (rows == 0) return;
  if (rows > kFewRows) {
    // the tile kernel's, unless max_new said that there is none of these
    if (a.split_rows == 0 && threadIdx.x == 0 && a.status) atomicOr(a.status, VASE_STATUS_PAGE_BAD);
    return;
  }
  const int row = min(l16, rows - 1);
  const int tok = row / a.G, g = row - tok * a.G;
  const int lim = sp.sees(a, tok);
  const int least = sp.sees(a, 0);
  const int kb = split * a.keys;
  const int ke = split < a.n_split - 1 ? min(sp.L, kb + a.keys) : sp.L;
  if (kb >= ke && a.n_split > 1) return;
  if (threadIdx.x < D) s_bad[threadIdx.x] = 0x7fffffff;
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
      const int64_t at = bases.at(j0 / 16 + n);
      const u4* kp = reinterpret_cast<const u4*>(a.c.k) + at + l16 * PPR + quad;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) rk[n][ks] = kp[4 * ks];
      const u4* vp = reinterpret_cast<const u4*>(a.c.v) + at + lane;
#pragma unroll
      for (int i = 0; i < NP / NS; ++i) rv[n * (NP / NS) + i] = vp[i * kWave];
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
      const int at = here(lane);
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
      const float alpha = m == -INFINITY ? 0.f : exp2_((m - now) * a.scale_log2);
      m = now;
      l *= alpha;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[b][i] *= alpha;
    }
    const float mc = m == -INFINITY ? 0.f : m * a.scale_log2;
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
      const pbf16x8 pb = to_bf16x8(x);   // rounded as in the tile kernel
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
      const float f = mw == -INFINITY ? 0.f : exp2_((mw - mm) * a.scale_log2);
      ll += s_ml[w][r][1] * f;
      const float4 y = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(s_v[w]) + r * D + d0);
      x[0] += y.x * f;
      x[1] += y.y * f;
      x[2] += y.z * f;
      x[3] += y.w * f;
    }
    const int ti = r / a.G, t = sp.c0 + ti, hq = h * a.G + r - ti * a.G;
    const float mul = a.n_split > 1 ? 1.f : ll > 0.f ? 1.f / ll : ll;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = s_bad[d0 + i] < sp.sees(a, ti) ? __builtin_nanf("") : x[i] * mul;
    store4<T, D>(a, split, t, hq, d0, x);
    if (d0 == 0) store_ml(a, split, t, hq, mm * a.scale_log2, ll);
  }
}

// ---------------------------------------------------------------------------
// A wave per (token, query head): the ranges that hold a key the token sees, joined in order.
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
  const bool few = sp.n * a.G <= a.split_rows;
  const int n_split = few ? a.few_split : a.n_split, keys = few ? a.few_keys : a.keys;
  if (n_split == 1) return;   // already written
  const int sees = sp.sees(a, t - sp.c0);
  const int n = min(n_split, (sees + keys - 1) / keys);
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
  const float f = m == -INFINITY ? 0.f : exp2_(m - top);
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
  if (a.lse && lane == 0) a.lse[at] = sum > 0.f ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
}

template <typename T, int D>
hipError_t launch_td(AttnArgs a, const PageAttnPlan& pl, hipStream_t stream) {
  if (pl.few) {
    AttnArgs f = a;
    f.n_split = pl.split_f;
    f.keys = pl.keys_f;
    f.split_rows = pl.tile ? kFewRows : 0;
    hipLaunchKernelGGL((page_few_kernel<T, D>), dim3((unsigned)(a.c.S * a.c.H * pl.split_f)), dim3(kBlock), 0,
                       stream, f);
  }
  a.n_split = pl.split_t;
  a.keys = pl.keys_t;
  a.split_rows = pl.few ? kFewRows : 0;
  if (pl.tile)
    hipLaunchKernelGGL((page_tile_kernel<T, D>), dim3((unsigned)(pl.n_tile * a.c.H * pl.split_t)), dim3(kBlock), 0,
                       stream, a);
  if (pl.split_t > 1 || pl.split_f > 1) {
    a.few_split = pl.split_f;
    a.few_keys = pl.keys_f;
    const int64_t n = (int64_t)a.T * a.HG;
    hipLaunchKernelGGL((page_combine_kernel<T, D>), dim3((unsigned)((n + kWaves - 1) / kWaves)), dim3(kBlock), 0,
                       stream, a);
  }
  return hipGetLastError();
}

// ranges of a multiple of `unit` keys, about `want` of them but none below `least` keys
void split_keys(int max_len, int64_t want, int least, int unit, int& n, int& keys) {
  int64_t s = want < kMaxSplit ? want : kMaxSplit;
  if (s > max_len / least) s = max_len / least;
  if (s < 1) s = 1;
  keys = (int)(((max_len + s - 1) / s + unit - 1) / unit * unit);
  n = (max_len + keys - 1) / keys;
}

}  // namespace

PageAttnPlan page_attn_plan(const vase_pages& c, int T, int G, int max_new, int max_len) {
  PageAttnPlan p;
  const int slots = c.S < T ? c.S : T;      // that can have tokens
  p.tile = (int64_t)max_new * G > kFewRows;
  p.few = !p.tile || (slots > 1 && (int64_t)T * G < 64 * (int64_t)slots);
  p.n_tile = (int)((int64_t)T * G / kTileRows) + c.S;
  p.split_t = p.split_f = 1;
  p.keys_t = p.keys_f = max_len;
  // a range is worth its partials from about 512 keys (tile) or 256 (few) on
  if (p.tile) {
    const int64_t wgs = ((int64_t)T * G / kTileRows + 1) * c.H;
    split_keys(max_len, 512 / wgs, 512, 64, p.split_t, p.keys_t);
  }
  if (p.few) split_keys(max_len, 2048 / ((int64_t)slots * c.H) + 1, 256, 128, p.split_f, p.keys_f);
  const int n = p.split_t > p.split_f ? p.split_t : p.split_f;
  const size_t rows = (size_t)T * c.H * G;
  p.off_ml = n > 1 ? (size_t)n * rows * c.d * sizeof(float) : 0;
  p.bytes = n > 1 ? p.off_ml + (size_t)n * rows * 2 * sizeof(float) : 0;
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
  a.part_ml = ws ? reinterpret_cast<float*>(static_cast<char*>(ws) + plan.off_ml) : nullptr;
  a.n_tile = plan.n_tile;
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)c.d);
  a.status = status;
  if (c.dtype == VASE_BF16)
    return c.d == 128 ? launch_td<bf16_t, 128>(a, plan, stream) : launch_td<bf16_t, 64>(a, plan, stream);
  return c.d == 128 ? launch_td<float, 128>(a, plan, stream) : launch_td<float, 64>(a, plan, stream);
}

}  // namespace vase
