// Attention of a unit's query rows over its cache under a causal mask, a sliding window and first rows that stay visible:
//   out[q] = sum_t exp(e_t) V[t] / sum_t c_t exp(e_t),   e_t = scale * q . k_t,   over the rows t that q sees
// (sees()); a query that sees none gets zeros.  The cache is plain rows (fp32, bf16) or rows in 4 bits.
//
// A workgroup takes a block of 16 or 32 (16 NQ) query rows of one unit and a piece of the rows that they see; its wavefronts take
// the piece's tiles of 32 rows in turn, each with a softmax of its own (running maximum, denominator and numerators), and
// never wait for each other until the piece is done.  Both products are on the matrix cores, 16 query rows per column
// block (a decode step of one token has 4 to 8, so that 16 waste the least), and nothing passes through LDS:
//   S = K Q^T       the lane's row of K as it lies in memory (the contraction index, a channel, may be split between the
//                   lane groups in any way that both operands share);
//   O^T += V^T P    a lane holds D / 16 neighbouring channels of the eight rows that are its share of the contraction:
//                   those whose logits the first product has left in the same lane group, so that P is already in
//                   operand order.  bf16 pairs of neighbouring channels become pairs of neighbouring rows by byte moves.
// Memory bounds it.  Plain rows: one token on 64 caches of 8224 rows, 269 MB, 41 us (6.5 TB/s, part of it from the memory-side
// cache) and 4 to 5 for adding up the pieces; 256 of 4096 93 us (5.8 TB/s).  Rows in 4 bits: 147 MB in 30 us (4.9 TB/s) with 4 query
// rows, 143 MB in 39 (3.7) with 32, where vector work (64 conversions, 32 byte moves and 16 exponentials per lane and tile) is
// next.  Short calls are two launches of 5.8 and 3.5 us, a chain of dependent trips to memory each.
// 4-bit rows are turned into bf16 in registers (exact: four significant bits times a power of two), two values per
// instruction, and fp32 rows go through the fp32 matrix instructions.
//
// A product with P = 0 is not nothing where V is not finite, so in a tile that some query of the block does not see whole
// such values are left out of the product; when the piece is done they are added for the queries that see their row.
#include <type_traits>

#include "kvs_fp4.h"
#include "kvs_window.h"

namespace kvs {
namespace {

using fp4::scale_of;
using fp4::two_of;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = kWindowTile;
constexpr int kReduceThreads = 256;

// Of a tile: one base, the same for all lanes, and 32-bit offsets.
template <typename T>
__device__ __forceinline__ T at(const char* base, uint32_t offset) { return *(const T*)(base + offset); }

// x as a sum of N bf16 numbers, each the rounding of what the ones before leave (N = 3: 2^-24 of x, the last bit
// of fp32; N = 2: 2^-16).  An infinity or NaN stays one in the first.
template <int N>
__device__ __forceinline__ void split8(const float (&x)[8], bf16x8 (&s)[N]) {
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = x[i];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = cvt_pk_bf16(r[2 * i], r[2 * i + 1]);
    s[n] = __builtin_bit_cast(bf16x8, w);
    if (n + 1 < N) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float lo = bf16_lo(w[i]), hi = bf16_hi(w[i]);
        // (what is left of an infinity would be a NaN)
        r[2 * i] = __builtin_isfinite(lo) ? r[2 * i] - lo : 0.f;
        r[2 * i + 1] = __builtin_isfinite(hi) ? r[2 * i + 1] - hi : 0.f;
      }
    }
  }
}

// What a wavefront reads of a tile of 32 rows.  Lane l of the wavefront is column / row c = l % 16 of lane group g = l / 16;
// key rows: 16 h + c (h = 0, 1), value rows: i < 4: 4 g + i, else 12 + 4 g + i.  A tile that its range's end cuts is read row by
// row (rows past the end repeat the last one), any other from one address per lane.
__device__ __forceinline__ int value_row(int g, int i) { return (i < 4 ? 0 : 12) + 4 * g + i; }
typedef uint32_t u32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_at2 __attribute__((ext_vector_type(2), aligned(2)));

template <CacheKind KIND, int D> struct Rows;

template <int D>
struct Rows<CacheKind::kBf16, D> {
  typedef uint16_t Io;
  static constexpr bool kMatrixF32 = false;
  static constexpr int kQ = 1, kP = 2;     // bf16 numbers that a query value and a weight are taken as
  static constexpr int kSteps = D / 32;
  static constexpr int CPL = D / 16;       // channels of a value row per lane
  typedef uint32_t vpiece __attribute__((ext_vector_type(CPL / 2)));
  u32x4 k[2][kSteps];
  vpiece v[8];
  static __device__ __forceinline__ int channel(int s, int g) { return 32 * s + 8 * g; }
  // t0: the tile's first row within the unit, last: its last row within the tile
  __device__ __forceinline__ void load_keys(const Cache& cache, size_t row0, int t0, int last, int c, int g) {
    const char* base = (const char*)cache.k + (row0 + t0) * (2 * D);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t row = last >= kTile - 1 ? 16 * h + c : min(16 * h + c, last);
#pragma unroll
      for (int s = 0; s < kSteps; ++s) k[h][s] = at<u32x4>(base, row * (2 * D) + 16 * g + 64 * s);
    }
  }
  __device__ __forceinline__ void load_values(const Cache& cache, size_t row0, int t0, int last, int c, int g) {
    const char* base = (const char*)cache.v + (row0 + t0) * (2 * D);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t row = last >= kTile - 1 ? value_row(g, i) : min(value_row(g, i), last);
      v[i] = at<vpiece>(base, row * (2 * D) + c * (D / 8));
    }
  }
  __device__ __forceinline__ bf16x8 key(int h, int s) const { return __builtin_bit_cast(bf16x8, k[h][s]); }
  // channels 2 W, 2 W + 1 of the lane's
  template <int W> __device__ __forceinline__ uint32_t value(int i, int) const { return v[i][W]; }
};

template <int D, bool F32>
struct PackedRows {
  typedef std::conditional_t<F32, float, uint16_t> Io;
  static constexpr bool kMatrixF32 = false;
  // (one number per weight: its error, at most 2^-8 and of any sign, is far below that of the rows)
  static constexpr int kQ = F32 ? 3 : 1, kP = F32 ? 3 : 1;
  static constexpr int kSteps = D / 32;
  static constexpr int CPL = D / 16;
  typedef uint32_t kpiece __attribute__((ext_vector_type(D / 32)));
  typedef std::conditional_t<D == 128, uint32_t, uint16_t> vpiece;
  kpiece k[2];
  uint8_t ks[2];
  vpiece v[8];
  uint32_t vs[D == 128 ? 8 : 4];           // the value rows' scales, all of a row's beside each other
  static __device__ __forceinline__ int channel(int s, int g) { return (D / 4) * g + 8 * s; }
  __device__ __forceinline__ void load_keys(const Cache& cache, size_t row0, int t0, int last, int c, int g) {
    const char* base = (const char*)cache.k + (row0 + t0) * (D / 2);
    const char* scales = (const char*)cache.ks + (row0 + t0) * (D / 32);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t row = last >= kTile - 1 ? 16 * h + c : min(16 * h + c, last);
      k[h] = at<kpiece>(base, row * (D / 2) + g * (D / 8));
      ks[h] = at<uint8_t>(scales, row * (D / 32) + g * (D / 4) / 32);
    }
  }
  __device__ __forceinline__ void load_values(const Cache& cache, size_t row0, int t0, int last, int c, int g) {
    const char* base = (const char*)cache.v + (row0 + t0) * (D / 2);
    const char* scales = (const char*)cache.vs + (row0 + t0) * (D / 32);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t row = last >= kTile - 1 ? value_row(g, i) : min(value_row(g, i), last);
      v[i] = at<vpiece>(base, row * (D / 2) + c * (D / 32));
    }
    if (last >= kTile - 1) {                 // four rows' scales lie together
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if constexpr (D == 128) {
          const u32x4_at4 x = at<u32x4_at4>(scales, (16 * h + 4 * g) * 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) vs[4 * h + i] = x[i];
        } else {
          const u32x2_at2 x = at<u32x2_at2>(scales, (16 * h + 4 * g) * 2);
          vs[2 * h] = x[0];
          vs[2 * h + 1] = x[1];
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t row = min(value_row(g, i), last);
        if constexpr (D == 128) vs[i] = at<uint32_t>(scales, row * 4);
        else if (i % 2 == 0) vs[i / 2] = at<uint16_t>(scales, row * 2);
        else vs[i / 2] |= (uint32_t)at<uint16_t>(scales, row * 2) << 16;
      }
    }
  }
  __device__ __forceinline__ bf16x8 key(int h, int s) const {
    const float sc = scale_of(ks[h]);
    const u32x4 w = {two_of<0>(k[h][s], sc), two_of<1>(k[h][s], sc), two_of<2>(k[h][s], sc), two_of<3>(k[h][s], sc)};
    return __builtin_bit_cast(bf16x8, w);
  }
  template <int W> __device__ __forceinline__ uint32_t value(int i, int c) const {
    // byte c / 4 (D = 64: c / 8, of the upper half-word for an odd row) turned to where a float has its exponent, which is all
    // that the conversion looks at
    const uint32_t s = D == 128 ? vs[i] : vs[i / 2];
    const uint32_t by = D == 128 ? c / 4 * 8 + 9 : c / 8 * 8 + i % 2 * 16 + 9;
    return two_of<W>(v[i], __uint_as_float(__builtin_amdgcn_alignbit(s, s, by)));
  }
};
template <int D> struct Rows<CacheKind::kPackedBf16, D> : PackedRows<D, false> {};
template <int D> struct Rows<CacheKind::kPackedF32, D> : PackedRows<D, true> {};

template <int D>
struct Rows<CacheKind::kF32, D> {
  typedef float Io;
  static constexpr bool kMatrixF32 = true;
  static constexpr int kQ = 1, kP = 1;
  static constexpr int kSteps = D / 16;
  f32x4 k[2][kSteps];
  f32x4 v[8][D / 64];
  static __device__ __forceinline__ int channel(int s, int g) { return 16 * s + 4 * g; }
  __device__ __forceinline__ void load_keys(const Cache& cache, size_t row0, int t0, int last, int c, int g) {
    const char* base = (const char*)cache.k + (row0 + t0) * (4 * D);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t row = last >= kTile - 1 ? 16 * h + c : min(16 * h + c, last);
#pragma unroll
      for (int s = 0; s < kSteps; ++s) k[h][s] = at<f32x4>(base, row * (4 * D) + 16 * g + 64 * s);
    }
  }
  __device__ __forceinline__ void load_values(const Cache& cache, size_t row0, int t0, int last, int c, int g) {
    const char* base = (const char*)cache.v + (row0 + t0) * (4 * D);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t row = last >= kTile - 1 ? value_row(g, i) : min(value_row(g, i), last);
#pragma unroll
      for (int e = 0; e < D / 64; ++e) v[i][e] = at<f32x4>(base, row * (4 * D) + 16 * c + 256 * e);
    }
  }
};

// The block's query rows as the second operand of S = K Q^T.
template <typename L, int D, int NQ>
struct Queries {
  std::conditional_t<L::kMatrixF32, f32x4, bf16x8> q[NQ][L::kQ][L::kSteps];
  __device__ __forceinline__ void load(const typename L::Io* Q, const WindowShape& sh, int unit, int row0, int c, int g) {
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const int r = min(row0 + 16 * n + c, sh.R - 1);        // rows past R repeat the last one
      const typename L::Io* src = Q + query_row(sh, unit, r) * D;
#pragma unroll
      for (int s = 0; s < L::kSteps; ++s) {
        const typename L::Io* at = src + L::channel(s, g);
        if constexpr (L::kMatrixF32) {
          q[n][0][s] = *(const f32x4*)at;
        } else if constexpr (std::is_same_v<typename L::Io, float>) {
          float x[8];
          *(f32x4*)&x[0] = *(const f32x4*)at;
          *(f32x4*)&x[4] = *((const f32x4*)at + 1);
          bf16x8 part[L::kQ];
          split8<L::kQ>(x, part);
#pragma unroll
          for (int k = 0; k < L::kQ; ++k) q[n][k][s] = part[k];
        } else {
          q[n][0][s] = *(const bf16x8*)at;
        }
      }
    }
  }
};

// First of the four neighbouring channels that accumulators 4 j4 .. 4 j4 + 3 of O^T hold in accumulator row r.
template <bool F32, int D>
__device__ __forceinline__ int channel_of(int j4, int r) {
  return F32 ? 64 * j4 + 4 * r : (D / 16) * r + 4 * j4;
}

template <typename T>
__device__ __forceinline__ void store_two(T* at, float a, float b) {
  if constexpr (std::is_same_v<T, float>) *(float2*)at = make_float2(a, b);
  else *(uint32_t*)at = cvt_pk_bf16(a, b);
}

// Wavefronts per SIMD that the registers are allotted for: the operands of a tile and of the queries, and the accumulators.  One
// more would have some of them spilled (fp32 queries over rows in 4 bits of 128 channels, one token on 256 caches of 4096 rows:
// 43.6 us with two wavefronts, 47.7 with three, with cardinalities 51 and 105; listed units with cardinalities, 32 query rows on 64
// caches of 2250 to 9000 bf16 rows: 52 us with one, 85 with two).
template <CacheKind KIND, int D, int NQ, bool COUNTS, typename Tab>
constexpr int waves_per_simd() {
  if (KIND == CacheKind::kF32 || KIND == CacheKind::kPackedF32) return (NQ == 1 ? 2 : 1) + (D == 64);
  if (KIND == CacheKind::kBf16) return NQ == 2 && D == 128 && COUNTS && Tab::kListed ? 1 : 2;
  return NQ == 1 ? 3 : 2;
}

template <CacheKind KIND, int D, int NQ, int WAVES, bool COUNTS, typename Tab>
__global__ __launch_bounds__(WAVES * kWave, (waves_per_simd<KIND, D, NQ, COUNTS, Tab>())) void window_rows_kernel(
    const Tab tab, const WindowShape sh, const Cache cache, const void* __restrict__ Q, void* __restrict__ out,
    float* __restrict__ part) {
  typedef Rows<KIND, D> L;
  typedef typename L::Io Io;
  constexpr bool F32 = L::kMatrixF32;
  constexpr int NJ = D / 16;                // accumulators of O^T per column block
  constexpr int ACCW = D + 4;               // numerators, maximum, denominator; rows stay 16-byte aligned
  __shared__ __attribute__((aligned(16))) float sm_acc[WAVES][16][ACCW];

  const int id = blockIdx.x;
  int piece = 0, block, at_unit;
  if (Tab::kListed || sh.n_parts == 1) {
    block = id % sh.n_blocks;
    at_unit = id / sh.n_blocks;
    if constexpr (Tab::kListed) {
      if (sh.n_parts > 1) {
        piece = at_unit + tab.before;
        at_unit = tab.unit_of(at_unit);
        piece -= tab.entry(at_unit).before;
      }
    }
  } else {
    piece = id % sh.n_parts;
    block = id / sh.n_parts % sh.n_blocks;
    at_unit = id / sh.n_parts / sh.n_blocks;
  }
  const CacheUnit un = tab.unit(sh, at_unit);
  const Reach re = reach_of<kTile>(sh, un.len, block);
  const int n_parts = parts_of(re.tiles, sh.part_tiles);
  if (piece >= n_parts) return;             // (a block whose reach is shorter than others of the unit)
  const int tile1 = min(re.tiles, (piece + 1) * sh.part_tiles);
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
  const int c = lane % 16, g = lane / 16;
  const int row0 = block * sh.block;

  int pos[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    pos[n] = sh.causal ? un.len - sh.W + min(row0 + 16 * n + c, sh.R - 1) / sh.G : un.len - 1;
  }
  f32x4 acc[NQ][NJ];
  float m[NQ], l[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m[n] = -INFINITY;
    l[n] = 0.f;
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  int j = piece * sh.part_tiles + wave;
  if (j < tile1) {
    Queries<L, D, NQ> qs;
    qs.load((const Io*)Q, sh, un.index, row0, c, g);
    // tile j: its first row, and the end of the range of rows that it is in (rows past it repeat the last one)
    auto start_of = [&](int t) { return t < re.sink_tiles ? t * kTile : re.first + (t - re.sink_tiles) * kTile; };
    auto end_of = [&](int t) { return t < re.sink_tiles ? re.sink_end : re.end; };
    // every row of the tile is seen by the whole block
    auto seen_whole = [&](int t0, int end) {
      return t0 + kTile <= end && t0 + kTile - 1 <= re.pos_min &&
             (sh.span == 0 || t0 > re.pos_max - sh.span || t0 + kTile <= sh.sinks);
    };
    L rows;
    uint32_t cnt[8];
    auto load_keys = [&](int t) __attribute__((always_inline)) {
      const int t0 = start_of(t);
      rows.load_keys(cache, un.in_row, t0, end_of(t) - 1 - t0, c, g);
    };
    auto load_values = [&](int t) __attribute__((always_inline)) {
      const int t0 = start_of(t), last = end_of(t) - 1 - t0;
      rows.load_values(cache, un.in_row, t0, last, c, g);
      if constexpr (COUNTS) {
        const char* base = (const char*)(cache.counts + un.in_row + t0);
        if (last >= kTile - 1) {               // four rows' cardinalities lie together
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const u32x4_at4 x = at<u32x4_at4>(base, (16 * h + 4 * g) * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) cnt[4 * h + i] = x[i];
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) cnt[i] = at<uint32_t>(base, min(value_row(g, i), last) * 4);
        }
      }
    };
    const int j0 = j;
    bool odd = false;                       // a value that is not finite was left out
    load_keys(j);
    load_values(j);
    while (true) {
      const int t0 = start_of(j), end = end_of(j);
      const int next = j + WAVES;
      // S[t, q]: element v of half h is row 16 h + 4 g + v of the tile, query column c
      f32x4 s[NQ][2];
#pragma unroll
      for (int n = 0; n < NQ; ++n) s[n][0] = s[n][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int st = 0; st < L::kSteps; ++st) {
          if constexpr (F32) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
#pragma unroll
              for (int n = 0; n < NQ; ++n)
                s[n][h] = __builtin_amdgcn_mfma_f32_16x16x4f32(rows.k[h][st][e], qs.q[n][0][st][e], s[n][h], 0, 0, 0);
            }
          } else {
            const bf16x8 a = rows.key(h, st);
#pragma unroll
            for (int k = L::kQ - 1; k >= 0; --k) {           // (the small parts first)
#pragma unroll
              for (int n = 0; n < NQ; ++n)
                s[n][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qs.q[n][k][st], s[n][h], 0, 0, 0);
            }
          }
        }
      }
      if (next < tile1) load_keys(next);
      const bool whole = seen_whole(t0, end);
      float p[NQ][8];
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) p[n][i] = s[n][i / 4][i % 4];
        if (!whole) {
          // the lane's rows are x = i or 12 + i plus this: limits that x is compared with
          const int base = t0 + 4 * g, before_sinks = sh.sinks - base;
          const int last = min(pos[n], end - 1) - base;
          const int hidden = sh.span > 0 ? pos[n] - sh.span - base : -1 - base;  // rows up to here are seen as sinks only
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int x = value_row(0, i);
            p[n][i] = (x <= last) & ((x > hidden) | (x < before_sinks)) ? p[n][i] : -INFINITY;
          }
        }
#pragma unroll
        for (int i = 0; i < 8; i += 2) top = fmaxf(fmaxf(top, p[n][i]), p[n][i + 1]);
        top *= sh.scale_log2;
        if (__ballot(top > m[n] + kSlack) != 0) {            // rare after the first tiles
          top = fmaxf(top, __shfl_xor(top, 16, kWave));      // the four lane groups feed the same columns of O^T
          top = fmaxf(top, __shfl_xor(top, 32, kWave));
          top = fmaxf(top, m[n]);
          const float corr = m[n] == top ? 1.f : __builtin_amdgcn_exp2f(m[n] - top);
          l[n] *= corr;
#pragma unroll
          for (int k = 0; k < NJ; ++k) acc[n][k] *= corr;
          m[n] = top;
        }
        const float ref = m[n] == -INFINITY ? 0.f : m[n];    // (a query that has seen nothing yet)
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[n][i] = __builtin_amdgcn_exp2f(fmaf(p[n][i], sh.scale_log2, -ref));
          if constexpr (COUNTS) sum = fmaf((float)(int)cnt[i], p[n][i], sum);   // c copies of the slot in the denominator
          else sum += p[n][i];
        }
        l[n] += sum;
      }
      // V^T: of bf16 pairs of channels become pairs of rows, operand k is channel k of the lane's, element i the lane's row i
      u32x4 vt[F32 ? 1 : NJ];
      if constexpr (!F32) {
        auto turn = [&](auto w) {
          constexpr int W2 = decltype(w)::value;
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            const uint32_t a = rows.template value<W2>(i, c), b = rows.template value<W2>(i + 1, c);
            vt[2 * W2][i / 2] = __builtin_amdgcn_perm(b, a, 0x05040100u);
            vt[2 * W2 + 1][i / 2] = __builtin_amdgcn_perm(b, a, 0x07060302u);
          }
        };
        turn(std::integral_constant<int, 0>{});
        turn(std::integral_constant<int, 1>{});
        if constexpr (NJ == 8) {
          turn(std::integral_constant<int, 2>{});
          turn(std::integral_constant<int, 3>{});
        }
      }
      if (!whole) {
#pragma unroll
        for (int k = 0; k < NJ; ++k) {
          if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float x = rows.v[i][k / 4][k % 4];
              const bool bad = !__builtin_isfinite(x);
              odd |= bad;
              rows.v[i][k / 4][k % 4] = bad ? 0.f : x;
            }
          } else {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const uint32_t x = vt[k][w];
              const bool lo = (x & 0x7f80u) == 0x7f80u, hi = (x & 0x7f800000u) == 0x7f800000u;
              odd |= lo | hi;
              vt[k][w] = x & ((lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u));
            }
          }
        }
      }
      if constexpr (F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
#pragma unroll
          for (int k = 0; k < NJ; ++k) {
#pragma unroll
            for (int n = 0; n < NQ; ++n)
              acc[n][k] = __builtin_amdgcn_mfma_f32_16x16x4f32(rows.v[i][k / 4][k % 4], p[n][i], acc[n][k], 0, 0, 0);
          }
        }
      } else {
        bf16x8 pp[NQ][L::kP];
#pragma unroll
        for (int n = 0; n < NQ; ++n) split8<L::kP>(p[n], pp[n]);
#pragma unroll
        for (int k = 0; k < NJ; ++k) {
#pragma unroll
          for (int h = L::kP - 1; h >= 0; --h) {
#pragma unroll
            for (int n = 0; n < NQ; ++n)
              acc[n][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vt[k]), pp[n][h], acc[n][k], 0, 0, 0);
          }
        }
      }
      if (next >= tile1) break;
      load_values(next);
      j = next;
    }
    if (__ballot(odd) != 0) {
      // What is not finite makes the sums of the queries that see it what it is itself, whatever its weight.
      for (j = j0; j < tile1; j += WAVES) {
        const int t0 = start_of(j), end = end_of(j);
        if (seen_whole(t0, end)) continue;
#pragma unroll 1
        for (int t = t0; t < min(t0 + kTile, end); ++t) {
#pragma unroll
          for (int j4 = 0; j4 < NJ / 4; ++j4) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const f32x4 y = four_values<KIND, D>(cache, un.in_row + t, channel_of<F32, D>(j4, 4 * g + v));
#pragma unroll
              for (int n = 0; n < NQ; ++n) {
                const bool seen = sees(sh, pos[n], t);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[n][4 * j4 + e][v] += seen && !__builtin_isfinite(y[e]) ? y[e] : 0.f;
              }
            }
          }
        }
      }
    }
  }

  // the wavefronts of the workgroup, in wavefront order
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    float den = l[n] + __shfl_xor(l[n], 16, kWave);
    den += __shfl_xor(den, 32, kWave);
    if (n > 0) __syncthreads();
#pragma unroll
    for (int j4 = 0; j4 < NJ / 4; ++j4) {
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        *(float4*)&sm_acc[wave][c][channel_of<F32, D>(j4, 4 * g + v)] =
            make_float4(acc[n][4 * j4][v], acc[n][4 * j4 + 1][v], acc[n][4 * j4 + 2][v], acc[n][4 * j4 + 3][v]);
      }
    }
    if (g == 0) { sm_acc[wave][c][D] = m[n]; sm_acc[wave][c][D + 1] = den; }
    __syncthreads();
    for (int o = tid; o < 16 * D / 2; o += WAVES * kWave) {
      const int q = o / (D / 2), ch = o % (D / 2) * 2, row = row0 + 16 * n + q;
      if (row >= min(sh.R, row0 + sh.block)) continue;
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) M = fmaxf(M, sm_acc[w][q][D]);
      float a = 0.f, b = 0.f, den_q = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const float lw = sm_acc[w][q][D + 1];
        if (lw != 0.f) {                                     // (a wavefront that saw no row has m = -inf)
          const float wgt = __builtin_amdgcn_exp2f(sm_acc[w][q][D] - M);
          a = fmaf(sm_acc[w][q][ch], wgt, a);
          b = fmaf(sm_acc[w][q][ch + 1], wgt, b);
          den_q = fmaf(lw, wgt, den_q);
        }
      }
      if (n_parts == 1) {
        store_two((Io*)out + query_row(sh, un.index, row) * D + ch, quotient(a, den_q), quotient(b, den_q));
      } else {
        float* dst = part + part_at(sh, un, row, piece);
        *(float2*)(dst + ch) = make_float2(a, b);
        if (ch == 0) { dst[D] = M; dst[D + 1] = den_q; }
      }
    }
  }
}

// out[row] from its pieces, in order.  One workgroup per (unit, query row): thread (g, d) adds up every PARTS-th piece of
// channel d, and the sums are added in order.
template <typename Io, int D, int TILE, typename Tab>
__global__ __launch_bounds__(kReduceThreads) void window_reduce_kernel(const Tab tab, const WindowShape sh, int unit0,
                                                                       const float* __restrict__ part,
                                                                       void* __restrict__ out) {
  constexpr int PARTS = kReduceThreads / D;
  __shared__ float sm_w[kMaxParts];
  __shared__ float sm_num[PARTS][D];
  __shared__ float sm_top[kReduceThreads / kWave], sm_den[kReduceThreads / kWave];
  const CacheUnit un = tab.unit(sh, unit0 + blockIdx.x / sh.R);
  const int row = blockIdx.x % sh.R;
  const int n = parts_of(reach_of<TILE>(sh, un.len, row / sh.block).tiles, sh.part_tiles);
  if (n == 1) return;                      // (stored already)
  const float* src = part + part_at(sh, un, row, 0);
  const size_t step = (size_t)sh.R * (D + 2);
  const int tid = threadIdx.x, d = tid % D, g = tid / D;
  const float m = tid < n ? src[tid * step + D] : -INFINITY;
  const float l = tid < n ? src[tid * step + D + 1] : 0.f;
  float M = m;
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) M = fmaxf(M, __shfl_xor(M, k, kWave));
  if (tid % kWave == 0) sm_top[tid / kWave] = M;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kReduceThreads / kWave; ++w) M = fmaxf(M, sm_top[w]);
  const float wgt = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - M);
  if (tid < n) sm_w[tid] = wgt;
  float den = l == 0.f ? 0.f : l * wgt;
#pragma unroll
  for (int k = 1; k < kWave; k <<= 1) den += __shfl_xor(den, k, kWave);
  if (tid % kWave == 0) sm_den[tid / kWave] = den;
  __syncthreads();
  float num = 0.f;
  for (int i0 = g; i0 < n; i0 += 8 * PARTS) {                // eight loads at a time
    float x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = src[min(i0 + u * PARTS, n - 1) * step + d];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (i0 + u * PARTS < n) num = fmaf(x[u], sm_w[i0 + u * PARTS], num);
    }
  }
  sm_num[g][d] = num;
  __syncthreads();
  if (tid < D / 2) {
    float a = 0.f, b = 0.f, total = 0.f;
#pragma unroll
    for (int i = 0; i < PARTS; ++i) { a += sm_num[i][2 * tid]; b += sm_num[i][2 * tid + 1]; }
#pragma unroll
    for (int w = 0; w < kReduceThreads / kWave; ++w) total += sm_den[w];
    store_two((Io*)out + query_row(sh, un.index, row) * D + 2 * tid, quotient(a, total), quotient(b, total));
  }
}

// The same where no reach has more than kFewParts pieces: a thread takes two channels of a query row and requests everything at
// once, so that the partials cost one round trip and nobody meets.
constexpr int kFewParts = 8;
template <typename Io, int D, int TILE, typename Tab>
__global__ __launch_bounds__(kReduceThreads) void window_reduce_few_kernel(const Tab tab, const WindowShape sh, int unit0,
                                                                           int n_rows,
                                                                           const float* __restrict__ part,
                                                                           void* __restrict__ out) {
  constexpr int PER = D / 2;               // threads per row
  const int at = (int)blockIdx.x * (kReduceThreads / PER) + (int)threadIdx.x / PER, ch = (int)threadIdx.x % PER * 2;
  if (at >= n_rows) return;
  const CacheUnit un = tab.unit(sh, unit0 + at / sh.R);
  const int row = at % sh.R;
  const int n = parts_of(reach_of<TILE>(sh, un.len, row / sh.block).tiles, sh.part_tiles);
  if (n == 1) return;                      // (stored already)
  const float* src = part + part_at(sh, un, row, 0);
  float2 x[kFewParts], ml[kFewParts];
#pragma unroll
  for (int i = 0; i < kFewParts; ++i) {
    const float* p = src + (size_t)min(i, n - 1) * sh.R * (D + 2);
    x[i] = *(const float2*)(p + ch);
    ml[i] = *(const float2*)(p + D);
  }
  float M = -INFINITY;
#pragma unroll
  for (int i = 0; i < kFewParts; ++i) M = fmaxf(M, ml[i].x);
  float a = 0.f, b = 0.f, den = 0.f;
#pragma unroll
  for (int i = 0; i < kFewParts; ++i) {
    if (i < n && ml[i].y != 0.f) {
      const float wgt = __builtin_amdgcn_exp2f(ml[i].x - M);
      a = fmaf(x[i].x, wgt, a);
      b = fmaf(x[i].y, wgt, b);
      den = fmaf(ml[i].y, wgt, den);
    }
  }
  store_two((Io*)out + query_row(sh, un.index, row) * D + ch, quotient(a, den), quotient(b, den));
}

// Unit descriptors of a launch that has too many for its arguments, stored by a kernel that carries some in its own.
constexpr int kTableBatch = 224;
struct UnitBatch { UnitEntry u[kTableBatch]; };
__global__ __launch_bounds__(256) void unit_table_kernel(const UnitBatch batch, int n, UnitEntry* __restrict__ dst) {
  const int i = threadIdx.x;
  if (i < n) dst[i] = batch.u[i];
}

template <CacheKind KIND, int D, typename Tab>
hipError_t launch_kind(const Tab& tab, const WindowShape& sh, const Cache& cache, const void* Q, void* out, float* part,
                       hipStream_t stream) {
  const dim3 grid((unsigned)(pieces_of(tab, sh) * sh.n_blocks));
  auto go = [&](auto nq, auto counts, auto waves) {
    constexpr int NQ = decltype(nq)::value, WAVES = decltype(waves)::value;
    hipLaunchKernelGGL((window_rows_kernel<KIND, D, NQ, WAVES, decltype(counts)::value, Tab>), grid, dim3(WAVES * kWave), 0,
                       stream, tab, sh, cache, Q, out, part);
  };
  auto counted = [&](auto nq, auto counts) {
    constexpr int MANY = 4 * waves_per_simd<KIND, D, decltype(nq)::value, decltype(counts)::value, Tab>();
    if (sh.large) go(nq, counts, std::integral_constant<int, MANY>{});
    else go(nq, counts, std::integral_constant<int, 4>{});
  };
  auto sized = [&](auto nq) {
    if (cache.counts) counted(nq, std::true_type{});
    else counted(nq, std::false_type{});
  };
  if (sh.block == 16) sized(std::integral_constant<int, 1>{});
  else sized(std::integral_constant<int, 2>{});
  return hipGetLastError();
}

template <CacheKind KIND, typename Tab>
hipError_t launch_d(const Tab& tab, const WindowShape& sh, const Cache& cache, const void* Q, void* out, float* part,
                    hipStream_t stream) {
  return sh.D == 64 ? launch_kind<KIND, 64>(tab, sh, cache, Q, out, part, stream)
                    : launch_kind<KIND, 128>(tab, sh, cache, Q, out, part, stream);
}

template <typename Tab>
hipError_t launch_tab(const Tab& tab, const WindowShape& sh, CacheKind kind, const Cache& cache, const void* Q, void* out,
                      float* part, hipStream_t stream) {
  switch (kind) {
    case CacheKind::kF32: return launch_d<CacheKind::kF32>(tab, sh, cache, Q, out, part, stream);
    case CacheKind::kBf16: return launch_d<CacheKind::kBf16>(tab, sh, cache, Q, out, part, stream);
    case CacheKind::kPackedF32: return launch_d<CacheKind::kPackedF32>(tab, sh, cache, Q, out, part, stream);
    default: return launch_d<CacheKind::kPackedBf16>(tab, sh, cache, Q, out, part, stream);
  }
}

}  // namespace

hipError_t launch_window_rows(const EqualUnits* equal, const ListedUnits* listed, const WindowShape& sh, CacheKind kind,
                              const Cache& cache, const void* Q, void* out, float* part, hipStream_t stream) {
  return equal ? launch_tab(*equal, sh, kind, cache, Q, out, part, stream)
               : launch_tab(*listed, sh, kind, cache, Q, out, part, stream);
}

hipError_t launch_window_reduce(const EqualUnits* equal, const ListedUnits* listed, int at, int n, const WindowShape& sh, bool f32,
                                int tile, const float* part, void* out, hipStream_t stream) {
  const int rows = n * sh.R;
  auto go = [&](const auto& tab, auto io, auto d, auto t) {
    constexpr int D = decltype(d)::value, TILE = decltype(t)::value, PER = kReduceThreads / (D / 2);
    typedef std::decay_t<decltype(tab)> Tab;
    if (sh.n_parts <= kFewParts) {
      hipLaunchKernelGGL((window_reduce_few_kernel<decltype(io), D, TILE, Tab>), dim3((rows + PER - 1) / PER),
                         dim3(kReduceThreads), 0, stream, tab, sh, at, rows, part, out);
    } else {
      hipLaunchKernelGGL((window_reduce_kernel<decltype(io), D, TILE, Tab>), dim3(rows), dim3(kReduceThreads), 0, stream, tab,
                         sh, at, part, out);
    }
  };
  auto typed = [&](const auto& tab, auto d) {
    if (f32) go(tab, float{}, d, std::integral_constant<int, kWindowTile>{});
    else if (tile == kWindowTile) go(tab, uint16_t{}, d, std::integral_constant<int, kWindowTile>{});
    else go(tab, uint16_t{}, d, std::integral_constant<int, kWideTile>{});
  };
  auto sized = [&](const auto& tab) {
    if (sh.D == 64) typed(tab, std::integral_constant<int, 64>{});
    else typed(tab, std::integral_constant<int, 128>{});
  };
  if (equal) sized(*equal);
  else sized(*listed);
  return hipGetLastError();
}

hipError_t launch_window_table(const kvs_problem* p, const WindowShape& sh, int tile, UnitEntry* dst, hipStream_t stream) {
  int before = 0;
  for (int at = 0; at < p->n_units; at += kTableBatch) {
    const int n = p->n_units - at < kTableBatch ? p->n_units - at : kTableBatch;
    UnitBatch batch = {};
    for (int i = 0; i < n; ++i) {
      batch.u[i] = {(long long)p->in_row[at + i], (int)p->len[at + i], before};
      before += unit_pieces(sh, p->len[at + i], tile);
    }
    hipLaunchKernelGGL(unit_table_kernel, dim3(1), dim3(256), 0, stream, batch, n, dst + at);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace kvs
