// The attention of kvs_window_rows.hip for more than 32 bf16 query rows: a prompt, a chunk of new tokens on a cache, drafts of many
// heads.  Rows in 4 bits become bf16 on their way into LDS.
//
// What bounds it is the matrix cores (4 D operations per query and row against 4 D bytes per row of the cache), so tiles of 64
// cache rows go through LDS, once for the 128 or 256 query rows of a workgroup.  A wavefront takes 32 query rows, and a tile in
// two halves of 32 cache rows:
//   S[t, q] = K Q^T on v_mfma_f32_32x32x16_bf16: a lane holds one query column and 16 of 32 rows, so that the softmax of a
//             column is the lane's and its partner's (half a wavefront away) alone;
//   O^T[d, q] += V^T P: P is in operand order as it leaves the softmax, rounded to one bf16 number (its error, at most 2^-8 of
//             each weight and of any sign, disappears in the sum beside the rounding of the output), and V^T comes from LDS by
//             transposing reads.
// A half's exponentials are issued beside the next half's products with Q, whose K operands were read a half before: the
// transcendental unit (16 cycles per instruction), the other vector work and the matrix cores are each busy for about 256, 260
// and 512 cycles of a half.  There is no maximum per half: terms are formed against the reference at hand, and only a sum that
// is too large (or not a number) has the largest logit looked for.  One barrier per tile: while tile j is worked on, K of tile
// j + 2 and V of tile j + 1 travel through registers into the buffers of LDS that nobody reads.  Pieces of 16 bytes are
// swizzled within a row of LDS so that neither kind of read meets a bank twice (no conflicts counted).
// Measured on a prompt of 8192 tokens, 32 heads of 128 channels, causal (0.55 TFLOP): 530 to 600 us on different cards, 0.92 to
// 1.04 PFLOP/s where a large matrix product reaches 1.29; matrix cores busy for 0.48 of the cycles.  Without memory, LDS and
// barrier it would take 409.  Slower: the products and their exponentials one after the other with all operands read ahead
// (576), loads straight into LDS (545; the transposing reads then wait for all of them, or have to be assembly), 64 query rows
// per wavefront at one wavefront per SIMD (1016), and a maximum per half with two products in a chain of their own (571).
#include <type_traits>

#include "kvs_window.h"

namespace kvs {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kTile = kWideTile;
// A lane's sixteen terms may add up to this before their reference is raised to the largest logit: sixteen logits that are equal,
// of slots with up to 4096 copies (512 tokens of 32 heads on 32 caches of 2560 slots, 1 to 200 copies, logits close together: 93 us,
// with 1024 130).
constexpr float kMostSum = 65536.f;

// Where piece `p` (16 bytes) of row r is within its row.
template <int D> __device__ __forceinline__ int key_slot(int r, int p) { return D == 128 ? p ^ (r % 16) : p ^ (r / 2 % 8); }
template <int D> __device__ __forceinline__ int value_slot(int r, int p) {
  return D == 128 ? p ^ (r % 4 * 4) : p ^ (r / 2 % 2 * 4);
}

// A 16-byte piece of bf16 values without those that are not finite; sets `odd` if there were any.
__device__ __forceinline__ u32x4 finite_only(u32x4 x, bool& odd) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool lo = (x[i] & 0x7f80u) == 0x7f80u, hi = (x[i] & 0x7f800000u) == 0x7f800000u;
    odd |= lo | hi;
    x[i] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
  }
  return x;
}

__device__ __forceinline__ float of_both_halves_max(float x) { return fmaxf(x, __shfl_xor(x, 32, kWave)); }

// A thread's pieces of a tile of K or V on their way from memory: piece `p` (eight channels) of every (THREADS * 8 / D)-th row,
// from row `srow` of the tile on.  Rows past the range's end, row `last` of the tile, repeat it.
template <CacheKind KIND, int D, int THREADS>
struct Staged {
  static constexpr int kStep = THREADS * 8 / D, kPer = kTile / kStep;
  u32x4 r[kPer];
  __device__ __forceinline__ void request(const void* rows, const uint8_t*, long long first, int last, int srow, int p) {
    const char* base = (const char*)rows + (size_t)first * (2 * D);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const uint32_t row = last >= kTile - 1 ? srow + i * kStep : min(srow + i * kStep, last);
      r[i] = *(const u32x4*)(base + (uint32_t)(row * (2 * D) + 16 * p));
    }
  }
  __device__ __forceinline__ u32x4 piece(int i) const { return r[i]; }
};
template <int D, int THREADS>
struct Staged<CacheKind::kPackedBf16, D, THREADS> {
  static constexpr int kStep = THREADS * 8 / D, kPer = kTile / kStep;
  uint32_t r[kPer];
  uint8_t s[kPer];
  __device__ __forceinline__ void request(const void* rows, const uint8_t* scales, long long first, int last, int srow, int p) {
    const char* base = (const char*)rows + (size_t)first * (D / 2);
    const uint8_t* sbase = scales + (size_t)first * (D / 32);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const uint32_t row = last >= kTile - 1 ? srow + i * kStep : min(srow + i * kStep, last);
      r[i] = *(const uint32_t*)(base + (uint32_t)(row * (D / 2) + 4 * p));
      s[i] = sbase[row * (D / 32) + p / 4];
    }
  }
  __device__ __forceinline__ u32x4 piece(int i) const {
    const float sc = fp4::scale_of(s[i]);
    return u32x4{fp4::two_of<0>(r[i], sc), fp4::two_of<1>(r[i], sc), fp4::two_of<2>(r[i], sc), fp4::two_of<3>(r[i], sc)};
  }
};

// Wavefronts per SIMD that the registers are allotted for, i.e. workgroups of four wavefronts that share a compute unit.  64 channels:
// three, with cardinalities two (a prompt of 8192 tokens 324 us with three, 352 with two, 359 with one workgroup of eight
// wavefronts).  128 channels: two where the pieces on their way are rows in 4 bits (8 caches of 131072 rows, 64 query rows:
// 86 us, one workgroup 126); those of plain rows would have to be spilled (64 of 8224: 84 us, one workgroup 77).
template <CacheKind KIND, int D, int WAVES, bool COUNTS>
constexpr int waves_per_simd() {
  return WAVES == 8 ? 2 : D == 64 ? (COUNTS ? 2 : 3) : KIND == CacheKind::kPackedBf16 ? 2 : 1;
}

template <CacheKind KIND, int D, int WAVES, bool COUNTS, typename Tab>
__global__ __launch_bounds__(WAVES * kWave, (waves_per_simd<KIND, D, WAVES, COUNTS>())) void window_tiles_kernel(
    const Tab tab, const WindowShape sh, const Cache cache, int width, const uint16_t* __restrict__ Q,
    uint16_t* __restrict__ out, float* __restrict__ part) {
  constexpr int kThreads = WAVES * kWave;
  constexpr int KS = D / 16;                // steps of the contraction over channels
  constexpr int DB = D / 32;                // blocks of 32 channels
  constexpr int PPR = D / 8;                // pieces per row
  constexpr int PER = kTile * PPR / kThreads;    // pieces per thread of a tile of K, and of V
  __shared__ u32x4 sm_k[2][kTile * PPR], sm_v[2][kTile * PPR];
  // cardinalities as pairs hi + lo of bf16 numbers (exact up to 65536, to 2^-16 beyond): of four rows both hi pairs, then both lo
  __shared__ u32x4 sm_cnt[2][kTile / 4];

  // Workgroups on the same rows are `width` apart, which puts them on one XCD where it is a multiple of eight (as it is of listed
  // units), and the last blocks, which see most under a causal mask, come first.  Pieces of one unit are spread over the XCDs (512
  // tokens on 31 caches of 100 rows and one of 131072: 194 us, with all of a unit's on one 3812).
  const int id = blockIdx.x;
  int at_unit = id % width, piece = 0, block = id / width;
  if constexpr (Tab::kListed) {
    if (at_unit >= tab.pieces) return;
    if (sh.n_parts > 1) {
      piece = at_unit + tab.before;
      at_unit = tab.unit_of(at_unit);
      piece -= tab.entry(at_unit).before;
    }
  } else {
    piece = block % sh.n_parts;
    block /= sh.n_parts;
  }
  block = sh.n_blocks - 1 - block;
  const CacheUnit un = tab.unit(sh, at_unit);
  const Reach re = reach_of<kTile>(sh, un.len, block);
  const int n_parts = parts_of(re.tiles, sh.part_tiles);
  if (piece >= n_parts) return;             // (a block whose reach is shorter than others of the unit)
  const int j0 = piece * sh.part_tiles, j1 = min(re.tiles, j0 + sh.part_tiles);
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
  const int col = lane % 32, half = lane / 32;
  const int row = block * sh.block + wave * 32 + col;          // the lane's query row
  const int pos = sh.causal ? un.len - sh.W + min(row, sh.R - 1) / sh.G : un.len - 1;
  const int pos_min = __builtin_amdgcn_readfirstlane(pos), pos_max = __builtin_amdgcn_readlane(pos, 31);

  f32x16 acc[DB];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int d = 0; d < DB; ++d) acc[d] = f32x16{};
  bool odd = false;                         // a value that is not finite was left out

  auto start_of = [&](int t) { return t < re.sink_tiles ? t * kTile : re.first + (t - re.sink_tiles) * kTile; };
  auto end_of = [&](int t) { return t < re.sink_tiles ? re.sink_end : re.end; };
  // every row of the tile is seen by all queries between positions a and b
  auto seen_whole = [&](int t0, int end, int a, int b) {
    return t0 + kTile <= end && t0 + kTile - 1 <= a && (sh.span == 0 || t0 > b - sh.span || t0 + kTile <= sh.sinks);
  };

  if (j0 < j1) {
    bf16x8 q[KS];
    const uint16_t* src = Q + query_row(sh, un.index, min(row, sh.R - 1)) * D + 8 * half;
#pragma unroll
    for (int k = 0; k < KS; ++k) q[k] = *(const bf16x8*)(src + 16 * k);
    // A tile travels through registers: requested when a tile is begun, written to LDS when that one is nearly done.
    const int srow = tid / PPR, spiece = tid % PPR;
    Staged<KIND, D, kThreads> rk, rv;
    float rc = 1.f;
    auto request = [&](auto& r, const void* rows, const uint8_t* scales, int t) __attribute__((always_inline)) {
      const int t0 = start_of(t);
      r.request(rows, scales, un.in_row + t0, end_of(t) - 1 - t0, srow, spiece);
    };
    auto request_keys = [&](int t) __attribute__((always_inline)) { request(rk, cache.k, cache.ks, t); };
    auto request_values = [&](int t) __attribute__((always_inline)) {
      request(rv, cache.v, cache.vs, t);
      if (COUNTS && tid < kTile) rc = (float)cache.counts[un.in_row + start_of(t) + min(tid, end_of(t) - 1 - start_of(t))];
    };
    auto store_keys = [&](int b) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int row = srow + i * (kThreads / PPR);
        sm_k[b][row * PPR + key_slot<D>(row, spiece)] = rk.piece(i);
      }
    };
    auto store_values = [&](int t, int b) __attribute__((always_inline)) {
      u32x4 x[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) x[i] = rv.piece(i);
      if (!seen_whole(start_of(t), end_of(t), re.pos_min, re.pos_max)) {
#pragma unroll
        for (int i = 0; i < PER; ++i) x[i] = finite_only(x[i], odd);
      }
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int row = srow + i * (kThreads / PPR);
        sm_v[b][row * PPR + value_slot<D>(row, spiece)] = x[i];
      }
      if (COUNTS && tid < kTile) {
        const uint32_t hi = cvt_pk_bf16(rc, 0.f);
        uint16_t* at = (uint16_t*)&sm_cnt[b][tid / 4] + tid % 4;
        at[0] = (uint16_t)hi;
        at[4] = (uint16_t)cvt_pk_bf16(rc - bf16_lo(hi), 0.f);
      }
    };
    // K operands of half a of the tile in buffer b, and V^T operands of its rows 16 st ..: element i of the one of channels
    // 32 d .. is row 16 st + 8 (i / 4) + 4 half + i % 4
    bf16x8 kf[KS];
    auto read_keys = [&](int b, int a) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < KS; ++k)
        kf[k] = __builtin_bit_cast(bf16x8, sm_k[b][(32 * a + col) * PPR + key_slot<D>(col, 2 * k + half)]);
    };
    const int vrow = 4 * half + lane % 16 / 4, vpiece = 2 * (lane / 16 % 2) + lane % 4 / 2;
    auto value_operand = [&](int b, int st, int d) __attribute__((always_inline)) {
      s16x4 x[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const short* at = (const short*)&sm_v[b][(16 * st + 8 * h + vrow) * PPR + value_slot<D>(vrow, 4 * d + vpiece)];
        x[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + lane % 2 * 4));
      }
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto products_with_keys = [&](f32x16& to) __attribute__((always_inline)) {
      to = f32x16{};
#pragma unroll
      for (int k = 0; k < KS; ++k) to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k], q[k], to, 0, 0, 0);
    };

    // Half A of tile j (buffer B), whose logits are in s.  On the way: the products of the K operands that are in kf, the next
    // half's, to s2, and the operands of the half after that.
    auto step = [&](auto half_c, auto buffer_c, int j, f32x16& s, f32x16& s2) __attribute__((always_inline)) {
      constexpr int A = decltype(half_c)::value, B = decltype(buffer_c)::value;
      const int t0 = start_of(j), end = end_of(j);
      if (!seen_whole(t0, end, pos_min, pos_max)) {
        // row 32 A + x of the tile for x = 8 (v / 4) + v % 4 plus this: limits that x is compared with
        const int base = t0 + 32 * A + 4 * half;
        const int before_end = end - base, before_sinks = sh.sinks - base;
        const int last = min(pos - base, before_end - 1);
        const int hidden = sh.span > 0 ? pos - sh.span - base : -1 - base;       // rows up to here are seen as sinks only
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int x = 8 * (v / 4) + v % 4;
          const bool seen = (x <= last) & ((x > hidden) | (x < before_sinks));
          s[v] = seen ? s[v] : -INFINITY;
        }
      }
      bf16x8 vf[DB];
#pragma unroll
      for (int d = 0; d < DB; ++d) vf[d] = value_operand(B, 2 * A, d);
      products_with_keys(s2);
      uint32_t p[8];
      float sum;
      auto terms = [&](float ref) __attribute__((always_inline)) {
        float x[16];
#pragma unroll
        for (int v = 0; v < 16; ++v) x[v] = __builtin_amdgcn_exp2f(fmaf(s[v], sh.scale_log2, -ref));
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = cvt_pk_bf16(x[2 * i], x[2 * i + 1]);
        // (of the terms as they enter the product with V)
        sum = 0.f;
        auto add = [&](uint32_t x, uint32_t y) {
          sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x), __builtin_bit_cast(bf16x2, y), sum, false);
        };
#pragma unroll
        for (int v4 = 0; v4 < 4; ++v4) {
          if (COUNTS) {                                      // c copies of the slot in the denominator
            const u32x4 c4 = sm_cnt[B][8 * A + 2 * v4 + half];
            add(p[2 * v4], c4[0]);
            add(p[2 * v4 + 1], c4[1]);
            add(p[2 * v4], c4[2]);
            add(p[2 * v4 + 1], c4[3]);
          } else {
            add(p[2 * v4], 0x3f803f80u);                     // (ones)
            add(p[2 * v4 + 1], 0x3f803f80u);
          }
        }
      };
      terms(m);
      if (__ballot(!(sum <= kMostSum)) != 0) {
        // The reference is below the logits by too much (or there is none yet): rare after the first tiles.
        float top = s[0];
#pragma unroll
        for (int v = 1; v < 16; ++v) top = fmaxf(top, s[v]);
        top = fmaxf(of_both_halves_max(top) * sh.scale_log2, m);
        const float corr = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top);
        l *= corr;
#pragma unroll
        for (int d = 0; d < DB; ++d) {
#pragma unroll
          for (int v = 0; v < 16; ++v) acc[d][v] *= corr;
        }
        m = top;
        terms(m == -INFINITY ? 0.f : m);                     // (a query that has seen nothing yet)
      }
      l += sum;
      if (A == 0) read_keys(B ^ 1, 0);
      else if (j + 1 < j1) read_keys(B ^ 1, 1);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32x4 w = {p[4 * h], p[4 * h + 1], p[4 * h + 2], p[4 * h + 3]};
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[d], __builtin_bit_cast(bf16x8, w), acc[d], 0, 0, 0);
          if (h == 0) vf[d] = value_operand(B, 2 * A + 1, d);
        }
      }
    };

    request_keys(j0);
    request_values(j0);
    store_keys(0);
    if (j0 + 1 < j1) request_keys(j0 + 1);
    store_values(j0, 0);
    if (j0 + 1 < j1) store_keys(1);
    __syncthreads();
    f32x16 s0, s1;
    read_keys(0, 0);
    products_with_keys(s0);
    read_keys(0, 1);

    // Tile j: the logits of its first half are in s0 and the K operands of its second in kf, and those of the next tile
    // afterwards (behind the last tile they are of whatever the buffer holds, and nobody looks at them).
    auto tile = [&](int j, auto buffer_c) __attribute__((always_inline)) {
      constexpr int B = decltype(buffer_c)::value;
      if (j + 1 < j1) request_values(j + 1);
      if (j + 2 < j1) request_keys(j + 2);
      step(std::integral_constant<int, 0>{}, buffer_c, j, s0, s1);
      step(std::integral_constant<int, 1>{}, buffer_c, j, s1, s0);
      if (j + 1 < j1) {
        store_values(j + 1, B ^ 1);
        if (j + 2 < j1) store_keys(B);
        __syncthreads();
      }
    };
    for (int j = j0;;) {
      tile(j, std::integral_constant<int, 0>{});
      if (++j == j1) break;
      tile(j, std::integral_constant<int, 1>{});
      if (++j == j1) break;
    }
  }

  if (__syncthreads_or(odd)) {
    // What is not finite makes the sums of the queries that see it what it is itself, whatever its weight.
    for (int j = j0; j < j1; ++j) {
      const int t0 = start_of(j), end = end_of(j);
      if (seen_whole(t0, end, re.pos_min, re.pos_max)) continue;
#pragma unroll 1
      for (int t = t0; t < min(t0 + kTile, end); ++t) {
#pragma unroll
        for (int d = 0; d < DB; ++d) {
#pragma unroll
          for (int v4 = 0; v4 < 4; ++v4) {
            const f32x4_t y = four_values<KIND, D>(cache, un.in_row + t, 32 * d + 8 * v4 + 4 * half);
            const bool seen = sees(sh, pos, t);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[d][4 * v4 + e] += seen && !__builtin_isfinite(y[e]) ? y[e] : 0.f;
          }
        }
      }
    }
  }

  // element v of block d: channel 32 d + 8 (v / 4) + 4 half + v % 4 of the lane's query
  const float den = l + __shfl_xor(l, 32, kWave);
  if (row >= sh.R) return;
  if (n_parts == 1) {
    uint16_t* dst = out + query_row(sh, un.index, row) * D + 4 * half;
    const float inv = quotient(1.f, den);
#pragma unroll
    for (int d = 0; d < DB; ++d) {
#pragma unroll
      for (int v4 = 0; v4 < 4; ++v4) {
        *(uint2*)(dst + 32 * d + 8 * v4) = make_uint2(cvt_pk_bf16(acc[d][4 * v4] * inv, acc[d][4 * v4 + 1] * inv),
                                                      cvt_pk_bf16(acc[d][4 * v4 + 2] * inv, acc[d][4 * v4 + 3] * inv));
      }
    }
  } else {
    float* dst = part + part_at(sh, un, row, piece);
#pragma unroll
    for (int d = 0; d < DB; ++d) {
#pragma unroll
      for (int v4 = 0; v4 < 4; ++v4) {
        *(float2*)(dst + 32 * d + 8 * v4 + 4 * half) = make_float2(acc[d][4 * v4], acc[d][4 * v4 + 1]);
        *(float2*)(dst + 32 * d + 8 * v4 + 4 * half + 2) = make_float2(acc[d][4 * v4 + 2], acc[d][4 * v4 + 3]);
      }
    }
    if (half == 0) *(float2*)(dst + D) = make_float2(m, den);
  }
}

template <CacheKind KIND, int D, int WAVES, typename Tab>
hipError_t launch_waves(const Tab& tab, const WindowShape& sh, const Cache& cache, const void* Q, void* out, float* part,
                        hipStream_t stream) {
  const long long pieces = pieces_of(tab, sh);
  const int width = Tab::kListed ? (int)((pieces + 7) / 8 * 8) : tab.n;
  const dim3 grid((unsigned)((Tab::kListed ? width : pieces) * sh.n_blocks));
  if (cache.counts) {
    hipLaunchKernelGGL((window_tiles_kernel<KIND, D, WAVES, true, Tab>), grid, dim3(WAVES * kWave), 0, stream, tab, sh, cache, width,
                       (const uint16_t*)Q, (uint16_t*)out, part);
  } else {
    hipLaunchKernelGGL((window_tiles_kernel<KIND, D, WAVES, false, Tab>), grid, dim3(WAVES * kWave), 0, stream, tab, sh, cache, width,
                       (const uint16_t*)Q, (uint16_t*)out, part);
  }
  return hipGetLastError();
}

template <CacheKind KIND, typename Tab>
hipError_t launch_sized(const Tab& tab, const WindowShape& sh, const Cache& cache, const void* Q, void* out, float* part,
                        hipStream_t stream) {
  if (sh.D == 64) return launch_waves<KIND, 64, 4>(tab, sh, cache, Q, out, part, stream);
  return sh.block == 128 ? launch_waves<KIND, 128, 4>(tab, sh, cache, Q, out, part, stream)
                         : launch_waves<KIND, 128, 8>(tab, sh, cache, Q, out, part, stream);
}

}  // namespace

hipError_t launch_window_tiles(const EqualUnits* equal, const ListedUnits* listed, const WindowShape& sh, CacheKind kind,
                               const Cache& cache, const void* Q, void* out, float* part, hipStream_t stream) {
  auto go = [&](const auto& tab) {
    return kind == CacheKind::kBf16 ? launch_sized<CacheKind::kBf16>(tab, sh, cache, Q, out, part, stream)
                                    : launch_sized<CacheKind::kPackedBf16>(tab, sh, cache, Q, out, part, stream);
  };
  return equal ? go(*equal) : go(*listed);
}

}  // namespace kvs
