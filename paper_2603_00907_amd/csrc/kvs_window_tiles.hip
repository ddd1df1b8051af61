// The attention of kvs_window_rows.hip for blocks of many query rows, bf16: a prompt, or a chunk of new tokens on a cache.
//
// What bounds it is the matrix cores (4 D operations per query and row against 4 D bytes per row of the cache), so tiles of 64
// cache rows go through LDS, once for the 128 NB query rows of a workgroup, and every operand read feeds NB products.
// A wavefront takes 32 NB query rows:
//   S[t, q] = K Q^T on v_mfma_f32_32x32x16_bf16: a lane holds one query column and 16 of 32 rows, so that the softmax of a
//             column is the lane's and its partner's (half a wavefront away) alone;
//   O^T[d, q] += V^T P: P is in operand order as it leaves the softmax, rounded to one bf16 number (its error, at most 2^-9 of
//             each weight and of any sign, disappears in the sum beside the rounding of the output), and V^T comes from LDS by
//             transposing reads.
// The products of tile j + 1 with Q are issued beside the exponentials of tile j.  One barrier per tile: while tile j is worked
// on, K of tile j + 2 and V of tile j + 1 travel through registers into the halves of LDS that nobody reads.
// Pieces of 16 bytes are swizzled within a row of LDS so that neither kind of read meets a bank twice.
#include <type_traits>

#include "kvs_window.h"

namespace kvs {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kTile = kWideTile;

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

template <CacheKind KIND, int D, int NB, bool COUNTS, typename Tab>
__global__ __launch_bounds__(kThreads, NB == 1 ? 2 : 1) void window_tiles_kernel(
    const Tab tab, const WindowShape sh, const Cache cache, int n_units, const uint16_t* __restrict__ Q,
    uint16_t* __restrict__ out, float* __restrict__ part) {
  constexpr int KS = D / 16;                // steps of the contraction over channels
  constexpr int DB = D / 32;                // blocks of 32 channels
  constexpr int PPR = D / 8;                // pieces per row
  constexpr int PER = kTile * PPR / kThreads;    // pieces per thread of a tile of K, and of V
  __shared__ u32x4 sm_k[2][kTile * PPR];
  __shared__ u32x4 sm_v[2][kTile * PPR];
  __shared__ __attribute__((aligned(16))) float sm_cnt[2][kTile];

  // A unit's workgroups are n_units apart, which puts them on one XCD where n_units is a multiple of eight, and the last
  // blocks, which see most under a causal mask, come first.
  const int id = blockIdx.x;
  const int piece = id / n_units % sh.n_parts;
  const int block = sh.n_blocks - 1 - id / n_units / sh.n_parts;
  const CacheUnit un = tab.unit(id % n_units);
  const Reach re = reach_of<kTile>(sh, un.len, block);
  if (piece >= parts_of(re.tiles, sh.part_tiles)) return;     // the grid is as wide as the longest reach needs
  const int j0 = piece * sh.part_tiles, j1 = min(re.tiles, j0 + sh.part_tiles);
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
  const int col = lane % 32, half = lane / 32;
  const int row0 = block * sh.block + wave * 32 * NB;          // the wavefront's first query row

  int pos[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) pos[n] = sh.causal ? un.len - sh.W + min(row0 + 32 * n + col, sh.R - 1) / sh.G : un.len - 1;
  const int pos_min = __builtin_amdgcn_readfirstlane(pos[0]);
  const int pos_max = __builtin_amdgcn_readlane(pos[NB - 1], 31);

  f32x16 acc[NB][DB];
  float m[NB], l[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    m[n] = -INFINITY;
    l[n] = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[n][d] = f32x16{};
  }
  bool odd = false;                         // a value that is not finite was left out

  auto start_of = [&](int t) { return t < re.sink_tiles ? t * kTile : re.first + (t - re.sink_tiles) * kTile; };
  auto end_of = [&](int t) { return t < re.sink_tiles ? re.sink_end : re.end; };
  // every row of the tile is seen by all queries between positions a and b
  auto seen_whole = [&](int t0, int end, int a, int b) {
    return t0 + kTile <= end && t0 + kTile - 1 <= a && (sh.span == 0 || t0 > b - sh.span || t0 + kTile <= sh.sinks);
  };

  if (j0 < j1) {
    bf16x8 q[NB][KS];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const uint16_t* src = Q + query_row(sh, un.index, min(row0 + 32 * n + col, sh.R - 1)) * D + 8 * half;
#pragma unroll
      for (int k = 0; k < KS; ++k) q[n][k] = *(const bf16x8*)(src + 16 * k);
    }
    const char* kbase = (const char*)cache.k + (size_t)un.in_row * (2 * D);
    const char* vbase = (const char*)cache.v + (size_t)un.in_row * (2 * D);
    const int32_t* counts = COUNTS ? cache.counts + un.in_row : nullptr;
    const int srow = tid / PPR, spiece = tid % PPR;
    // (rows past the range's end repeat the last one)
    auto load = [&](const char* base, int t, u32x4 (&r)[PER]) {
      const int t0 = start_of(t), last = end_of(t) - 1;
#pragma unroll
      for (int i = 0; i < PER; ++i)
        r[i] = *(const u32x4*)(base + (uint32_t)(min(t0 + srow + i * (kThreads / PPR), last) * (2 * D) + 16 * spiece));
    };
    auto store_keys = [&](int b, const u32x4 (&r)[PER]) {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int row = srow + i * (kThreads / PPR);
        sm_k[b][row * PPR + key_slot<D>(row, spiece)] = r[i];
      }
    };
    auto store_values = [&](int b, int t, u32x4 (&r)[PER]) {
      if (!seen_whole(start_of(t), end_of(t), re.pos_min, re.pos_max)) {
#pragma unroll
        for (int i = 0; i < PER; ++i) r[i] = finite_only(r[i], odd);
      }
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int row = srow + i * (kThreads / PPR);
        sm_v[b][row * PPR + value_slot<D>(row, spiece)] = r[i];
      }
    };
    auto load_count = [&](int t) {
      return COUNTS && tid < kTile ? (float)counts[min(start_of(t) + tid, end_of(t) - 1)] : 1.f;
    };

    f32x16 s[NB][2];
    auto products_with_keys = [&](int b, f32x16 (&to)[NB][2]) {
#pragma unroll
      for (int n = 0; n < NB; ++n) to[n][0] = to[n][1] = f32x16{};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          const bf16x8 key = __builtin_bit_cast(bf16x8, sm_k[b][(32 * a + col) * PPR + key_slot<D>(col, 2 * k + half)]);
#pragma unroll
          for (int n = 0; n < NB; ++n) to[n][a] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key, q[n][k], to[n][a], 0, 0, 0);
        }
      }
    };

    // V^T operand of channels 32 d .. and of rows 16 st ..: element i is row 16 st + 8 (i / 4) + 4 half + i % 4
    const int vrow = 4 * half + lane % 16 / 4, vpiece = 2 * (lane / 16 % 2) + lane % 4 / 2;
    auto value_operand = [&](int b, int st, int d) {
      s16x8 x;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const short* at = (const short*)&sm_v[b][(16 * st + 8 * h + vrow) * PPR + value_slot<D>(vrow, 4 * d + vpiece)];
        const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + lane % 2 * 4));
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * h + i] = y[i];
      }
      return __builtin_bit_cast(bf16x8, x);
    };

    u32x4 rk[PER], rv[PER];
    {
      load(kbase, j0, rk);
      load(vbase, j0, rv);
      const float c = load_count(j0);
      store_keys(0, rk);
      if (j0 + 1 < j1) load(kbase, j0 + 1, rk);
      store_values(0, j0, rv);
      if (COUNTS && tid < kTile) sm_cnt[0][tid] = c;
      if (j0 + 1 < j1) store_keys(1, rk);
    }
    __syncthreads();
    products_with_keys(0, s);

    auto tile = [&](int j, auto last_c) {
      constexpr bool LAST = decltype(last_c)::value;
      const int b = (j - j0) & 1;
      float next_count = 1.f;
      if (!LAST) {
        load(vbase, j + 1, rv);
        next_count = load_count(j + 1);
        if (j + 2 < j1) load(kbase, j + 2, rk);
      }
      const int t0 = start_of(j), end = end_of(j);
      if (!seen_whole(t0, end, pos_min, pos_max)) {
#pragma unroll
        for (int n = 0; n < NB; ++n) {
#pragma unroll
          for (int a = 0; a < 2; ++a) {
#pragma unroll
            for (int v = 0; v < 16; ++v) {
              const int t = t0 + 32 * a + 8 * (v / 4) + 4 * half + v % 4;
              s[n][a][v] = t < end && sees(sh, pos[n], t) ? s[n][a][v] : -INFINITY;
            }
          }
        }
      }
      float ref[NB];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        float top = -INFINITY;
#pragma unroll
        for (int v = 0; v < 16; ++v) top = fmaxf(fmaxf(top, s[n][0][v]), s[n][1][v]);
        top *= sh.scale_log2;
        if (__ballot(top > m[n] + kSlack) != 0) {            // rare after the first tiles
          top = fmaxf(of_both_halves_max(top), m[n]);
          const float corr = m[n] == top ? 1.f : __builtin_amdgcn_exp2f(m[n] - top);
          l[n] *= corr;
#pragma unroll
          for (int d = 0; d < DB; ++d) {
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[n][d][v] *= corr;
          }
          m[n] = top;
        }
        ref[n] = m[n] == -INFINITY ? 0.f : m[n];             // (a query that has seen nothing yet)
      }
      // the next tile's products and this one's exponentials
      f32x16 s2[NB][2];
      if (!LAST) products_with_keys(b ^ 1, s2);
      bf16x8 p[NB][4];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        float sum = 0.f;
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          float x[16];
#pragma unroll
          for (int v = 0; v < 16; ++v) x[v] = __builtin_amdgcn_exp2f(fmaf(s[n][a][v], sh.scale_log2, -ref[n]));
#pragma unroll
          for (int v4 = 0; v4 < 4; ++v4) {
            if (COUNTS) {                                    // c copies of the slot in the denominator
              const float4 c4 = *(const float4*)&sm_cnt[b][32 * a + 8 * v4 + 4 * half];
              sum = fmaf(c4.x, x[4 * v4], sum);
              sum = fmaf(c4.y, x[4 * v4 + 1], sum);
              sum = fmaf(c4.z, x[4 * v4 + 2], sum);
              sum = fmaf(c4.w, x[4 * v4 + 3], sum);
            } else {
              sum += (x[4 * v4] + x[4 * v4 + 1]) + (x[4 * v4 + 2] + x[4 * v4 + 3]);
            }
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = cvt_pk_bf16(x[8 * h + 2 * i], x[8 * h + 2 * i + 1]);
            p[n][2 * a + h] = __builtin_bit_cast(bf16x8, w);
          }
        }
        l[n] += sum;
      }
#pragma unroll
      for (int st = 0; st < 4; ++st) {
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          const bf16x8 a = value_operand(b, st, d);
#pragma unroll
          for (int n = 0; n < NB; ++n) acc[n][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, p[n][st], acc[n][d], 0, 0, 0);
        }
      }
      if (!LAST) {
#pragma unroll
        for (int n = 0; n < NB; ++n) { s[n][0] = s2[n][0]; s[n][1] = s2[n][1]; }
        store_values(b ^ 1, j + 1, rv);
        if (COUNTS && tid < kTile) sm_cnt[b ^ 1][tid] = next_count;
        if (j + 2 < j1) store_keys(b, rk);
        __syncthreads();
      }
    };
    int j = j0;
    for (; j + 1 < j1; ++j) tile(j, std::false_type{});
    tile(j, std::true_type{});
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
#pragma unroll
            for (int n = 0; n < NB; ++n) {
              const bool seen = sees(sh, pos[n], t);
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[n][d][4 * v4 + e] += seen && !__builtin_isfinite(y[e]) ? y[e] : 0.f;
            }
          }
        }
      }
    }
  }

  // element v of block d: channel 32 d + 8 (v / 4) + 4 half + v % 4 of the lane's query
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const int row = row0 + 32 * n + col;
    const float den = l[n] + __shfl_xor(l[n], 32, kWave);
    if (row >= sh.R) continue;
    if (sh.n_parts == 1) {
      uint16_t* dst = out + query_row(sh, un.index, row) * D + 4 * half;
      const float inv = quotient(1.f, den);
#pragma unroll
      for (int d = 0; d < DB; ++d) {
#pragma unroll
        for (int v4 = 0; v4 < 4; ++v4) {
          *(uint2*)(dst + 32 * d + 8 * v4) = make_uint2(cvt_pk_bf16(acc[n][d][4 * v4] * inv, acc[n][d][4 * v4 + 1] * inv),
                                                        cvt_pk_bf16(acc[n][d][4 * v4 + 2] * inv, acc[n][d][4 * v4 + 3] * inv));
        }
      }
    } else {
      float* dst = part + part_at(sh, un.index, row, piece);
#pragma unroll
      for (int d = 0; d < DB; ++d) {
#pragma unroll
        for (int v4 = 0; v4 < 4; ++v4) {
          *(float2*)(dst + 32 * d + 8 * v4 + 4 * half) = make_float2(acc[n][d][4 * v4], acc[n][d][4 * v4 + 1]);
          *(float2*)(dst + 32 * d + 8 * v4 + 4 * half + 2) = make_float2(acc[n][d][4 * v4 + 2], acc[n][d][4 * v4 + 3]);
        }
      }
      if (half == 0) *(float2*)(dst + D) = make_float2(m[n], den);
    }
  }
}

template <CacheKind KIND, int D, int NB, typename Tab>
hipError_t launch_nb(const Tab& tab, int n_units, const WindowShape& sh, const Cache& cache, const void* Q, void* out,
                     float* part, hipStream_t stream) {
  const dim3 grid((unsigned)((long long)n_units * sh.n_blocks * sh.n_parts));
  if (cache.counts) {
    hipLaunchKernelGGL((window_tiles_kernel<KIND, D, NB, true, Tab>), grid, dim3(kThreads), 0, stream, tab, sh, cache, n_units,
                       (const uint16_t*)Q, (uint16_t*)out, part);
  } else {
    hipLaunchKernelGGL((window_tiles_kernel<KIND, D, NB, false, Tab>), grid, dim3(kThreads), 0, stream, tab, sh, cache, n_units,
                       (const uint16_t*)Q, (uint16_t*)out, part);
  }
  return hipGetLastError();
}

template <CacheKind KIND, typename Tab>
hipError_t launch_sized(const Tab& tab, int n_units, const WindowShape& sh, const Cache& cache, const void* Q, void* out,
                        float* part, hipStream_t stream) {
  if (sh.D == 64) {
    return sh.block == 128 ? launch_nb<KIND, 64, 1>(tab, n_units, sh, cache, Q, out, part, stream)
                           : launch_nb<KIND, 64, 2>(tab, n_units, sh, cache, Q, out, part, stream);
  }
  return sh.block == 128 ? launch_nb<KIND, 128, 1>(tab, n_units, sh, cache, Q, out, part, stream)
                         : launch_nb<KIND, 128, 2>(tab, n_units, sh, cache, Q, out, part, stream);
}

}  // namespace

hipError_t launch_window_tiles(const EqualUnits* equal, const ListedUnits* listed, int n_units, const WindowShape& sh,
                               CacheKind, const Cache& cache, const void* Q, void* out, float* part, hipStream_t stream) {
  const hipError_t e = equal ? launch_sized<CacheKind::kBf16>(*equal, n_units, sh, cache, Q, out, part, stream)
                             : launch_sized<CacheKind::kBf16>(*listed, n_units, sh, cache, Q, out, part, stream);
  if (e != hipSuccess || sh.n_parts == 1) return e;
  return launch_window_reduce(equal, listed, n_units, sh, false, kTile, part, out, stream);
}

}  // namespace kvs
