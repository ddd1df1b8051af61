// A unit's cache rows into rows in 4 bits (kvs_fp4.h) and back.
//
// Both are copies: memory bounds them, 2 D bytes (bf16) against D / 2 + D / 32 for each of K and V.  A thread takes eight
// neighbouring values of a row of K and the same of V, so that the lanes of a wavefront cover whole rows; the four threads
// of a block of 32 exchange the largest magnitude by lane moves.
#include "kvs_fp4.h"
#include "kvs_pack.h"

namespace kvs {
namespace {

constexpr int kThreads = 256;
constexpr int kEach = 8;                 // values per thread and row
constexpr int kSteps = 4;                // rows per thread, all loads issued before the first use
template <int D> constexpr int rows_per_step() { return kThreads * kEach / D; }
template <int D> constexpr int rows_per_group() { return rows_per_step<D>() * kSteps; }

template <typename T> struct Eight;
template <> struct Eight<uint16_t> {
  uint4 r;
  __device__ __forceinline__ void load(const uint16_t* p) { r = *(const uint4*)p; }
  __device__ __forceinline__ void unpack(float (&x)[8]) const { Piece<uint16_t>::unpack(r, x); }
  static __device__ __forceinline__ void store(uint16_t* p, const uint32_t (&pairs)[4]) {
    *(uint4*)p = make_uint4(pairs[0], pairs[1], pairs[2], pairs[3]);
  }
};
template <> struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = ((const float4*)p)[0]; b = ((const float4*)p)[1]; }
  __device__ __forceinline__ void unpack(float (&x)[8]) const {
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
  static __device__ __forceinline__ void store(float* p, const uint32_t (&w)[4]) {
    ((float4*)p)[0] = make_float4(bf16_lo(w[0]), bf16_hi(w[0]), bf16_lo(w[1]), bf16_hi(w[1]));
    ((float4*)p)[1] = make_float4(bf16_lo(w[2]), bf16_hi(w[2]), bf16_lo(w[3]), bf16_hi(w[3]));
  }
};

__device__ __forceinline__ uint32_t max_of_quad(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true));   // quad_perm [1,0,3,2]
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true));   // quad_perm [2,3,0,1]
}

// The codes of eight values and, in every thread of the block's four, its scale byte.
__device__ __forceinline__ uint32_t encode(const float (&x)[8], uint32_t& scale) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  scale = fp4::scale_byte(max_of_quad(top));
  if (scale == fp4::kNanScale) return 0;
  const float s = __uint_as_float(scale << 23);
  uint32_t codes = 0;                    // (the conversion divides by its scale and rounds to the nearest code, ties to even)
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], s, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], s, 1);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], s, 2);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], s, 3);
  return codes;
}

template <typename T, int D, typename Tab>
__global__ __launch_bounds__(kThreads) void pack_kernel(const Tab tab, const T* __restrict__ K, const T* __restrict__ V,
                                                        uint8_t* __restrict__ kc, uint8_t* __restrict__ ks,
                                                        uint8_t* __restrict__ vc, uint8_t* __restrict__ vs) {
  const RowMove mv = tab.unit(blockIdx.y);
  const int r = (int)blockIdx.x * rows_per_group<D>() + (int)threadIdx.x * kEach / D;
  const int ch = (int)threadIdx.x * kEach % D;
  if ((int)blockIdx.x * rows_per_group<D>() >= mv.len) return;
  Eight<T> k[kSteps], v[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const size_t at = ((size_t)mv.src + min(r + i * rows_per_step<D>(), mv.len - 1)) * D + ch;
    k[i].load(K + at);
    v[i].load(V + at);
  }
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int row = r + i * rows_per_step<D>();
    float x[8], y[8];
    k[i].unpack(x);
    v[i].unpack(y);
    uint32_t sx, sy;
    const uint32_t cx = encode(x, sx), cy = encode(y, sy);
    if (row < mv.len) {
      const size_t at = ((size_t)mv.dst + row) * D + ch;
      *(uint32_t*)(kc + at / 2) = cx;
      *(uint32_t*)(vc + at / 2) = cy;
      if (ch % fp4::kBlock == 0) {
        ks[at / fp4::kBlock] = (uint8_t)sx;
        vs[at / fp4::kBlock] = (uint8_t)sy;
      }
    }
  }
}

template <typename T, int D, typename Tab>
__global__ __launch_bounds__(kThreads) void unpack_kernel(const Tab tab, const uint8_t* __restrict__ kc,
                                                          const uint8_t* __restrict__ ks, const uint8_t* __restrict__ vc,
                                                          const uint8_t* __restrict__ vs, T* __restrict__ K,
                                                          T* __restrict__ V) {
  const RowMove mv = tab.unit(blockIdx.y);
  const int r = (int)blockIdx.x * rows_per_group<D>() + (int)threadIdx.x * kEach / D;
  const int ch = (int)threadIdx.x * kEach % D;
  if ((int)blockIdx.x * rows_per_group<D>() >= mv.len) return;
  uint32_t c[2][kSteps];
  uint8_t s[2][kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const size_t at = ((size_t)mv.src + min(r + i * rows_per_step<D>(), mv.len - 1)) * D + ch;
    c[0][i] = *(const uint32_t*)(kc + at / 2);
    c[1][i] = *(const uint32_t*)(vc + at / 2);
    s[0][i] = ks[at / fp4::kBlock];
    s[1][i] = vs[at / fp4::kBlock];
  }
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int row = r + i * rows_per_step<D>();
    if (row >= mv.len) break;
    const size_t at = ((size_t)mv.dst + row) * D + ch;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const float scale = fp4::scale_of(s[x][i]);
      const uint32_t w[4] = {fp4::two_of<0>(c[x][i], scale), fp4::two_of<1>(c[x][i], scale),
                             fp4::two_of<2>(c[x][i], scale), fp4::two_of<3>(c[x][i], scale)};
      Eight<T>::store((x == 0 ? K : V) + at, w);
    }
  }
}

// f(table, type, dimension): a launch with the table, element type and head dimension at hand.
template <typename F>
hipError_t with_types(const EqualMoves* equal, const ListedMoves* listed, kvs_dtype dt, int D, F&& f) {
  auto typed = [&](const auto& tab) {
    if (dt == KVS_F32) {
      if (D == 64) f(tab, (float*)nullptr, std::integral_constant<int, 64>{});
      else f(tab, (float*)nullptr, std::integral_constant<int, 128>{});
    } else {
      if (D == 64) f(tab, (uint16_t*)nullptr, std::integral_constant<int, 64>{});
      else f(tab, (uint16_t*)nullptr, std::integral_constant<int, 128>{});
    }
  };
  if (equal) typed(*equal);
  else typed(*listed);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_pack(const EqualMoves* equal, const ListedMoves* listed, int n_units, int longest, kvs_dtype dt, int D,
                       const void* K, const void* V, const PackedRange& to, hipStream_t stream) {
  return with_types(equal, listed, dt, D, [&](const auto& tab, auto* t, auto d) {
    typedef std::remove_pointer_t<decltype(t)> T;
    constexpr int DIM = decltype(d)::value, per = rows_per_group<DIM>();
    hipLaunchKernelGGL((pack_kernel<T, DIM, std::decay_t<decltype(tab)>>), dim3((longest + per - 1) / per, n_units),
                       dim3(kThreads), 0, stream, tab, (const T*)K, (const T*)V, to.kc, to.ks, to.vc, to.vs);
  });
}

hipError_t launch_unpack(const EqualMoves* equal, const ListedMoves* listed, int n_units, int longest, kvs_dtype dt, int D,
                         const PackedRange& from, void* K, void* V, hipStream_t stream) {
  return with_types(equal, listed, dt, D, [&](const auto& tab, auto* t, auto d) {
    typedef std::remove_pointer_t<decltype(t)> T;
    constexpr int DIM = decltype(d)::value, per = rows_per_group<DIM>();
    hipLaunchKernelGGL((unpack_kernel<T, DIM, std::decay_t<decltype(tab)>>), dim3((longest + per - 1) / per, n_units),
                       dim3(kThreads), 0, stream, tab, from.kc, from.ks, from.vc, from.vs, (T*)K, (T*)V);
  });
}

}  // namespace kvs
