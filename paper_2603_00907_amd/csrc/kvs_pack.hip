// A unit's cache rows into rows in 4 bits (kvs_fp4.h) and back.
//
// Both are copies: memory bounds them, 2 D bytes (bf16) against D / 2 + D / 32 for each of K and V.  A thread takes eight
// neighbouring values of a row of K and the same of V, so that the lanes of a wavefront cover whole rows; the four threads
// of a block of 32 exchange the largest magnitude by lane moves.  One row per thread: the wavefronts of many short workgroups
// have as much on its way as memory takes, and several rows per thread are slower (256 caches of 4096 bf16 rows of 128 channels,
// 679 MB: packing 116 us, 5.8 TB/s, 120 with two rows and 124 with four; unpacking 120; 100 fp32 caches of unequal lengths up to
// 9000 rows of 64 channels 65 and 68 us).
#include "kvs_fp4.h"
#include "kvs_pack.h"

namespace kvs {
namespace {

constexpr int kThreads = 256;
constexpr int kEach = kPackValues / kThreads;      // values per thread and row

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

// The thread's unit and row.
template <int D, typename Tab>
__device__ __forceinline__ int place(const Tab& tab, RowMove& mv) {
  int group = blockIdx.x;
  if constexpr (Tab::kListed) {
    const int i = tab.unit_of(group);
    mv = tab.unit(i);
    group -= tab.before[i];
  } else {
    mv = tab.unit(blockIdx.y);
  }
  return group * (kPackValues / D) + (int)threadIdx.x * kEach / D;
}

template <typename T, int D, typename Tab>
__global__ __launch_bounds__(kThreads) void pack_kernel(const Tab tab, const T* __restrict__ K, const T* __restrict__ V,
                                                        uint8_t* __restrict__ kc, uint8_t* __restrict__ ks,
                                                        uint8_t* __restrict__ vc, uint8_t* __restrict__ vs) {
  RowMove mv;
  const int row = place<D>(tab, mv);
  const int ch = (int)threadIdx.x * kEach % D;
  if (row >= mv.len) return;               // (a row's threads go together)
  const size_t from = ((size_t)mv.src + row) * D + ch, to = ((size_t)mv.dst + row) * D + ch;
  Eight<T> k, v;
  k.load(K + from);
  v.load(V + from);
  float x[8], y[8];
  k.unpack(x);
  v.unpack(y);
  uint32_t sx, sy;
  const uint32_t cx = encode(x, sx), cy = encode(y, sy);
  *(uint32_t*)(kc + to / 2) = cx;
  *(uint32_t*)(vc + to / 2) = cy;
  if (ch % fp4::kBlock == 0) {
    ks[to / fp4::kBlock] = (uint8_t)sx;
    vs[to / fp4::kBlock] = (uint8_t)sy;
  }
}

template <typename T, int D, typename Tab>
__global__ __launch_bounds__(kThreads) void unpack_kernel(const Tab tab, const uint8_t* __restrict__ kc,
                                                          const uint8_t* __restrict__ ks, const uint8_t* __restrict__ vc,
                                                          const uint8_t* __restrict__ vs, T* __restrict__ K,
                                                          T* __restrict__ V) {
  RowMove mv;
  const int row = place<D>(tab, mv);
  const int ch = (int)threadIdx.x * kEach % D;
  if (row >= mv.len) return;
  const size_t from = ((size_t)mv.src + row) * D + ch, to = ((size_t)mv.dst + row) * D + ch;
  const uint32_t c[2] = {*(const uint32_t*)(kc + from / 2), *(const uint32_t*)(vc + from / 2)};
  const uint8_t s[2] = {ks[from / fp4::kBlock], vs[from / fp4::kBlock]};
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const float scale = fp4::scale_of(s[x]);
    const uint32_t w[4] = {fp4::two_of<0>(c[x], scale), fp4::two_of<1>(c[x], scale), fp4::two_of<2>(c[x], scale),
                           fp4::two_of<3>(c[x], scale)};
    Eight<T>::store((x == 0 ? K : V) + to, w);
  }
}

// f(table, type, dimension, grid): a launch with the table, element type and head dimension at hand.
template <typename F>
hipError_t with_types(const EqualMoves* equal, const ListedMoves* listed, kvs_dtype dt, int D, F&& f) {
  auto typed = [&](const auto& tab, dim3 grid) {
    if (dt == KVS_F32) {
      if (D == 64) f(tab, (float*)nullptr, std::integral_constant<int, 64>{}, grid);
      else f(tab, (float*)nullptr, std::integral_constant<int, 128>{}, grid);
    } else {
      if (D == 64) f(tab, (uint16_t*)nullptr, std::integral_constant<int, 64>{}, grid);
      else f(tab, (uint16_t*)nullptr, std::integral_constant<int, 128>{}, grid);
    }
  };
  const int per = kPackValues / D;
  if (equal) typed(*equal, dim3((equal->first.len + per - 1) / per, equal->n));
  else typed(*listed, dim3(listed->groups));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_pack(const EqualMoves* equal, const ListedMoves* listed, kvs_dtype dt, int D, const void* K, const void* V,
                       const PackedRange& to, hipStream_t stream) {
  return with_types(equal, listed, dt, D, [&](const auto& tab, auto* t, auto d, dim3 grid) {
    typedef std::remove_pointer_t<decltype(t)> T;
    hipLaunchKernelGGL((pack_kernel<T, decltype(d)::value, std::decay_t<decltype(tab)>>), grid, dim3(kThreads), 0, stream, tab,
                       (const T*)K, (const T*)V, to.kc, to.ks, to.vc, to.vs);
  });
}

hipError_t launch_unpack(const EqualMoves* equal, const ListedMoves* listed, kvs_dtype dt, int D, const PackedRange& from, void* K,
                         void* V, hipStream_t stream) {
  return with_types(equal, listed, dt, D, [&](const auto& tab, auto* t, auto d, dim3 grid) {
    typedef std::remove_pointer_t<decltype(t)> T;
    hipLaunchKernelGGL((unpack_kernel<T, decltype(d)::value, std::decay_t<decltype(tab)>>), grid, dim3(kThreads), 0, stream, tab,
                       from.kc, from.ks, from.vc, from.vs, (T*)K, (T*)V);
  });
}

}  // namespace kvs
