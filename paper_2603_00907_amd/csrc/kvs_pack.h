// Shared by the host layer and the kernels of kvs_pack and kvs_unpack.
#pragma once

#include <type_traits>

#include "kvs_device.h"

namespace kvs {

// A unit's rows: from row src of the source to row dst of the destination.
struct RowMove {
  long long src, dst;
  int len;
};
// Units of a launch: equal lengths at equal distances follow from the first, others are listed.
struct EqualMoves {
  RowMove first;
  long long src_step, dst_step;
  __device__ __forceinline__ RowMove unit(int i) const {
    return {first.src + i * src_step, first.dst + i * dst_step, first.len};
  }
};
constexpr int kListedMoves = 128;
struct ListedMoves {
  RowMove u[kListedMoves];
  __device__ __forceinline__ RowMove unit(int i) const { return u[i]; }
};
constexpr int kMostMoves = 65535;        // units of a launch (its grid's second dimension)

// Keys and Values in 4 bits: codes and scales.
struct PackedRange {
  uint8_t *kc, *ks, *vc, *vs;
};

// `equal` or, where it is null, `listed`; longest: rows of the launch's longest unit (at least one).
hipError_t launch_pack(const EqualMoves* equal, const ListedMoves* listed, int n_units, int longest, kvs_dtype dt, int D,
                       const void* K, const void* V, const PackedRange& to, hipStream_t stream);
hipError_t launch_unpack(const EqualMoves* equal, const ListedMoves* listed, int n_units, int longest, kvs_dtype dt, int D,
                         const PackedRange& from, void* K, void* V, hipStream_t stream);

}  // namespace kvs
