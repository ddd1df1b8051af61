// Shared by the host layer and the kernels of kvs_pack and kvs_unpack.
#pragma once

#include <type_traits>

#include "kvs_device.h"

namespace kvs {

constexpr int kPackValues = 2048;        // values of a workgroup, of K and of V

// A unit's rows: from row src of the source to row dst of the destination.
struct RowMove {
  long long src, dst;
  int len;
};
// Units of a launch: equal lengths at equal distances follow from the first, others are listed and have their workgroups one after
// the other.
struct EqualMoves {
  static constexpr bool kListed = false;
  RowMove first;
  long long src_step, dst_step;
  int n;
  __device__ __forceinline__ RowMove unit(int i) const {
    return {first.src + i * src_step, first.dst + i * dst_step, first.len};
  }
};
constexpr int kListedMoves = 2 * kWave;
struct ListedMoves {
  static constexpr bool kListed = true;
  RowMove u[kListedMoves];
  int before[kListedMoves];              // workgroups of the units before it, behind the last unit more than there are
  int n, groups;
  __device__ __forceinline__ RowMove unit(int i) const { return u[i]; }
  // The whole list is looked at in one load.  (A grid as wide for every unit as the longest needs: 99 caches of 100 bf16 rows and one
  // of 131072 187 us, so 20; 100 fp32 caches of unequal lengths up to 9000 rows, unpacked, 64 and 68.  Found in the descriptors by
  // two dependent loads the latter take 82.)
  __device__ __forceinline__ int unit_of(int group) const {
    const int2 two = *(const int2*)&before[threadIdx.x % kWave * 2];
    return __popcll(__ballot(two.x <= group)) + __popcll(__ballot(two.y <= group)) - 1;
  }
};
constexpr int kMostMoves = 65535;        // equal units of a launch (its grid's second dimension)
constexpr int kMostMoveGroups = 1 << 23; // workgroups that listed units are added up to

// Keys and Values in 4 bits: codes and scales.
struct PackedRange {
  uint8_t *kc, *ks, *vc, *vs;
};

// `equal` or, where it is null, `listed`; some unit has rows.
hipError_t launch_pack(const EqualMoves* equal, const ListedMoves* listed, kvs_dtype dt, int D, const void* K, const void* V,
                       const PackedRange& to, hipStream_t stream);
hipError_t launch_unpack(const EqualMoves* equal, const ListedMoves* listed, kvs_dtype dt, int D, const PackedRange& from, void* K,
                         void* V, hipStream_t stream);

}  // namespace kvs
