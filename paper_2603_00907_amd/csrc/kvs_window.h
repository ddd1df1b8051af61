// Shared by the host layer and the kernels of the masked attention over a cache (kvs_window_attention and its _packed form).
#pragma once

#include "kvs_fp4.h"

namespace kvs {

// The cache of a launch.  Plain: k and v are rows of D values.  4 bits: k and v are codes (D / 2 bytes a row), ks and vs the
// blocks' scales (D / 32 bytes a row).
struct Cache {
  const void* k;
  const void* v;
  const uint8_t* ks;
  const uint8_t* vs;
  const int32_t* counts;
};

constexpr int kMaxParts = 256;           // pieces that the rows of a unit are cut into at most
constexpr int kWindowTile = 32;          // cache rows per tile of the kernels in kvs_window_rows.hip
constexpr int kWideTile = 64;            // and of those in kvs_window_tiles.hip

struct WindowShape {
  int R, G, W, D;
  int causal;           // 0, or 1: query w is at position len - W + w (0: at len - 1)
  int span;             // rows up to the query's own that it sees, 0: all
  int sinks;            // first rows that it sees in any case (and that are not after it)
  float scale_log2;
  int block;            // query rows per workgroup
  int n_blocks;         // per unit
  int n_parts;          // pieces of the unit and block that has most of them
  int part_tiles;       // tiles per piece
  int large;            // kvs_window_rows.hip: workgroups of all the wavefronts that a compute unit holds, and no pieces
};

// Query rows are taken in the order (window position, head), so that a block of them has few positions and its rows of the
// cache lie together: row r is head r % G at window position r / G.  What a block sees are the rows [0, sink_end) and
// [first, end), in tiles that start at 0 and at `first`.
struct Reach {
  int pos_min, pos_max; // positions of the block's first and last query
  int sink_end, first, end;
  int sink_tiles, tiles;
};
template <int TILE>
__host__ __device__ inline Reach reach_of(const WindowShape& sh, int len, int block) {
  Reach r;
  const int r0 = block * sh.block;
  const int r1 = (r0 + sh.block < sh.R ? r0 + sh.block : sh.R) - 1;
  r.pos_min = sh.causal ? len - sh.W + r0 / sh.G : len - 1;
  r.pos_max = sh.causal ? len - sh.W + r1 / sh.G : len - 1;
  r.end = r.pos_max + 1 > 0 ? r.pos_max + 1 : 0;
  r.first = sh.span > 0 && r.pos_min - sh.span + 1 > 0 ? r.pos_min - sh.span + 1 : 0;
  if (r.first > r.end) r.first = r.end;
  r.sink_end = sh.sinks < r.first ? sh.sinks : r.first;
  r.sink_tiles = (r.sink_end + TILE - 1) / TILE;
  r.tiles = r.sink_tiles + (r.end - r.first + TILE - 1) / TILE;
  return r;
}
// Whether the query at position `pos` sees row t (0 <= t < the reach's end of t's range).
__device__ __forceinline__ bool sees(const WindowShape& sh, int pos, int t) {
  return t <= pos && (sh.span == 0 || t > pos - sh.span || t < sh.sinks);
}
// Pieces that a reach of `tiles` tiles is cut into (at least one: it writes the zeros of queries that see nothing).
__host__ __device__ inline int parts_of(int tiles, int part_tiles) {
  return tiles <= part_tiles ? 1 : (tiles + part_tiles - 1) / part_tiles;
}

// Most tiles that a block of query rows of a unit of this length reaches (an upper bound of Reach::tiles), and the pieces that
// the unit is given.
inline int most_tiles(const WindowShape& sh, int len, int tile) {
  auto tiles = [&](long long rows) { return (int)((rows + tile - 1) / tile); };
  auto less = [](long long a, long long b) { return a < b ? a : b; };
  if (sh.span == 0) return tiles(len);
  const long long positions = sh.causal ? less(sh.W, (sh.block - 1) / sh.G + 2) : 1;
  return tiles(less(len, sh.span + positions - 1)) + tiles(less(sh.sinks, len));
}
inline int unit_pieces(const WindowShape& sh, int len, int tile) { return parts_of(most_tiles(sh, len, tile), sh.part_tiles); }

// One unit of a launch: its rows of the cache.
struct CacheUnit {
  long long in_row;
  int len;
  int index;            // position in the caller's problem (indexes Q and out)
  int before;           // pieces of the problem's units before it (indexes partial results)
};

// The units of a launch.  Equal lengths at equal distances (the heads of a layer, or of all layers) follow from the first;
// up to kInlineUnits others travel in the kernel arguments, more of them through the workspace.  Two types, because a
// launch with a table in its arguments takes longer (see UnitTableT).
struct EqualUnits {
  static constexpr bool kListed = false;
  long long in_row, step;
  int len, first, n;
  __device__ __forceinline__ CacheUnit unit(const WindowShape& sh, int i) const {
    return {in_row + i * step, len, first + i, (first + i) * sh.n_parts};
  }
};
struct UnitEntry {
  long long in_row;
  int len, before;
};
struct ListedUnits {
  static constexpr bool kListed = true;
  const UnitEntry* ext;   // DEVICE, or null: u
  int first, n;           // position in the caller's problem of the first, and how many
  int before, pieces;     // pieces of the units before them, and theirs
  UnitEntry u[kInlineUnits];
  __device__ __forceinline__ UnitEntry entry(int i) const {
#if defined(__HIP_DEVICE_COMPILE__)
    if (ext != nullptr) return ((const __attribute__((address_space(4))) UnitEntry*)ext)[i];
#endif
    return u[i];
  }
  __device__ __forceinline__ CacheUnit unit(const WindowShape&, int i) const {
    const UnitEntry e = entry(i);
    return {e.in_row, e.len, first + i, e.before};
  }
  // The unit of piece f (0 <= f < pieces).  (A grid as wide for every unit as the longest needs spends 2 ns on each workgroup that
  // finds nothing to do: one token on 999 caches of 100 rows and one of 131072: 60 us, in such a grid 589.)
  __device__ __forceinline__ int unit_of(int f) const {
    return last_not_above(n, f + before, [&](int i) { return ext != nullptr ? ext[i].before : u[i].before; });
  }
};

// Pieces of all units of a launch.
inline long long pieces_of(const EqualUnits& tab, const WindowShape& sh) { return (long long)tab.n * sh.n_parts; }
inline long long pieces_of(const ListedUnits& tab, const WindowShape&) { return tab.pieces; }

// Partial results: [piece, all units'][query row in the order above] of D numerators, the maximum and the denominator.  Where a
// block's reach is one piece, its workgroup stores the output itself.
__device__ __forceinline__ size_t part_at(const WindowShape& sh, const CacheUnit& un, int row, int piece) {
  return ((size_t)(un.before + piece) * sh.R + row) * (size_t)(sh.D + 2);
}
// Where query row r of a unit is in Q and out, in rows of D.
__device__ __forceinline__ size_t query_row(const WindowShape& sh, int unit, int r) {
  return (size_t)unit * sh.R + (size_t)(r % sh.G) * sh.W + r / sh.G;
}

enum class CacheKind { kF32, kBf16, kPackedF32, kPackedBf16 };   // the cache, and the type of Q and out

// Four neighbouring values of a row from channel ch on (a multiple of four), wherever speed does not matter.
typedef float f32x4_t __attribute__((ext_vector_type(4)));
template <CacheKind KIND, int D>
__device__ __forceinline__ f32x4_t four_values(const Cache& cache, size_t row, int ch) {
  const size_t at = row * D + ch;
  if constexpr (KIND == CacheKind::kF32) {
    return *(const f32x4_t*)((const float*)cache.v + at);
  } else if constexpr (KIND == CacheKind::kBf16) {
    const uint2 x = *(const uint2*)((const uint16_t*)cache.v + at);
    return f32x4_t{bf16_lo(x.x), bf16_hi(x.x), bf16_lo(x.y), bf16_hi(x.y)};
  } else {
    const uint32_t x = *(const uint16_t*)((const uint8_t*)cache.v + at / 2);
    const float sc = fp4::scale_of(cache.vs[at / fp4::kBlock]);
    const uint32_t a = fp4::two_of<0>(x, sc), b = fp4::two_of<1>(x, sc);
    return f32x4_t{bf16_lo(a), bf16_hi(a), bf16_lo(b), bf16_hi(b)};
  }
}
// A numerator over its denominator; zero where no term was seen.
__device__ __forceinline__ float quotient(float num, float den) { return den == 0.f ? 0.f : num / den; }
// The running maximum of a softmax is raised only when a logit exceeds it by this many powers of two: terms of up to 2^8 are
// as exact as terms of up to 1.
constexpr float kSlack = 8.f;

// The launchers: `equal` or, where it is null, `listed`.
hipError_t launch_window_rows(const EqualUnits* equal, const ListedUnits* listed, const WindowShape& sh, CacheKind kind,
                              const Cache& cache, const void* Q, void* out, float* part, hipStream_t stream);
// bf16 outputs, blocks of 128 or 256 query rows (kvs_window_tiles.hip).
hipError_t launch_window_tiles(const EqualUnits* equal, const ListedUnits* listed, const WindowShape& sh, CacheKind kind,
                               const Cache& cache, const void* Q, void* out, float* part, hipStream_t stream);
// out from the partial results of the units at, .., at + n - 1 of a launch of kernels whose tiles have `tile` rows (kWindowTile or
// kWideTile).
hipError_t launch_window_reduce(const EqualUnits* equal, const ListedUnits* listed, int at, int n, const WindowShape& sh, bool f32,
                                int tile, const float* part, void* out, hipStream_t stream);
// Descriptors of all units into the workspace.
hipError_t launch_window_table(const kvs_problem* p, const WindowShape& sh, int tile, UnitEntry* dst, hipStream_t stream);

}  // namespace kvs
