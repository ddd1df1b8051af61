// Host layer of the attention with a window and sinks (kvs_window_attention, plain and 4-bit caches) and of the conversions
// between the two kinds of cache (kvs_pack, kvs_unpack): argument checks, workspace, unit tables, launches.  Everything that
// can fail because of the arguments fails before the first launch.  Nothing here throws.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <memory>
#include <new>

#include "kvs_host.h"
#include "kvs_pack.h"
#include "kvs_window.h"

namespace kvs {
namespace {

constexpr long long kMostRow = 1ll << 48;      // rows that a cache may have: byte offsets stay far below 2^63
constexpr long long kComputeUnits = 256;
constexpr long long kMostGroups = 1ll << 22;   // workgroups of one launch, which have less than 2^32 threads together

// The fields that every one of these calls reads.
kvs_status check_common(const kvs_problem* p, int* elt) {
  if (p == nullptr || p->n_units < 1) return KVS_ERR_INVALID_ARG;
  if (p->head_dim != 64 && p->head_dim != 128) return KVS_ERR_INVALID_ARG;
  int io_dtype;                                // (a caller may have put any integer into the field)
  std::memcpy(&io_dtype, &p->io_dtype, sizeof(int));
  if (io_dtype != KVS_F32 && io_dtype != KVS_BF16) return KVS_ERR_DTYPE;
  if (p->len == nullptr || p->in_row == nullptr) return KVS_ERR_INVALID_ARG;
  for (int u = 0; u < p->n_units; ++u) {
    if (p->len[u] < 0 || p->len[u] > KVS_MAX_LEN || p->in_row[u] < 0 || p->in_row[u] > kMostRow) return KVS_ERR_INVALID_ARG;
  }
  *elt = io_dtype == KVS_F32 ? 4 : 2;
  return KVS_OK;
}

// Rows that the units' ranges reach to.
size_t rows_to(const kvs_problem* p, const int64_t* first) {
  long long rows = 0;
  for (int u = 0; u < p->n_units; ++u) {
    if (p->len[u] > 0) rows = std::max<long long>(rows, first[u] + p->len[u]);
  }
  return (size_t)rows;
}

kvs_status launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return KVS_OK;
  if (debug_switch(KVS_DEBUG_VERBOSE)) std::fprintf(stderr, "libkvs: %s failed: %s\n", what, hipGetErrorString(e));
  return KVS_ERR_DEVICE;
}

// ---- attention
struct WindowPlan {
  WindowShape sh{};
  bool wide = false;           // kvs_window_tiles.hip, else kvs_window_rows.hip
  bool equal = false;          // units of one length at equal distances
  size_t part_bytes = 0, table_bytes = 0;
  int tile() const { return wide ? kWideTile : kWindowTile; }
  size_t bytes() const { return part_bytes + table_bytes; }
};

// How the rows that a block of query rows sees are cut into pieces, of at most kMaxParts.
struct Cut {
  const kvs_problem* p;
  const WindowShape& sh;
  int tile;
  long long most = 1;                            // tiles of the longest reach
  bool equal = true;                             // reaches of one length
  Cut(const kvs_problem* problem, const WindowShape& shape, int rows) : p(problem), sh(shape), tile(rows) {
    for (int u = 0; u < p->n_units; ++u) {
      most = std::max<long long>(most, most_tiles(sh, p->len[u], tile));
      equal = equal && p->len[u] == p->len[0];
    }
  }
  struct Sums { long long groups, tiles, partial; };   // workgroups, their tiles, workgroups that store partial results
  // of a call whose pieces have `per` tiles at most
  Sums with(long long per) const {
    Sums s = {0, 0, 0};
    long long parts = 0, t = 0;
    const int units = equal ? 1 : p->n_units;
    for (int u = 0; u < units; ++u) {
      if (u == 0 || p->len[u] != p->len[u - 1]) {
        t = most_tiles(sh, p->len[u], tile);
        parts = std::max(1ll, (t + per - 1) / per);
      }
      s.groups += parts;
      s.tiles += t;
      s.partial += parts > 1 ? parts : 0;
    }
    const long long times = (equal ? p->n_units : 1ll) * sh.n_blocks;
    return {s.groups * times, s.tiles * times, s.partial * times};
  }
};

// kvs_window_rows.hip: the longest pieces that make no more workgroups than run at once, since memory bounds all of them alike and
// what one does for its piece, a partial result written and read again, is done as rarely as possible.
void cut_rows(const kvs_problem* p, long long at_once, WindowShape& sh) {
  const Cut cut(p, sh, kWindowTile);
  // A workgroup of all the wavefronts that a compute unit holds for a whole reach, which spares the partial results: where there
  // is one for most compute units (one token on 256 caches of 4096 slots in 4 bits 35.8 us, in three pieces each 41.2), and for
  // reaches that are a round or two of its tiles (8 caches of 300 rows 8.0 us, in pieces 9.2; of 777 rows 12.0 and 9.4).
  const long long whole = (long long)p->n_units * sh.n_blocks;
  if (whole <= kComputeUnits && (cut.most <= 12 || whole >= kComputeUnits * 3 / 4)) {
    sh.large = 1;
    sh.part_tiles = (int)cut.most;
    sh.n_parts = 1;
    return;
  }
  constexpr long long kLeastTiles = 4;           // a tile for each wavefront of a workgroup
  // (more units than that: whole reaches, or the longest of unequal ones cut)
  const long long limit = whole <= at_once ? at_once : cut.equal ? whole : whole + at_once;
  long long per = std::max(kLeastTiles, (cut.most + kMaxParts - 1) / kMaxParts);
  const Cut::Sums shortest = cut.with(per);
  if (shortest.groups > limit) {
    // (tiles / per <= workgroups < tiles / per + whole)
    long long fits = std::max(per, cut.most);
    if (limit > whole) fits = std::min(fits, shortest.tiles / (limit - whole) + 1);
    per = std::max(per, (shortest.tiles + limit - 1) / limit - 1);
    while (fits - per > 1) {
      const long long mid = (per + fits) / 2;
      if (cut.with(mid).groups > limit) per = mid;
      else fits = mid;
    }
    per = fits;
  }
  sh.part_tiles = (int)per;
  sh.n_parts = (int)((cut.most + per - 1) / per);
}

// kvs_window_tiles.hip, whose workgroups keep a compute unit busy by themselves and whose partial results are many: the number of
// pieces with the shortest time, counted in tiles.  A workgroup takes kOnce tiles' time besides its tiles, and pieces cost a
// launch that adds them up and their partials' way to memory and back.  (512 tokens of 32 heads on 8, 16 and 24 caches of 9000
// rows: 95 us in four pieces, 173 in two (whole 265) and 268 whole; 24 of 2250 to 9000 218, whole 258, in the longest pieces of
// at most 256 workgroups 378.)
void cut_tiles(const kvs_problem* p, long long at_once, WindowShape& sh) {
  constexpr long long kOnce = 3;
  constexpr double kTileUs = 2.06, kLaunchUs = 6, kBytesPerUs = 4e6;
  const Cut cut(p, sh, kWideTile);
  double best = 0;
  // (1, 2, 3, 4, 6, 8, 12, 16, .. pieces)
  for (long long n = 1; n <= kMaxParts; n = n < 3 ? n + 1 : (n & (n - 1)) != 0 ? n / 3 * 4 : n / 2 * 3) {
    const long long per = std::max(4ll, (cut.most + n - 1) / n);
    const auto [groups, tiles, partial] = cut.with(per);
    double time = cut.equal ? (double)((groups + at_once - 1) / at_once * (per + kOnce))
                            : (double)(tiles + groups * kOnce) / at_once + (double)(per + kOnce) / 2;
    if (n > 1) {
      const double partials = 8.0 * std::min(sh.R, sh.block) * (sh.D + 2) * (double)partial;
      time += (kLaunchUs + partials / kBytesPerUs) / kTileUs;
    }
    if (n == 1 || time < best) {
      best = time;
      sh.part_tiles = (int)per;
      sh.n_parts = (int)((cut.most + per - 1) / per);
    }
    if (per == 4 || (n == 1 && groups >= 8 * at_once)) break;   // (nothing to gain)
  }
}

kvs_status make_window_plan(const kvs_problem* p, int32_t span, bool packed, WindowPlan* plan, int* elt) {
  const kvs_status st = check_common(p, elt);
  if (st != KVS_OK) return st;
  if (p->group < 1 || p->window < 1 || (long long)p->group * p->window > KVS_MAX_WINDOW_ROWS) return KVS_ERR_INVALID_ARG;
  if (p->n_sink < 0 || span < 0 || (p->causal != 0 && p->causal != 1)) return KVS_ERR_INVALID_ARG;
  if (!(p->scale >= 0.f) || !std::isfinite(p->scale)) return KVS_ERR_INVALID_ARG;
  WindowShape& sh = plan->sh;
  sh.R = p->group * p->window;
  sh.G = p->group;
  sh.W = p->window;
  sh.D = p->head_dim;
  sh.causal = p->causal;
  sh.span = std::min(span, KVS_MAX_LEN);       // (a longer one hides nothing, and position - span stays an int)
  sh.sinks = std::min(p->n_sink, KVS_MAX_LEN);
  const double scale = p->scale == 0.f ? 1.0 / std::sqrt((double)p->head_dim) : (double)p->scale;
  sh.scale_log2 = (float)(scale * 1.4426950408889634);
  // From 33 bf16 query rows on tiles go through LDS (64 caches of 8224 rows: 64 query rows 76.7 us against 102, in 4 bits 55 against
  // 85; 32 rows 71.7 against 59.8).
  plan->wide = *elt == 2 && sh.R > 32;
  // Blocks of 32 query rows below that and with fp32 outputs, whose rows from 17 on would otherwise read the cache once per 16 (fp32,
  // 64 caches of 8192 rows, 64 query rows: 178 us against 229; blocks of 64 leave one wavefront per SIMD, 240).  Blocks of 16
  // where an fp32 cache stays in the memory-side cache, since the matrix cores then bound it and one wavefront more hides
  // what the others wait for (16 of 4096, 256 rows: 91 against 102).
  bool small = sh.R <= 16;
  if (*elt == 4 && !packed) {
    long long bytes = 0;
    for (int u = 0; u < p->n_units; ++u) bytes += 2ll * p->len[u] * sh.D * 4;
    small = small || bytes <= kStreamBytes;
  }
  // (of 64 channels several workgroups of 128 rows share a compute unit)
  sh.block = plan->wide ? (sh.R <= 128 || sh.D == 64 ? 128 : 256) : small ? 16 : 32;
  sh.n_blocks = (sh.R + sh.block - 1) / sh.block;
  // Workgroups that run at once.  One per compute unit keeps memory busy with plain rows (one token on 64 caches of 8224 rows:
  // 54.7 us with 256 workgroups, 57.2 with 512, 58.2 with 768).  Of those that read rows in 4 bits as many as fit the registers
  // (64 channels, pieces of 22 and 65 tiles: 768 workgroups 18.9 us, 256 26.0; 16 query rows of 128 channels 27.4 and 37.8;
  // fp32 queries, which take more registers, 8 caches of 131072 rows: 49.5 with 512, 59.2 with 768).
  // The wide kernel's are one or two (see there).
  int per_unit = 1;
  if (plan->wide) per_unit = sh.D == 64 || (packed && sh.block == 128) ? 2 : 1;
  else if (packed) per_unit = (sh.block == 16 ? 3 : 2) - (*elt == 4 && sh.D == 128);
  if (plan->wide) cut_tiles(p, kComputeUnits * per_unit, sh);
  else cut_rows(p, kComputeUnits * per_unit, sh);
  plan->equal = true;
  for (int u = 1; u < p->n_units; ++u) {
    plan->equal = plan->equal && p->len[u] == p->len[0] && p->in_row[u] - p->in_row[u - 1] == p->in_row[1] - p->in_row[0];
  }
  if (sh.n_parts > 1) {
    long long pieces = (long long)p->n_units * sh.n_parts;
    if (!plan->equal) {
      pieces = 0;
      for (int u = 0; u < p->n_units; ++u) pieces += unit_pieces(sh, p->len[u], plan->tile());
    }
    plan->part_bytes = align_up((size_t)pieces * sh.R * (sh.D + 2) * sizeof(float));
  }
  if (!plan->equal && p->n_units > kInlineUnits) plan->table_bytes = align_up((size_t)p->n_units * sizeof(UnitEntry));
  return KVS_OK;
}

// The plans of both forms, [0] of the plain one, and the size of the workspace that serves both.
kvs_status make_window_plans(const kvs_problem* p, int32_t span, WindowPlan (&plans)[2], int* elt, size_t* bytes) {
  for (const int packed : {0, 1}) {
    const kvs_status st = make_window_plan(p, span, packed != 0, &plans[packed], elt);
    if (st != KVS_OK) return st;
  }
  *bytes = std::max(plans[0].bytes(), plans[1].bytes());
  return KVS_OK;
}

struct Buffers {
  Range r[10];
  size_t n = 0;
  void add(const void* p, size_t bytes, bool is_output) {
    if (bytes > 0) r[n++] = {p, bytes, is_output};           // (a buffer of no rows may be anything)
  }
};

kvs_status window_attention(const kvs_problem* p, int32_t span, bool packed, const void* Q, const Cache& cache, void* out,
                            void* ws, size_t ws_bytes, void* hip_stream) {
  WindowPlan plans[2];
  int elt = 0;
  size_t need = 0;
  kvs_status st = make_window_plans(p, span, plans, &elt, &need);
  if (st != KVS_OK) return st;
  const WindowPlan& plan = plans[packed];
  const WindowShape& sh = plan.sh;
  if (need > 0 && (ws == nullptr || ((uintptr_t)ws % kAlign) != 0 || ws_bytes < need)) return KVS_ERR_WORKSPACE;
  const size_t rows = rows_to(p, p->in_row), qo = (size_t)p->n_units * sh.R * sh.D * elt;
  const size_t row_bytes = packed ? (size_t)sh.D / 2 : (size_t)sh.D * elt;
  Buffers b;
  b.add(Q, qo, false);
  b.add(cache.k, rows * row_bytes, false);
  b.add(cache.v, rows * row_bytes, false);
  if (packed) {
    b.add(cache.ks, rows * (sh.D / 32), false);
    b.add(cache.vs, rows * (sh.D / 32), false);
  }
  if (cache.counts) b.add(cache.counts, rows * 4, false);
  b.add(out, qo, true);
  b.add(ws, need, true);
  if ((st = check_ranges(b.r, b.n)) != KVS_OK) return st;

  const hipStream_t s = (hipStream_t)hip_stream;
  (void)hipGetLastError();                     // an error left pending by the caller's earlier calls is not this call's
  float* part = sh.n_parts > 1 ? (float*)ws : nullptr;
  UnitEntry* table = nullptr;
  hipError_t e = hipSuccess;
  if (plan.table_bytes > 0) {
    table = (UnitEntry*)((char*)ws + plan.part_bytes);
    e = launch_window_table(p, sh, plan.tile(), table, s);
  }
  const CacheKind kind = elt == 4 ? (packed ? CacheKind::kPackedF32 : CacheKind::kF32)
                                  : (packed ? CacheKind::kPackedBf16 : CacheKind::kBf16);
  const auto launch = plan.wide ? launch_window_tiles : launch_window_rows;
  // (a call of more workgroups than a grid may have goes out in several launches)
  const int most_units = (int)std::max<long long>(1, kMostGroups / (sh.n_parts > 1 ? sh.R : 1));
  int before = 0;
  for (int first = 0, n = 0; e == hipSuccess && first < p->n_units; first += n) {
    EqualUnits equal;
    ListedUnits listed;
    int from = 0, to = 0;                      // units among these that are in pieces
    if (plan.equal) {
      n = (int)std::min<long long>({most_units, p->n_units - first,
                                    std::max<long long>(1, kMostGroups / ((long long)sh.n_blocks * sh.n_parts))});
      equal = {p->in_row[first], p->n_units > 1 ? p->in_row[1] - p->in_row[0] : 0, p->len[0], first, n};
      to = sh.n_parts > 1 ? n : 0;
    } else {
      listed.ext = table ? table + first : nullptr;
      listed.first = first;
      listed.before = before;
      long long pieces = 0;
      for (n = 0; n < most_units && first + n < p->n_units; ++n) {
        const int mine = unit_pieces(sh, p->len[first + n], plan.tile());
        if (n > 0 && (pieces + mine) * sh.n_blocks > kMostGroups) break;
        if (!table) listed.u[n] = {p->in_row[first + n], p->len[first + n], before + (int)pieces};
        if (mine > 1) {
          if (to == 0) from = n;
          to = n + 1;
        }
        pieces += mine;
      }
      for (int i = table ? 0 : n; i < kInlineUnits; ++i) listed.u[i] = UnitEntry{};
      listed.n = n;
      listed.pieces = (int)pieces;
      before += (int)pieces;
    }
    const EqualUnits* eq = plan.equal ? &equal : nullptr;
    const ListedUnits* li = plan.equal ? nullptr : &listed;
    e = launch(eq, li, sh, kind, cache, Q, out, part, s);
    if (e == hipSuccess && to > from) e = launch_window_reduce(eq, li, from, to - from, sh, elt == 4, plan.tile(), part, out, s);
  }
  return launched(e, "an attention launch");
}

// ---- conversions
// The units' destination ranges are disjoint.
kvs_status check_disjoint(const kvs_problem* p) {
  auto end = [&](int u) { return (long long)p->out_row[u] + p->len[u]; };
  bool ascending = true;
  for (int u = 1; u < p->n_units; ++u) ascending = ascending && end(u - 1) <= p->out_row[u];
  if (ascending) return KVS_OK;
  std::unique_ptr<int[]> order(new (std::nothrow) int[p->n_units]);
  if (!order) return KVS_ERR_DEVICE;
  int n = 0;
  for (int u = 0; u < p->n_units; ++u) {
    if (p->len[u] > 0) order[n++] = u;
  }
  std::sort(order.get(), order.get() + n, [&](int a, int b) { return p->out_row[a] < p->out_row[b]; });
  for (int i = 1; i < n; ++i) {
    if (end(order[i - 1]) > p->out_row[order[i]]) return KVS_ERR_INVALID_ARG;
  }
  return KVS_OK;
}

// The checks of both directions, then f(equal, listed) for every launch.  rows, packed: K, V and the four
// packed arrays; to_packed: which side is written.
template <typename F>
kvs_status convert(const kvs_problem* p, const void* K, const void* V, const PackedRange& c, bool to_packed, F&& f) {
  int elt = 0;
  kvs_status st = check_common(p, &elt);
  if (st != KVS_OK) return st;
  if (p->out_row == nullptr) return KVS_ERR_INVALID_ARG;
  for (int u = 0; u < p->n_units; ++u) {
    if (p->out_row[u] < 0 || p->out_row[u] > kMostRow) return KVS_ERR_INVALID_ARG;
  }
  if ((st = check_disjoint(p)) != KVS_OK) return st;
  const size_t plain = rows_to(p, to_packed ? p->in_row : p->out_row), coded = rows_to(p, to_packed ? p->out_row : p->in_row);
  const size_t D = (size_t)p->head_dim;
  Buffers b;
  b.add(K, plain * D * elt, !to_packed);
  b.add(V, plain * D * elt, !to_packed);
  b.add(c.kc, coded * (D / 2), to_packed);
  b.add(c.ks, coded * (D / 32), to_packed);
  b.add(c.vc, coded * (D / 2), to_packed);
  b.add(c.vs, coded * (D / 32), to_packed);
  if ((st = check_ranges(b.r, b.n)) != KVS_OK) return st;

  (void)hipGetLastError();
  const int per = kPackValues / p->head_dim;
  hipError_t e = hipSuccess;
  for (int first = 0, n = 0; e == hipSuccess && first < p->n_units; first += n) {
    EqualMoves equal = {{p->in_row[first], p->out_row[first], p->len[first]}, 0, 0, 1};
    n = 1;
    if (first + 1 < p->n_units) {
      equal.src_step = p->in_row[first + 1] - p->in_row[first];
      equal.dst_step = p->out_row[first + 1] - p->out_row[first];
    }
    while (n < kMostMoves && first + n < p->n_units && p->len[first + n] == p->len[first] &&
           p->in_row[first + n] - p->in_row[first + n - 1] == equal.src_step &&
           p->out_row[first + n] - p->out_row[first + n - 1] == equal.dst_step) {
      ++n;
    }
    if (n >= std::min(kListedMoves, p->n_units - first)) {     // the longer run of the two
      equal.n = n;
      if (equal.first.len > 0) e = f(&equal, (const ListedMoves*)nullptr);
      continue;
    }
    ListedMoves listed = {};
    for (n = 0; n < kListedMoves && first + n < p->n_units; ++n) {
      const int u = first + n, groups = (p->len[u] + per - 1) / per;
      if (n > 0 && listed.groups > kMostMoveGroups - groups) break;
      listed.u[n] = {p->in_row[u], p->out_row[u], p->len[u]};
      listed.before[n] = listed.groups;
      listed.groups += groups;
    }
    listed.n = n;
    for (int i = n; i < kListedMoves; ++i) listed.before[i] = INT_MAX;
    if (listed.groups > 0) e = f((const EqualMoves*)nullptr, &listed);
  }
  return launched(e, "a conversion launch");
}

}  // namespace
}  // namespace kvs

using namespace kvs;

extern "C" {

kvs_status kvs_window_attention_workspace_size(const kvs_problem* p, int32_t span, size_t* bytes) {
  if (bytes == nullptr) return KVS_ERR_INVALID_ARG;
  WindowPlan plans[2];
  int elt = 0;
  size_t need = 0;
  const kvs_status st = make_window_plans(p, span, plans, &elt, &need);
  if (st == KVS_OK) *bytes = need;
  return st;
}

kvs_status kvs_window_attention(const kvs_problem* p, int32_t span, const void* Q, const void* K, const void* V,
                                const int32_t* counts, void* out, void* ws, size_t ws_bytes, void* hip_stream) {
  const Cache cache = {K, V, nullptr, nullptr, counts};
  return window_attention(p, span, /*packed=*/false, Q, cache, out, ws, ws_bytes, hip_stream);
}

kvs_status kvs_window_attention_packed(const kvs_problem* p, int32_t span, const void* Q, const void* K_codes,
                                       const void* K_scales, const void* V_codes, const void* V_scales,
                                       const int32_t* counts, void* out, void* ws, size_t ws_bytes, void* hip_stream) {
  const Cache cache = {K_codes, V_codes, (const uint8_t*)K_scales, (const uint8_t*)V_scales, counts};
  return window_attention(p, span, /*packed=*/true, Q, cache, out, ws, ws_bytes, hip_stream);
}

kvs_status kvs_pack(const kvs_problem* p, const void* K, const void* V, void* K_codes, void* K_scales, void* V_codes,
                    void* V_scales, void* hip_stream) {
  const PackedRange to = {(uint8_t*)K_codes, (uint8_t*)K_scales, (uint8_t*)V_codes, (uint8_t*)V_scales};
  return convert(p, K, V, to, /*to_packed=*/true, [&](const EqualMoves* equal, const ListedMoves* listed) {
    return launch_pack(equal, listed, p->io_dtype, p->head_dim, K, V, to, (hipStream_t)hip_stream);
  });
}

kvs_status kvs_unpack(const kvs_problem* p, const void* K_codes, const void* K_scales, const void* V_codes,
                      const void* V_scales, void* K, void* V, void* hip_stream) {
  const PackedRange from = {(uint8_t*)K_codes, (uint8_t*)K_scales, (uint8_t*)V_codes, (uint8_t*)V_scales};
  return convert(p, K, V, from, /*to_packed=*/false, [&](const EqualMoves* equal, const ListedMoves* listed) {
    return launch_unpack(equal, listed, p->io_dtype, p->head_dim, from, K, V, (hipStream_t)hip_stream);
  });
}

}  // extern "C"
