// Drives the host layer of the masked attention and of the 4-bit conversions (kvs_window_api.hip) on the CPU, under sanitizers.
// The launchers are stand-ins that go over everything that a launch's kernels would index and check it against the call's
// buffers.  Test infrastructure.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <vector>

#include "kvs_pack.h"
#include "kvs_window.h"

namespace {
void fail(const char* what, int line) {
  std::fprintf(stderr, "check failed at line %d: %s\n", line, what);
  std::exit(1);
}
#define CHECK(x) do { if (!(x)) fail(#x, __LINE__); } while (0)

const kvs_problem* g_problem = nullptr;   // the call under way
size_t g_ws_bytes = 0;
char* g_ws = nullptr;
std::vector<int> g_done;                  // units launched
std::vector<kvs::UnitEntry> g_table;
long long g_before = 0;                   // pieces of the units launched
size_t g_reduced = 0;                     // units whose partial results have been added up
}  // namespace

namespace kvs {

int debug_switch(kvs_debug_switch) { return 0; }

hipError_t launch_window_table(const kvs_problem* p, const WindowShape& sh, int tile, UnitEntry* dst, hipStream_t) {
  CHECK((char*)dst >= g_ws && (char*)(dst + p->n_units) <= g_ws + g_ws_bytes);
  g_table.clear();
  int before = 0;
  for (int i = 0; i < p->n_units; ++i) {
    g_table.push_back({p->in_row[i], p->len[i], before});
    before += unit_pieces(sh, p->len[i], tile);
  }
  return hipSuccess;
}

// A unit of the launch, as its kernels see it.
CacheUnit unit_at(const EqualUnits* equal, const ListedUnits* listed, const WindowShape& sh, int i) {
  if (equal) return {equal->in_row + i * equal->step, equal->len, equal->first + i, (equal->first + i) * sh.n_parts};
  const UnitEntry e = listed->ext ? g_table[listed->first + i] : listed->u[i];
  return {e.in_row, e.len, listed->first + i, e.before};
}

template <int TILE>
hipError_t attended(const EqualUnits* equal, const ListedUnits* listed, const WindowShape& sh, float* part) {
  CHECK((equal != nullptr) != (listed != nullptr));
  const int n_units = equal ? equal->n : listed->n, first = equal ? equal->first : listed->first;
  const long long pieces = equal ? pieces_of(*equal, sh) : pieces_of(*listed, sh);
  CHECK(n_units > 0 && first == (int)g_done.size() && (listed == nullptr || listed->ext != nullptr || n_units <= kInlineUnits));
  CHECK(pieces >= n_units && pieces * sh.n_blocks < 1ll << 24);
  CHECK(sh.n_parts <= kMaxParts && (long long)sh.n_blocks * sh.block >= sh.R && sh.block <= 256);
  CHECK(listed == nullptr || listed->before == g_before);
  g_reduced = std::max(g_reduced, g_done.size());
  for (int i = 0; i < n_units; ++i) {
    const CacheUnit un = unit_at(equal, listed, sh, i);
    g_done.push_back(un.index);
    CHECK(un.len == g_problem->len[un.index] && un.in_row == g_problem->in_row[un.index]);
    CHECK(un.before == g_before);
    const int mine = unit_pieces(sh, un.len, TILE);
    CHECK(mine >= 1 && mine <= sh.n_parts);
    g_before += equal ? sh.n_parts : mine;
    for (int b = 0; b < sh.n_blocks; b += 1 + sh.n_blocks / 20) {
      const Reach r = reach_of<TILE>(sh, un.len, b);
      CHECK(parts_of(r.tiles, sh.part_tiles) <= mine);
      CHECK(0 <= r.sink_end && r.sink_end <= r.first && r.first <= r.end && r.end <= un.len);
      CHECK(r.sink_tiles * TILE >= r.sink_end && (r.tiles - r.sink_tiles) * TILE >= r.end - r.first);
    }
    if (mine > 1) {
      const size_t last = ((size_t)(un.before + mine - 1) * sh.R + sh.R - 1) * (sh.D + 2) + sh.D + 2;
      CHECK((char*)part >= g_ws && (char*)(part + last) <= g_ws + g_ws_bytes);
      // (the table lies behind the partial results)
      CHECK(listed == nullptr || listed->ext == nullptr || (char*)(part + last) <= (char*)(listed->ext - listed->first));
    }
  }
  if (listed) CHECK(g_before - listed->before == listed->pieces);
  return hipSuccess;
}
hipError_t launch_window_rows(const EqualUnits* equal, const ListedUnits* listed, const WindowShape& sh, CacheKind, const Cache&,
                              const void*, void*, float* part, hipStream_t) {
  CHECK(sh.block == 16 || sh.block == 32);
  return attended<kWindowTile>(equal, listed, sh, part);
}
hipError_t launch_window_tiles(const EqualUnits* equal, const ListedUnits* listed, const WindowShape& sh, CacheKind kind,
                               const Cache&, const void*, void*, float* part, hipStream_t) {
  CHECK(sh.block == 128 || sh.block == 256);
  CHECK(kind == CacheKind::kBf16 || kind == CacheKind::kPackedBf16);
  return attended<kWideTile>(equal, listed, sh, part);
}
hipError_t launch_window_reduce(const EqualUnits* equal, const ListedUnits* listed, int at, int n, const WindowShape& sh, bool,
                                int tile, const float* part, void*, hipStream_t) {
  const int n_units = equal ? equal->n : listed->n;
  CHECK(part != nullptr && sh.n_parts > 1 && n > 0 && at >= 0 && at + n <= n_units && (long long)n * sh.R < 1ll << 24);
  // every unit in pieces is among them
  const size_t first = g_done.size() - n_units;
  CHECK(g_reduced <= first);
  for (int i = 0; i < n_units; ++i) {
    CHECK((i >= at && i < at + n) || unit_pieces(sh, unit_at(equal, listed, sh, i).len, tile) == 1);
  }
  g_reduced = g_done.size();
  return hipSuccess;
}

namespace {
hipError_t moved(const EqualMoves* equal, const ListedMoves* listed, int D) {
  CHECK((equal != nullptr) != (listed != nullptr));
  CHECK(equal ? equal->n > 0 && equal->n <= kMostMoves && equal->first.len > 0 : listed->n > 0 && listed->n <= kListedMoves);
  const int n = equal ? equal->n : listed->n, per = kPackValues / D;
  int groups = 0;
  for (int i = 0; i < n; ++i) {
    const RowMove m = equal ? RowMove{equal->first.src + i * equal->src_step, equal->first.dst + i * equal->dst_step,
                                      equal->first.len}
                            : listed->u[i];
    if (listed) {
      CHECK(listed->before[i] == groups);
      groups += (m.len + per - 1) / per;
    }
    if (m.len == 0) continue;
    int u = g_done.empty() ? 0 : g_done.back() + 1;      // (in the order of the units)
    while (g_problem->len[u] == 0) ++u;
    CHECK(m.src == g_problem->in_row[u] && m.dst == g_problem->out_row[u] && m.len == g_problem->len[u]);
    g_done.push_back(u);
  }
  if (listed) for (int i = n; i < kListedMoves; ++i) CHECK(listed->before[i] > groups);
  if (listed) CHECK(groups > 0 && groups == listed->groups && groups < 1 << 24);
  return hipSuccess;
}
}  // namespace
hipError_t launch_pack(const EqualMoves* equal, const ListedMoves* listed, kvs_dtype, int D, const void*, const void*,
                       const PackedRange&, hipStream_t) {
  return moved(equal, listed, D);
}
hipError_t launch_unpack(const EqualMoves* equal, const ListedMoves* listed, kvs_dtype, int D, const PackedRange&, void*, void*,
                         hipStream_t) {
  return moved(equal, listed, D);
}

}  // namespace kvs

namespace {

struct Call {
  std::vector<int32_t> len;
  std::vector<int64_t> in, out;
  kvs_problem p{};
  explicit Call(std::vector<int32_t> lens, int G = 4, int W = 1, int D = 128) : len(std::move(lens)) {
    int64_t at = 0;
    for (int32_t n : len) { in.push_back(at); out.push_back(at); at += n; }
    p.n_units = (int)len.size(); p.group = G; p.window = W; p.head_dim = D; p.io_dtype = KVS_BF16; p.causal = 1;
    p.len = len.data(); p.in_row = in.data(); p.out_row = out.data(); p.budget = nullptr;
  }
};

// (addresses that are compared and never followed)
void* at(int i) { return (void*)((uintptr_t)(i + 1) << 42); }

kvs_status attend(const Call& c, int span, bool packed) {
  size_t bytes = 12345;
  kvs_status st = kvs_window_attention_workspace_size(&c.p, span, &bytes);
  if (st != KVS_OK) return st;
  CHECK(bytes % 256 == 0);
  g_problem = &c.p; g_ws = (char*)at(9); g_ws_bytes = bytes; g_done.clear(); g_table.clear(); g_before = 0; g_reduced = 0;
  if (bytes > 0) {
    auto with = [&](void* ws, size_t n) {
      return kvs_window_attention(&c.p, span, at(0), at(1), at(2), nullptr, at(3), ws, n, nullptr);
    };
    CHECK(with(g_ws, bytes - 1) == KVS_ERR_WORKSPACE && with(nullptr, bytes) == KVS_ERR_WORKSPACE);
    CHECK(with(g_ws + 16, bytes) == KVS_ERR_WORKSPACE && with(at(3), bytes) == KVS_ERR_ALIAS);
    CHECK(g_done.empty());
  }
  void* ws = bytes > 0 ? g_ws : nullptr;
  st = packed ? kvs_window_attention_packed(&c.p, span, at(0), at(1), at(4), at(2), at(5), nullptr, at(3), ws, bytes, nullptr)
              : kvs_window_attention(&c.p, span, at(0), at(1), at(2), (const int32_t*)at(6), at(3), ws, bytes, nullptr);
  if (st == KVS_OK) {
    CHECK((int)g_done.size() == c.p.n_units);
    for (int i = 0; i < c.p.n_units; ++i) CHECK(g_done[i] == i);
    CHECK(g_before == c.p.n_units || g_reduced > 0);     // (more pieces than units: they have been added up)
  }
  return st;
}

kvs_status convert(const Call& c) {
  g_problem = &c.p; g_done.clear();
  kvs_status st = kvs_pack(&c.p, at(0), at(1), at(2), at(3), at(4), at(5), nullptr);
  if (st != KVS_OK) return st;
  size_t filled = 0;
  for (int32_t n : c.len) filled += n > 0;
  CHECK(g_done.size() == filled);
  g_done.clear();
  return kvs_unpack(&c.p, at(2), at(3), at(4), at(5), at(0), at(1), nullptr);
}

}  // namespace

int main() {
  // problems of every size, every mask
  std::mt19937 rng(7);
  auto upto = [&](double most) { return (int)std::exp(std::uniform_real_distribution<>(0, std::log(most))(rng)); };
  for (int i = 0; i < 1000; ++i) {
    const int units = upto(i % 10 == 0 ? 3000 : 100), longest = upto(i % 7 == 0 ? 4194304 : 40000);
    std::vector<int32_t> lens(units, longest);
    if (i % 3) for (int32_t& n : lens) n = std::uniform_int_distribution<>(0, longest)(rng);
    Call c(lens, upto(64), i % 4 == 0 ? upto(30000) : upto(8), i % 2 ? 64 : 128);
    if ((long long)c.p.group * c.p.window > KVS_MAX_WINDOW_ROWS) continue;
    c.p.causal = i % 5 != 0;
    c.p.n_sink = i % 3 ? upto(5000) : 0;
    c.p.io_dtype = i % 2 ? KVS_F32 : KVS_BF16;
    CHECK(attend(c, i % 3 == 0 ? 0 : upto(5000000), i % 2) == KVS_OK);
    if (i % 4 == 0) {                                  // gaps, and an order of the units' rows of its own
      std::shuffle(c.in.begin(), c.in.end(), rng);     // (source ranges may overlap)
      for (size_t u = 0; u < c.out.size(); ++u) c.out[u] = (int64_t)(c.out.size() - u) * (longest + 3);
    }
    CHECK(convert(c) == KVS_OK);
  }
  // one long unit among many: its pieces are no reason for a large workspace
  for (int units : {50, 20000}) {
    std::vector<int32_t> lens(units, 100);
    lens[units / 2] = 1000000;
    Call c(lens);
    size_t bytes = 0;
    CHECK(attend(c, 0, false) == KVS_OK);
    CHECK(kvs_window_attention_workspace_size(&c.p, 0, &bytes) == KVS_OK);
    CHECK(bytes > 0 && bytes <= (units + 3 * 256ull) * (4 * 130 * 4 + 16) + 512);
  }
  // the largest calls
  CHECK(attend(Call({KVS_MAX_LEN}, 1, KVS_MAX_WINDOW_ROWS), 0, false) == KVS_OK);
  CHECK(attend(Call({KVS_MAX_LEN, 1, 0}, 64, 65536), 2147483647, true) == KVS_OK);
  CHECK(attend(Call(std::vector<int32_t>(100000, 1)), 0, true) == KVS_OK);
  CHECK(convert(Call(std::vector<int32_t>(200000, 2))) == KVS_OK);
  std::vector<int32_t> longs(150, KVS_MAX_LEN);
  for (int i = 0; i < 150; ++i) longs[i] -= i % 7;
  CHECK(convert(Call(longs)) == KVS_OK);

  // refusals, each before any launch
  auto refused = [&](kvs_status want, auto&& change, int span = 0) {
    Call c({100, 200});
    change(c);
    g_done.clear();
    CHECK(attend(c, span, false) == want);
    CHECK(g_done.empty() || want == KVS_OK);
  };
  refused(KVS_OK, [](Call&) {});
  refused(KVS_ERR_INVALID_ARG, [](Call&) {}, -1);
  refused(KVS_ERR_INVALID_ARG, [](Call& c) { c.p.n_units = 0; });
  refused(KVS_ERR_INVALID_ARG, [](Call& c) { c.p.head_dim = 96; });
  refused(KVS_ERR_INVALID_ARG, [](Call& c) { c.p.group = 0; });
  refused(KVS_ERR_INVALID_ARG, [](Call& c) { c.p.window = -1; });
  refused(KVS_ERR_INVALID_ARG, [](Call& c) { c.p.group = 2049; c.p.window = 2048; });
  refused(KVS_ERR_INVALID_ARG, [](Call& c) { c.p.n_sink = -1; });
  refused(KVS_ERR_INVALID_ARG, [](Call& c) { c.p.causal = 2; });
  refused(KVS_ERR_INVALID_ARG, [](Call& c) { c.p.scale = -1.f; });
  refused(KVS_ERR_INVALID_ARG, [](Call& c) { c.p.len = nullptr; });
  refused(KVS_ERR_INVALID_ARG, [](Call& c) { c.p.in_row = nullptr; });
  refused(KVS_ERR_INVALID_ARG, [](Call& c) { c.len[1] = -1; });
  refused(KVS_ERR_INVALID_ARG, [](Call& c) { c.len[1] = KVS_MAX_LEN + 1; });
  refused(KVS_ERR_INVALID_ARG, [](Call& c) { c.in[0] = -1; });
  refused(KVS_ERR_INVALID_ARG, [](Call& c) { c.in[0] = INT64_MAX; });
  refused(KVS_ERR_DTYPE, [](Call& c) { const int bad = 2; std::memcpy(&c.p.io_dtype, &bad, sizeof(int)); });
  size_t bytes;
  CHECK(kvs_window_attention_workspace_size(nullptr, 0, &bytes) == KVS_ERR_INVALID_ARG);
  Call c({10, 20});
  CHECK(kvs_window_attention_workspace_size(&c.p, 0, nullptr) == KVS_ERR_INVALID_ARG);
  g_problem = &c.p; g_done.clear(); g_before = 0; g_reduced = 0;
  auto win = [&](void* q, void* k, void* v, void* n, void* o) {
    return kvs_window_attention(&c.p, 0, q, k, v, (const int32_t*)n, o, nullptr, 0, nullptr);
  };
  CHECK(win(nullptr, at(1), at(2), nullptr, at(3)) == KVS_ERR_INVALID_ARG);
  CHECK(win(at(0), nullptr, at(2), nullptr, at(3)) == KVS_ERR_INVALID_ARG);
  CHECK(win(at(0), at(1), nullptr, nullptr, at(3)) == KVS_ERR_INVALID_ARG);
  CHECK(win(at(0), at(1), at(2), nullptr, nullptr) == KVS_ERR_INVALID_ARG);
  CHECK(win((char*)at(0) + 8, at(1), at(2), nullptr, at(3)) == KVS_ERR_INVALID_ARG);
  CHECK(win(at(0), at(1), at(2), (char*)at(4) + 4, at(3)) == KVS_ERR_INVALID_ARG);
  for (int i : {0, 1, 2, 4}) CHECK(win(at(0), at(1), at(2), at(4), at(i)) == KVS_ERR_ALIAS);
  CHECK(win(at(0), at(1), at(2), nullptr, (char*)at(1) + 30 * 256 - 16) == KVS_ERR_ALIAS);
  auto four = [&](void* kc, void* ks, void* vc, void* vs, void* o) {
    return kvs_window_attention_packed(&c.p, 0, at(0), kc, ks, vc, vs, nullptr, o, nullptr, 0, nullptr);
  };
  CHECK(four(at(1), nullptr, at(2), at(5), at(3)) == KVS_ERR_INVALID_ARG);
  CHECK(four(at(1), at(4), at(2), nullptr, at(3)) == KVS_ERR_INVALID_ARG);
  CHECK(four(at(1), at(4), at(2), at(5), (char*)at(5) + 112) == KVS_ERR_ALIAS);
  auto pack = [&](void* k, void* v, void* kc, void* ks, void* vc, void* vs) {
    return kvs_pack(&c.p, k, v, kc, ks, vc, vs, nullptr);
  };
  CHECK(pack(nullptr, at(1), at(2), at(3), at(4), at(5)) == KVS_ERR_INVALID_ARG);
  CHECK(pack(at(0), at(1), at(2), at(3), at(4), (char*)at(5) + 2) == KVS_ERR_INVALID_ARG);
  CHECK(pack(at(0), at(1), at(2), at(2), at(4), at(5)) == KVS_ERR_ALIAS);
  CHECK(pack(at(0), at(1), at(0), at(3), at(4), at(5)) == KVS_ERR_ALIAS);
  CHECK(kvs_unpack(&c.p, at(2), at(3), at(4), at(5), at(0), at(0), nullptr) == KVS_ERR_ALIAS);
  CHECK(g_done.empty());
  CHECK(kvs_unpack(&c.p, at(2), at(2), at(4), at(5), at(0), at(1), nullptr) == KVS_OK);    // (inputs may alias)
  CHECK(g_done.size() == 2);
  g_done.clear();
  c.out[1] = 5;                                        // into the first unit's rows
  CHECK(pack(at(0), at(1), at(2), at(3), at(4), at(5)) == KVS_ERR_INVALID_ARG);
  c.out[0] = 20, c.out[1] = 1;
  CHECK(pack(at(0), at(1), at(2), at(3), at(4), at(5)) == KVS_ERR_INVALID_ARG);
  c.out[1] = 0;
  CHECK(g_done.empty() && pack(at(0), at(1), at(2), at(3), at(4), at(5)) == KVS_OK);
  c.p.out_row = nullptr;
  CHECK(pack(at(0), at(1), at(2), at(3), at(4), at(5)) == KVS_ERR_INVALID_ARG);
  // units of no rows need no buffers of rows
  Call none({0, 0});
  g_problem = &none.p; g_done.clear(); g_before = 0; g_reduced = 0;
  CHECK(kvs_window_attention(&none.p, 0, at(0), nullptr, nullptr, nullptr, at(3), nullptr, 0, nullptr) == KVS_OK);
  CHECK(g_done.size() == 2);
  CHECK(kvs_pack(&none.p, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr) == KVS_OK && g_done.size() == 2);
  std::puts("all checks passed");
  return 0;
}
