// Host runtime and C ABI of the orthogonalised updates (declared in include/zo.h): the
// workspace's layout, the groups that share it, and the launches of a call.
#include <algorithm>
#include <array>
#include <cmath>
#include <cstring>
#include <functional>
#include <memory>
#include <new>
#include <queue>
#include <utility>
#include <vector>

#include "../../include/zo.h"
#include "zo_host.h"
#include "zo_ops.h"

namespace {

using namespace zo::host;

constexpr double kMuonA = 3.4445, kMuonB = -4.7750, kMuonC = 2.0315;
// Matrices are worked on in groups that share the iterates' buffers, of at most this many
// bytes (or one matrix): enough work in every launch to fill the device, without a second
// copy of a whole model's weights.
constexpr int64_t kGroupBytes = int64_t(1) << 30;

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// The tiles of one launch, dealt to the SM pairs: pair q's are tiles[first[q] .. first[q + 1]).
struct TileList {
  int32_t tile0 = 0, n = 0, pairs = 0, narrow = 0, first0 = 0;
};
struct Group {
  int32_t unit0 = 0, n_units = 0;
  int32_t list[2][3] = {{-1, -1, -1}, {-1, -1, -1}};   // tile lists by [pairs][OrthoPhase]
};

// Matrices that one launch of a one-launch kernel takes: one kernel (rows: zo_ortho_mma.cu's
// instance, 0 zo_ortho_small.cu's), one cluster size, and shared memories within a factor of two
// (they decide how many CTAs share an SM).
struct Small {
  int32_t rows = 0, cluster = 0, smem = 0, least = 0, first = 0, n = 0;
};

// Where everything lies in the workspace: the status word, the tables, the norm's partial
// sums, then the buffers that the groups share.
struct Layout {
  std::vector<zo::OrthoMat> mats;       // buffer pointers hold byte offsets until placed
  std::vector<int4> units;
  std::vector<zo::OrthoTile> tiles;
  std::vector<Group> groups;
  std::vector<TileList> lists;
  std::vector<int32_t> first;           // kOrthoMaxPairs + 1 of every list
  std::vector<int32_t> small_list;
  int32_t n_maps = 0;                   // matrices with tensor maps
  std::vector<Small> small;
  int64_t mats_at = 0, maps_at = 0, small_at = 0, units_at = 0, tiles_at = 0, first_at = 0, counter_at = 0, slot_counter_at = 0, inverse_at = 0, partial_at = 0, sums_at = 0, buffers_at = 0, bytes = 0;
  int64_t tables_end = 0;
};

zo_status check_matrix(const zo_muon_matrix& m) {
  if (!m.W || !m.G) return refuse(ZO_ERR_INVALID_ARG, "null W or G in zo_muon_matrix");
  if ((m.dtype != ZO_F32 && m.dtype != ZO_BF16) ||
      (m.grad_dtype != ZO_F32 && m.grad_dtype != ZO_BF16))
    return refuse(ZO_ERR_DTYPE, "unknown dtype in zo_muon_matrix");
  if (m.grade != ZO_MUON_GRADE_DTYPE && m.grade != ZO_MUON_GRADE_F32)
    return refuse(ZO_ERR_INVALID_ARG, "unknown grade in zo_muon_matrix");
  if (m.m < 1 || m.n < 1 || m.m >= (int64_t(1) << 24) || m.n >= (int64_t(1) << 24) ||
      m.ldw < m.n || m.ldg < m.n || m.ldw >= (int64_t(1) << 40) || m.ldg >= (int64_t(1) << 40) ||
      std::min(m.m, m.n) > (int64_t(1) << 16))
    return refuse(ZO_ERR_SHAPE, "zo_muon_matrix: need 1 <= m, n < 2^24, min(m, n) <= 2^16, "
                                "n <= ldw, ldg < 2^40");
  const auto aligned = [](const void* p, int32_t dtype) {
    return reinterpret_cast<uintptr_t>(p) % (dtype == ZO_BF16 ? 2 : 4) == 0;
  };
  if (!aligned(m.W, m.dtype) || !aligned(m.G, m.grad_dtype) || !aligned(m.M, ZO_F32))
    return refuse(ZO_ERR_ALIGN, "zo_muon_matrix: a buffer is not aligned to its elements");
  return ZO_OK;
}

zo_status check_matrices(const zo_muon_matrix* mats, int32_t n_mats) {
  if (!mats || n_mats <= 0) return refuse(ZO_ERR_INVALID_ARG, "need at least one matrix");
  for (int32_t i = 0; i < n_mats; ++i) {
    const zo_status st = check_matrix(mats[i]);
    if (st != ZO_OK) return st;
  }
  return ZO_OK;
}

int64_t depth(const zo::OrthoMat& d, int phase) { return phase == zo::kOrthoGram ? d.c : d.p; }

// What a tile costs, in SM cycles: its stages of 64 of K, and in a launch's time once more the
// epilogue behind the last one (measured at 2048 x 2048 and 1001 x 333).
struct TileCost {
  int64_t stage, tail;
};
TileCost tile_cost(bool pairs, bool narrow) {
  if (pairs) return narrow ? TileCost{600, 5500} : TileCost{950, 8000};
  return narrow ? TileCost{400, 6500} : TileCost{600, 11000};
}

// Parts of Gram's K for one matrix: where its own tiles are few, as many as make them about half
// of a GPU's SM pairs, each at least eight stages deep.  It goes by the matrix alone, so that its
// bits do not depend on what else the context holds.  (48 x 7680: one tile of 120 stages, 83 us
// of a 100 us step in one part.)
int32_t gram_parts(const zo::OrthoMat& d) {
  const int64_t blocks = (d.p + zo::kOrthoTileRows - 1) / zo::kOrthoTileRows;
  const int64_t tiles = blocks * (blocks + 1) / 2, stages = (d.c + 63) / 64;
  int32_t parts = 1;
  while (2 * parts <= zo::kOrthoMaxParts && 2 * parts * tiles <= 38 && 16 * parts <= stages) parts *= 2;
  return parts;
}

// Deals tiles, the deepest first, to n SM pairs, each to the pair with the least to do so far (a
// pair's tiles keep their order); returns the longest pair's cycles.
int64_t deal(const std::vector<zo::OrthoTile>& tiles, int32_t n, TileCost cost,
             std::vector<std::vector<zo::OrthoTile>>* dealt) {
  using Load = std::pair<int64_t, int32_t>;   // work so far, pair
  std::priority_queue<Load, std::vector<Load>, std::greater<Load>> least;
  for (int32_t q = 0; q < n; ++q) least.push({0, q});
  int64_t most = 0;
  for (const zo::OrthoTile& t : tiles) {
    Load to = least.top();
    least.pop();
    if (dealt) (*dealt)[to.second].push_back(t);
    to.first += (int64_t)(t.k1 - t.k0) * cost.stage + cost.tail / 4;
    most = std::max(most, to.first);
    least.push(to);
  }
  return most + cost.tail;
}

// The tiles of one product over the matrices [first, next) of a group: those of X X^T and
// b A + c A A that meet or lie left of the diagonal's blocks of rows, or all of X'.
std::vector<zo::OrthoTile> make_tiles(const Layout& L, size_t first, size_t next, int pr, int phase,
                                      bool narrow) {
  std::vector<zo::OrthoTile> tiles;
  int32_t slots = 0, sums = 0;
  for (size_t i = first; i < next; ++i) {
    const zo::OrthoMat& d = L.mats[i];
    if (d.small || d.pairs != pr) continue;
    const int32_t stages = (int32_t)((depth(d, phase) + 63) / 64);
    const int32_t of = phase == zo::kOrthoGram ? gram_parts(d) : 1;
    for (int64_t r = 0; r < d.p; r += zo::kOrthoTileRows) {
      const int64_t end = phase == zo::kOrthoApply ? d.c : std::min(r + zo::kOrthoTileRows, d.p);
      for (int64_t c = 0; c < end; c += zo::ortho_tile_cols(pr != 0, narrow)) {
        for (int32_t k = 0; k < of; ++k)
          tiles.push_back({(int32_t)i, (int32_t)r, (int32_t)c, d.maps, stages * k / of,
                           stages * (k + 1) / of, of > 1 ? slots : -1, k, of, sums});
        slots += of > 1;
        sums += of > 1 ? of : 0;
      }
    }
  }
  std::stable_sort(tiles.begin(), tiles.end(), [](const zo::OrthoTile& a, const zo::OrthoTile& b) {
    return a.k1 - a.k0 > b.k1 - b.k0;
  });
  return tiles;
}

// The tiling with the least estimated time on the SM pairs of a whole GPU: wide or narrow
// tiles, which give the same bits.
std::vector<zo::OrthoTile> best_tiles(const Layout& L, size_t first, size_t next, int pr, int phase,
                                      int32_t* narrow) {
  constexpr int32_t kPairsOfGpu = 76;
  std::vector<zo::OrthoTile> wide = make_tiles(L, first, next, pr, phase, false);
  if (wide.empty()) return wide;
  std::vector<zo::OrthoTile> thin = make_tiles(L, first, next, pr, phase, true);
  *narrow = deal(thin, kPairsOfGpu, tile_cost(pr != 0, true), nullptr) <
            deal(wide, kPairsOfGpu, tile_cost(pr != 0, false), nullptr);
  return *narrow ? thin : wide;
}

// Every list's tiles in the order of the n_pairs SM pairs that take them.
void deal_tiles(Layout& L, int32_t n_pairs) {
  L.first.assign(L.lists.size() * (zo::kOrthoMaxPairs + 1), 0);
  for (const TileList& list : L.lists) {
    const auto begin = L.tiles.begin() + list.tile0;
    const std::vector<zo::OrthoTile> tiles(begin, begin + list.n);
    std::vector<std::vector<zo::OrthoTile>> dealt(n_pairs);
    deal(tiles, n_pairs, tile_cost(list.pairs != 0, list.narrow != 0), &dealt);
    int32_t at = 0;
    for (int32_t q = 0; q <= zo::kOrthoMaxPairs; ++q) {
      L.first[list.first0 + q] = at;
      if (q < n_pairs)
        for (const zo::OrthoTile& t : dealt[q]) L.tiles[list.tile0 + at++] = t;
    }
  }
}

uint16_t* at_offset(int64_t off) { return reinterpret_cast<uint16_t*>(off); }

zo_status plan(const zo_muon_matrix* mats, int32_t n_mats, Layout* out) {
  Layout& L = *out;
  int64_t used = 0, most = 0, slots = 0;
  for (int32_t i = 0; i < n_mats; ++i) {
    const zo_muon_matrix& m = mats[i];
    zo::OrthoMat d{};
    d.G = m.G;
    d.W = m.W;
    d.M = m.M;
    d.ldg = m.ldg;
    d.ldw = m.ldw;
    d.m = m.m;
    d.n = m.n;
    d.p = std::min(m.m, m.n);
    d.c = std::max(m.m, m.n);
    d.grad_bf16 = m.grad_dtype == ZO_BF16;
    d.bf16 = m.dtype == ZO_BF16;
    d.tall = m.m > m.n;
    d.pairs = m.grade == ZO_MUON_GRADE_F32 || zo::ortho_pairs(d.bf16, d.p);
    d.wide_rows = aligned16(m.W) && m.ldw * (d.bf16 ? 2 : 4) % 16 == 0;
    d.small = zo::ortho_mma_cluster(d.p, d.c);
    if (d.small == 0) d.small = zo::ortho_small_cluster(d.p, d.c);
    if (d.small > 0) {
      L.mats.push_back(d);
      continue;
    }
    d.maps = L.n_maps++;
    d.ldx = round_up(d.c, 64);
    d.ldp = round_up(d.p, 64);
    const int64_t x_bytes = d.p * d.ldx * 2, a_bytes = d.p * d.ldp * 2;
    const int64_t bytes = (d.pairs ? 4 : 3) * x_bytes + (d.pairs ? 4 : 2) * a_bytes;
    if (L.groups.empty() || used + bytes > kGroupBytes) {
      L.groups.emplace_back();
      L.groups.back().unit0 = (int32_t)L.units.size();
      used = 0;
    }
    Group& g = L.groups.back();
    int64_t off = used;
    const auto take = [&](int64_t n) {
      const int64_t at = off;
      off += n;                                     // every size is a multiple of 128
      return at_offset(at);
    };
    d.xh[0] = take(x_bytes);
    d.xh[1] = take(x_bytes);
    d.xl[0] = take(x_bytes);
    d.xl[1] = d.pairs ? take(x_bytes) : d.xl[0];
    d.ah = take(a_bytes);
    d.bh = take(a_bytes);
    if (d.pairs) {
      d.al = take(a_bytes);
      d.bl = take(a_bytes);
    }
    used = round_up(off, 256);
    most = std::max(most, used);
    d.unit0 = (int32_t)slots;
    for (int64_t r = 0; r < d.m; r += zo::kOrthoUnitRows)
      for (int64_t c = 0; c < d.n; c += zo::kOrthoUnitCols)
        L.units.push_back(make_int4(i, (int)r, (int)c, (int)slots++));
    d.n_units = (int32_t)(slots - d.unit0);
    if (slots > (int64_t(1) << 30))
      return refuse(ZO_ERR_SHAPE, "zo_muon: too many elements in one context");
    g.n_units += d.n_units;
    L.mats.push_back(d);
  }
  // tiles, group by group
  int32_t slots_used = 0;
  int64_t sums_floats = 0;
  size_t next = 0;
  for (Group& g : L.groups) {
    const size_t first = next;
    int64_t units = 0;
    for (; next < L.mats.size() && units + L.mats[next].n_units <= g.n_units; ++next)
      units += L.mats[next].n_units;               // (a small matrix has none)
    for (int pr = 0; pr < 2; ++pr)
      for (const int phase : {zo::kOrthoGram, zo::kOrthoPoly, zo::kOrthoApply}) {
        TileList list{(int32_t)L.tiles.size(), 0, pr, 0, (int32_t)(L.lists.size() * (zo::kOrthoMaxPairs + 1))};
        const std::vector<zo::OrthoTile> tiles = best_tiles(L, first, next, pr, phase, &list.narrow);
        if (tiles.empty()) continue;
        L.tiles.insert(L.tiles.end(), tiles.begin(), tiles.end());
        list.n = (int32_t)tiles.size();
        for (const zo::OrthoTile& t : tiles)
          if (t.parts > 1) {
            slots_used = std::max(slots_used, t.slot + 1);
            sums_floats = std::max(sums_floats, (int64_t)(t.sum0 + t.parts) *
                                                    zo::ortho_part_floats(pr != 0, list.narrow != 0));
          }
        g.list[pr][phase] = (int32_t)L.lists.size();
        L.lists.push_back(list);
      }
    if (L.tiles.size() > (size_t(1) << 28))
      return refuse(ZO_ERR_SHAPE, "zo_muon: too many tiles in one context");
  }
  // the one-launch kernels' matrices by instance, cluster size and shared memory
  std::vector<std::array<int32_t, 4>> order;
  for (size_t i = 0; i < L.mats.size(); ++i) {
    const zo::OrthoMat& d = L.mats[i];
    if (d.small == 0) continue;
    const int32_t rows = zo::ortho_mma_rows(d.p);
    order.push_back({rows, d.small, rows ? zo::ortho_mma_smem(d.p, d.c, d.small)
                                         : zo::ortho_small_smem(d.p, d.c, d.small), (int32_t)i});
  }
  std::sort(order.begin(), order.end());
  for (const auto& o : order) {
    if (L.small.empty() || L.small.back().rows != o[0] || L.small.back().cluster != o[1] ||
        o[2] > 2 * L.small.back().least)
      L.small.push_back({o[0], o[1], o[2], o[2], (int32_t)L.small_list.size(), 0});
    L.small.back().smem = o[2];                    // the largest so far
    ++L.small.back().n;
    L.small_list.push_back(o[3]);
  }
  int64_t at = 256;                                 // the status word
  const auto place = [&](int64_t bytes) {
    const int64_t here = at;
    at = round_up(at + bytes, 256);
    return here;
  };
  L.mats_at = place(sizeof(zo::OrthoMat) * L.mats.size());
  L.maps_at = place((int64_t)sizeof(CUtensorMap) * zo::kOrthoMaps * L.n_maps);
  L.small_at = place(sizeof(int32_t) * L.small_list.size());
  L.units_at = place(sizeof(int4) * L.units.size());
  L.tiles_at = place(sizeof(zo::OrthoTile) * L.tiles.size());
  L.first_at = place((int64_t)sizeof(int32_t) * L.lists.size() * (zo::kOrthoMaxPairs + 1));
  L.counter_at = place(sizeof(uint32_t) * L.mats.size());       // zeros, uploaded too
  L.slot_counter_at = place((int64_t)sizeof(uint32_t) * zo::kOrthoSlotCounters * slots_used);
  L.tables_end = at;
  L.inverse_at = place(sizeof(float2) * L.mats.size());
  L.sums_at = place((int64_t)sizeof(float) * sums_floats);
  L.partial_at = place(sizeof(double) * slots);
  L.buffers_at = at;
  L.bytes = at + most;
  return ZO_OK;
}

// The tensor maps of one matrix (its buffers placed).
bool encode_maps(const zo::OrthoMat& d, CUtensorMap* m) {
  uint16_t* buf[8] = {d.xh[0], d.xh[1], d.xl[0], d.xl[1], d.ah, d.al, d.bh, d.bl};
  for (int k = 0; k < 8; ++k) {
    if (!buf[k]) continue;
    const int64_t cols = k < 4 ? d.c : d.p, ld = k < 4 ? d.ldx : d.ldp;
    if (!encode_f16_2d(m + k, buf[k], cols, d.p, ld * 2, 64, 64) ||
        !encode_16b_2d(m + zo::kMapStoreX + k, buf[k], cols, d.p, ld * 2, 32, 32, true,
                       CU_TENSOR_MAP_SWIZZLE_64B))
      return false;
  }
  return true;
}

// The extreme values of a s + b s^3 + c s^5 over 0 <= s <= u, and of b t + c t^2 over
// 0 <= t <= u^2.
double most_of_step(double a, double b, double c, double u) {
  double most = std::fabs(u * (a + u * u * (b + c * u * u)));
  // stationary where a + 3 b t + 5 c t^2 = 0, t = s^2
  double roots[2];
  int n = 0;
  if (c != 0.0) {
    const double disc = 9 * b * b - 20 * a * c;
    if (disc >= 0) {
      roots[n++] = (-3 * b + std::sqrt(disc)) / (10 * c);
      roots[n++] = (-3 * b - std::sqrt(disc)) / (10 * c);
    }
  } else if (b != 0.0) {
    roots[n++] = -a / (3 * b);
  }
  for (int k = 0; k < n; ++k)
    if (roots[k] > 0 && roots[k] < u * u) {
      const double s = std::sqrt(roots[k]);
      most = std::max(most, std::fabs(s * (a + roots[k] * (b + c * roots[k]))));
    }
  return most;
}
double most_of_poly(double b, double c, double u) {
  const double t = u * u;
  double most = std::fabs(t * (b + c * t));
  if (c != 0.0) {
    const double v = -b / (2 * c);
    if (v > 0 && v < t) most = std::max(most, std::fabs(v * (b + c * v)));
  }
  return most;
}

// The exponent e with bound 2^e in (2^14, 2^15.5]: below fp16's 65504 with room for rounding.
int32_t exponent_for(double bound) {
  int e = 0;
  std::frexp(std::max(bound, 1e-3) * 1.05, &e);     // bound 1.05 = f 2^e, 0.5 <= f < 1
  return 15 - e;
}

}  // namespace

bool zo::plan_ortho_steps(int32_t steps, const float* coeffs, OrthoStep* out) {
  const auto refused = [](const char* why) {
    set_last_error(why);
    return false;
  };
  if (steps < 1 || steps > kOrthoMaxSteps) return refused("zo_muon: need 1 <= steps <= 32");
  double u = 1.0;
  for (int32_t k = 0; k < steps; ++k) {
    OrthoStep s{};
    s.a = coeffs ? coeffs[3 * k] : (float)kMuonA;
    s.b = coeffs ? coeffs[3 * k + 1] : (float)kMuonB;
    s.c = coeffs ? coeffs[3 * k + 2] : (float)kMuonC;
    if (!std::isfinite(s.a) || !std::isfinite(s.b) || !std::isfinite(s.c))
      return refused("zo_muon: a coefficient is not finite");
    const double poly = most_of_poly(s.b, s.c, u), next = most_of_step(s.a, s.b, s.c, u);
    if (!(u * u < 4096.0) || !(poly < 4096.0) || !(next < 4096.0))
      return refused("zo_muon: with these coefficients the singular values can pass 2^12");
    s.ex = exponent_for(u);
    s.ea = exponent_for(u * u);
    s.eb = exponent_for(poly);
    s.ex_next = exponent_for(next);
    s.k = k;
    s.last = k + 1 == steps;
    out[k] = s;
    u = next;
  }
  return true;
}

struct zo_muon_ctx {
  int device = 0;
  cudaStream_t stream = nullptr;
  Layout plan;
  uint8_t* ws = nullptr;
  int32_t n_pairs = 0;
  int64_t launches = 0;
};

namespace {

zo_status run(zo_muon_ctx* c, const zo::OrthoUpdate& u, int32_t steps, const float* coeffs) {
  zo::OrthoStep st[zo::kOrthoMaxSteps];
  if (!zo::plan_ortho_steps(steps, coeffs, st)) return ZO_ERR_INVALID_ARG;
  const Layout& L = c->plan;
  const auto* mats = reinterpret_cast<const zo::OrthoMat*>(c->ws + L.mats_at);
  const auto* units = reinterpret_cast<const int4*>(c->ws + L.units_at);
  const auto* tiles = reinterpret_cast<const zo::OrthoTile*>(c->ws + L.tiles_at);
  auto* sums = reinterpret_cast<float*>(c->ws + L.sums_at);
  auto* slot_counters = reinterpret_cast<uint32_t*>(c->ws + L.slot_counter_at);
  const auto* firsts = reinterpret_cast<const int32_t*>(c->ws + L.first_at);
  const auto* maps = reinterpret_cast<const CUtensorMap*>(c->ws + L.maps_at);
  auto* status = reinterpret_cast<uint32_t*>(c->ws);
  auto* partial = reinterpret_cast<double*>(c->ws + L.partial_at);
  auto* counter = reinterpret_cast<uint32_t*>(c->ws + L.counter_at);
  auto* inverse = reinterpret_cast<float2*>(c->ws + L.inverse_at);
  const auto* which = reinterpret_cast<const int32_t*>(c->ws + L.small_at);
  for (const Small& g : L.small) {
    ZO_CUDA(g.rows ? zo::launch_ortho_mma(mats, which + g.first, g.n, g.rows, g.cluster, g.smem,
                                          st, steps, u, c->stream)
                   : zo::launch_ortho_small(mats, which + g.first, g.n, g.cluster, g.smem,
                                            st, steps, u, status, c->stream),
            "orthogonalisation: one-launch kernel");
    ++c->launches;
  }
  for (const Group& g : L.groups) {
    ZO_CUDA(zo::launch_ortho_momentum(mats, units + g.unit0, g.n_units, u, partial, counter,
                                      inverse, c->stream),
            "orthogonalisation: momentum kernel");
    ZO_CUDA(zo::launch_ortho_scale(mats, units + g.unit0, g.n_units, u, st[0].ex, inverse,
                                   c->stream),
            "orthogonalisation: scaling kernel");
    c->launches += 2;
    for (int32_t k = 0; k < steps; ++k)
      for (const zo::OrthoPhase phase : {zo::kOrthoGram, zo::kOrthoPoly, zo::kOrthoApply})
        for (int pr = 0; pr < 2; ++pr) {
          if (g.list[pr][phase] < 0) continue;
          const TileList& list = L.lists[g.list[pr][phase]];
          ZO_CUDA(zo::launch_ortho_product(mats, maps, tiles + list.tile0, firsts + list.first0,
                                           sums, slot_counters, pr != 0, list.narrow != 0,
                                           std::min(list.n, c->n_pairs), phase, st[k], u, status,
                                           c->stream),
                  "orthogonalisation: product kernel");
          ++c->launches;
        }
  }
  return ZO_OK;
}

}  // namespace

extern "C" {

int64_t zo_muon_workspace(const zo_muon_matrix* mats, int32_t n_mats) {
  try {
    Layout L;
    if (check_matrices(mats, n_mats) != ZO_OK || plan(mats, n_mats, &L) != ZO_OK) return 0;
    return L.bytes;
  } catch (const std::bad_alloc&) {
    refuse(ZO_ERR_NOMEM, "zo_muon_workspace: out of host memory");
    return 0;
  }
}

zo_status zo_muon_create(zo_muon_ctx** out, const zo_muon_matrix* mats, int32_t n_mats,
                         void* workspace, int64_t workspace_bytes, void* stream) {
  if (!out) return ZO_ERR_INVALID_ARG;
  *out = nullptr;
  try {
    zo_status st = check_matrices(mats, n_mats);
    if (st != ZO_OK) return st;
    std::unique_ptr<zo_muon_ctx> c(new zo_muon_ctx());
    st = plan(mats, n_mats, &c->plan);
    if (st != ZO_OK) return st;
    Layout& L = c->plan;
    if (!workspace || workspace_bytes < L.bytes)
      return refuse(ZO_ERR_INVALID_ARG,
                    "zo_muon_create: the workspace is missing or smaller than zo_muon_workspace");
    if (reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
      return refuse(ZO_ERR_ALIGN, "zo_muon_create: the workspace must be 256-byte aligned");
    int dev = 0, major = 0, minor = 0;
    ZO_CUDA(cudaGetDevice(&dev), "cudaGetDevice");
    ZO_CUDA(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev), "device");
    ZO_CUDA(cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev), "device");
    if (major != 10 || minor != 3)
      return refuse(ZO_ERR_CUDA, "this library is built for sm_103a (GB300) only");
    c->device = dev;
    c->stream = reinterpret_cast<cudaStream_t>(stream);
    c->ws = static_cast<uint8_t*>(workspace);
    uint8_t* buffers = c->ws + L.buffers_at;
    for (zo::OrthoMat& d : L.mats) {
      if (d.small) continue;
      const auto put = [&](uint16_t*& p) {
        p = reinterpret_cast<uint16_t*>(buffers + reinterpret_cast<int64_t>(p));
      };
      put(d.xh[0]);
      put(d.xh[1]);
      put(d.xl[0]);
      put(d.xl[1]);
      put(d.ah);
      put(d.bh);
      if (d.pairs) {
        put(d.al);
        put(d.bl);
      }
    }
    std::vector<CUtensorMap> maps((size_t)zo::kOrthoMaps * L.n_maps);
    for (const zo::OrthoMat& d : L.mats)
      if (!d.small && !encode_maps(d, &maps[(size_t)zo::kOrthoMaps * d.maps]))
        return refuse(ZO_ERR_CUDA, "zo_muon_create: cuTensorMapEncodeTiled rejected a descriptor");
    c->n_pairs = L.groups.empty() ? 0 : zo::ortho_max_pairs();
    if (!L.groups.empty() && c->n_pairs <= 0)
      return refuse(ZO_ERR_CUDA, "zo_muon_create: no cluster of the product kernel fits");
    c->n_pairs = std::min(c->n_pairs, zo::kOrthoMaxPairs);
    if (c->n_pairs > 0) deal_tiles(L, c->n_pairs);
    // one copy of the status word (0) and every table
    std::vector<uint8_t> image((size_t)L.tables_end, 0);
    std::memcpy(image.data() + L.mats_at, L.mats.data(), sizeof(zo::OrthoMat) * L.mats.size());
    if (!maps.empty())
      std::memcpy(image.data() + L.maps_at, maps.data(), sizeof(CUtensorMap) * maps.size());
    if (!L.small_list.empty())
      std::memcpy(image.data() + L.small_at, L.small_list.data(), sizeof(int32_t) * L.small_list.size());
    if (!L.units.empty()) std::memcpy(image.data() + L.units_at, L.units.data(), sizeof(int4) * L.units.size());
    if (!L.first.empty())
      std::memcpy(image.data() + L.first_at, L.first.data(), sizeof(int32_t) * L.first.size());
    if (!L.tiles.empty()) std::memcpy(image.data() + L.tiles_at, L.tiles.data(), sizeof(zo::OrthoTile) * L.tiles.size());
    ZO_CUDA(cudaMemcpyAsync(c->ws, image.data(), image.size(), cudaMemcpyHostToDevice, c->stream),
            "upload tables");
    // (a copy from pageable memory may be asynchronous where the GPU reads the host's page tables)
    ZO_CUDA(cudaStreamSynchronize(c->stream), "stream synchronize");
    L.mats.clear();
    L.units.clear();
    L.tiles.clear();
    *out = c.release();
    return ZO_OK;
  } catch (const std::bad_alloc&) {
    return refuse(ZO_ERR_NOMEM, "zo_muon_create: out of host memory");
  }
}

zo_status zo_muon_destroy(zo_muon_ctx* c) {
  if (!c) return ZO_OK;
  DeviceGuard guard(c->device);
  const cudaError_t e = cudaStreamSynchronize(c->stream);
  delete c;
  if (e != cudaSuccess) return cuda_fail(e, "zo_muon_destroy");
  return ZO_OK;
}

zo_status zo_orthogonalize(zo_muon_ctx* c, int32_t steps, const float* coeffs, float eps) {
  if (!c) return ZO_ERR_INVALID_ARG;
  if (!(eps >= 0.0f) || !std::isfinite(eps))
    return refuse(ZO_ERR_INVALID_ARG, "zo_orthogonalize: need a finite eps >= 0");
  DeviceGuard guard(c->device);
  zo::OrthoUpdate u{};
  u.eps = eps;
  try {
    return run(c, u, steps, coeffs);
  } catch (const std::bad_alloc&) {
    return refuse(ZO_ERR_NOMEM, "zo_orthogonalize: out of host memory");
  }
}

zo_status zo_muon_step(zo_muon_ctx* c, float momentum, int32_t nesterov, float lr,
                       float weight_decay, int32_t adjust, int32_t steps, const float* coeffs,
                       float eps) {
  if (!c) return ZO_ERR_INVALID_ARG;
  if (!(eps >= 0.0f) || !std::isfinite(eps) || !std::isfinite(lr) || !std::isfinite(weight_decay) ||
      !(momentum >= 0.0f && momentum < 1.0f))
    return refuse(ZO_ERR_INVALID_ARG,
                  "zo_muon_step: need finite scalars, eps >= 0 and momentum in [0, 1)");
  if (adjust < ZO_MUON_ADJUST_NONE || adjust > ZO_MUON_ADJUST_RMS)
    return refuse(ZO_ERR_INVALID_ARG, "zo_muon_step: unknown adjust");
  DeviceGuard guard(c->device);
  zo::OrthoUpdate u{};
  u.momentum = momentum;
  u.step = 1;
  u.nesterov = nesterov != 0;
  u.adjust = adjust;
  u.keep = (float)(1.0 - (double)lr * (double)weight_decay);
  u.lr = lr;
  u.eps = eps;
  try {
    return run(c, u, steps, coeffs);
  } catch (const std::bad_alloc&) {
    return refuse(ZO_ERR_NOMEM, "zo_muon_step: out of host memory");
  }
}

zo_status zo_muon_sync_status(zo_muon_ctx* c) {
  if (!c) return ZO_ERR_INVALID_ARG;
  DeviceGuard guard(c->device);
  uint32_t s = 0;
  ZO_CUDA(cudaMemcpyAsync(&s, c->ws, sizeof(s), cudaMemcpyDeviceToHost, c->stream), "read status");
  ZO_CUDA(cudaStreamSynchronize(c->stream), "stream synchronize");
  if (s != 0) {
    ZO_CUDA(cudaMemsetAsync(c->ws, 0, sizeof(uint32_t), c->stream), "clear status");
    // launches that gave up may have left counters of finished units and parts behind
    ZO_CUDA(cudaMemsetAsync(c->ws + c->plan.counter_at, 0,
                            (size_t)(c->plan.tables_end - c->plan.counter_at), c->stream),
            "clear counters");
    ZO_CUDA(cudaStreamSynchronize(c->stream), "stream synchronize");
    return refuse(ZO_ERR_TIMEOUT, "a device-side wait ran out");
  }
  return ZO_OK;
}

int64_t zo_muon_launches(const zo_muon_ctx* c) { return c ? c->launches : 0; }

}  // extern "C"
