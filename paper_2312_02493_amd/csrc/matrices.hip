// Host side of the entry points on matrices of a flat vector: argument checks, layout of the iterates' memory,
// tables of tiles, launches.

#include "artopk.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "host_common.h"
#include "matrices_kernels.h"

using namespace artopk;

namespace {

constexpr int kTileClasses = 5;
constexpr int kTileOf[kTileClasses] = {64, 128, 192, 256, 64};  // the last one deep
constexpr int32_t kMaxMatrices = 65535;
constexpr int32_t kMaxSide = 65536;
constexpr float kUsual[3] = {3.4445f, -4.7750f, 2.0315f};

// A list of blocks' work in the tables.
struct Span {
  size_t at = 0;  // entries from the table's start
  int count = 0;
};

// A product's blocks, and the tile they take.
struct Product {
  Span tiles;
  int cls = 0;
};

// The matrices whose products are of one kind, and what their launches work on.
struct Group {
  int parts = 1;             // of an operand
  int first = 0, count = 0;  // in the table of matrices
  Span begin;
  Product gram, square, apply;
  Span join;  // the tiles of Gram matrices whose sums are cut
  bool pairs = false;    // two steps at once
  size_t small_lds = 0;  // of every matrix on one compute unit, in one launch; 0: not so
  int64_t partial = 0;   // where the sums of its Gram products' shares lie, in floats
};

// What creation works out on the host: where everything lies, and the tables.
struct MatPlan {
  std::vector<MatDesc> mats;  // group by group
  std::vector<MatChunk> chunks;
  std::vector<MatTile> tiles;
  Group groups[2];
  int ngroups = 0;
  int64_t halves = 0;  // of the iterates' memory
  int64_t partial = 0;  // floats of the sums of shares
  int32_t sums = 0;
};

// What a product's block costs, in us, by tile class: alone on its compute unit (`fixed` and `alone` for each 64 of the
// summed index), and as the chip's time for one of very many blocks (`store` and `among` for each 64).  Fitted to products
// timed one kind at a time, tile by tile: 4096 x 4096 (64 of 64), sixteen matrices of 1280 x 1280 and eight of 1280 x 5120
// (20 of 64 where m is summed over), and the long sums of one 1280 x 5120 by itself.  What the rule has to get right (us,
// HALF, tiles of 64 / 128 / 192 / 256): X X^T of 4096 x 4096 130 / 100 / 75 / 89, Q X of it 227 / 131 / 154 / 110, X X^T of
// four 512 x 4608 18 / 44 / 54 / 87, Q X of the sixteen and eight 346 / 243 / 272 / 206.
struct TileCost {
  double fixed, alone, store, among;
  int slots;  // blocks that the chip holds
};
constexpr TileCost kNever = {1e9, 1e9, 1e9, 1e9, 256};  // (one part is fed as fast without, and Q X has two stages)
constexpr TileCost kCost[2][2][kTileClasses] = {  // [Q X][two parts]
    {{{3.0, 0.20, 0.0043, 0.00083, 512},
      {4.0, 0.63, 0.0258, 0.0017, 512},
      {5.0, 0.84, 0.0325, 0.0044, 256},
      {6.0, 1.28, 0.0890, 0.00575, 256},
      kNever},
     {{3.0, 0.60, 0.0110, 0.0018, 512},
      {4.0, 1.60, 0.0470, 0.0047, 512},
      {5.0, 1.93, 0.0820, 0.0100, 256},
      {6.0, 3.80, 0.1890, 0.0160, 256},
      {3.0, 0.38, 0.0110, 0.0018, 256}}},
    {{{3.0, 0.25, 0.0020, 0.00085, 1024},
      {4.0, 0.65, 0.0155, 0.00186, 512},
      {5.0, 0.90, 0.0330, 0.0049, 256},
      {6.0, 1.28, 0.0600, 0.0060, 256},
      kNever},
     {{3.0, 0.55, 0.0080, 0.0017, 512},
      {4.0, 1.60, 0.0400, 0.0047, 512},
      {5.0, 2.20, 0.0920, 0.0117, 256},
      {6.0, 3.60, 0.1100, 0.0168, 256},
      kNever}}};
// Shares that meet in memory: a launch, the shares of one tile one after the other, and their bytes (36 tiles of 64 x 64 in 9
// shares each 4.6, 10 of 128 x 128 in 18 9.1, one of 64 x 64 in 32 11.1).
constexpr double kJoinLaunch = 3.5, kJoinShare = 0.22, kJoinBytes = 1.0 / 2.5e6;

int tiles_of(int side, int tile) { return (side + tile - 1) / tile; }

// One kind of product over all matrices.
struct ProductKind {
  bool symmetric, long_sum;  // the result is, and n is summed over, not m
};

int64_t product_tiles(const MatDesc& d, const ProductKind& k, int tile) {
  const int64_t a = tiles_of(d.mp, tile), b = tiles_of(d.np, tile);
  return k.symmetric ? a * (a + 1) / 2 : a * b;
}

int product_shares(const MatDesc& d, const ProductKind& k, int each) {  // `each`: 64s of the summed index a share, 0: whole
  const int units = (k.long_sum ? d.np : d.mp) / 64;
  return each == 0 ? 1 : std::max(1, (units + each / 2) / each);
}

double product_cost(const std::vector<MatDesc>& mats, const ProductKind& k, int parts, int cls, int each) {
  const TileCost& c = kCost[k.symmetric ? 0 : 1][parts - 1][cls];
  double chip = 0.0, blocks = 0.0, units_in_all = 0.0, longest = 0.0, joined = 0.0;
  int most_shares = 1;
  for (const MatDesc& d : mats) {
    const double units = (k.long_sum ? d.np : d.mp) / 64;
    const int shares = product_shares(d, k, each);
    const double tiles = (double)product_tiles(d, k, kTileOf[cls]);
    chip += tiles * (shares * c.store + units * c.among);
    blocks += tiles * shares;
    units_in_all += tiles * units;
    longest = std::max(longest, std::ceil(units / shares));
    if (shares > 1) joined += tiles * shares * kTileOf[cls] * kTileOf[cls] * 8.0;
    most_shares = std::max(most_shares, shares);
  }
  // whole rounds of blocks at the chip's rate, and a last one that takes a block's own time at least, or half of that where
  // two blocks share a compute unit, since they do not end together
  const double rounds = std::floor(blocks / c.slots), rest = blocks - rounds * c.slots;
  double cost = chip * (rounds * c.slots / blocks);
  if (rest > 0.0)
    cost += std::max((c.fixed + c.alone * (units_in_all / blocks)) * (rounds > 0.0 ? 256.0 / c.slots : 1.0), chip * (rest / blocks));
  cost = std::max(cost, c.fixed + c.alone * longest);
  if (most_shares > 1) cost += kJoinLaunch + kJoinShare * most_shares + kJoinBytes * joined;
  return cost;
}

// The tile and, for the Gram products, the length of a share that cost least.
double choose_product(const std::vector<MatDesc>& mats, const ProductKind& k, int parts, Product* p, int* each_out) {
  double best = 1e300;
  for (int cls = 0; cls < kTileClasses; ++cls)
    for (int each : {0, 64, 32, 16, 8}) {
      if (each && (!k.long_sum || kTileOf[cls] > 128)) continue;
      const double cost = product_cost(mats, k, parts, cls, each);
      if (cost < best) {
        best = cost;
        p->cls = cls;
        if (each_out) *each_out = each;
      }
    }
  return best;
}

// What a step of small matrices costs, in us, by the 32 x 32 x 32 products of the largest (measured, five steps and some 6 us
// besides, HALF / SPLIT: 64 x 64 15.6 / 20, 64 x 128 19.4 / 25, 96 x 160 32 / 43, 128 x 128 38 / too large; the same in
// launches of their own 46 / 56, 51 / 63, 62 / 82, 60 / 76; 600 of 64 x 64 34 / 62 and 102 / 153).
constexpr int64_t kSmallLds = 156 * 1024;
double small_cost(const std::vector<MatDesc>& mats, int parts, size_t lds) {
  double longest = 0.0;
  for (const MatDesc& d : mats) {
    const double m = small_pad(d.m) / 32, n = small_pad(d.n) / 32;
    const double blocks = m * m * (n + m) + m * n * m;
    longest = std::max(longest, parts == 2 ? 1.8 + 0.048 * blocks : 1.2 + 0.032 * blocks);
  }
  const int64_t together = 256 * std::max<int64_t>(1, std::min<int64_t>(2, 160 * 1024 / (int64_t)lds));
  return longest * std::ceil((double)mats.size() / (double)together);
}

// The blocks of one kind of product, in the order in which they start.  Blocks go to the chip's eight dies in turn, and
// each die has a cache of its own: the tiles of all matrices with equally long sums are cut into eight runs of neighbours,
// one for each die, and the longest sums come first.  (Every matrix cut into eight instead: Q X of sixteen 1280 x 1280
// and eight 1280 x 5120 234 us, so 228.)  `slots` counts the places of shares' sums.
void list_product(MatPlan* plan, const std::vector<MatDesc>& mats, const ProductKind& k, Product* p, int each, int64_t* slots) {
  const int tile = kTileOf[p->cls];
  std::vector<int> order(mats.size());
  for (size_t i = 0; i < order.size(); ++i) order[i] = (int)i;
  auto units = [&](int i) {
    const MatDesc& d = mats[i];
    return (k.long_sum ? d.np : d.mp) / 64 / product_shares(d, k, each);
  };
  std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return units(a) > units(b); });
  std::vector<MatTile> die[8];
  std::vector<MatTile> own;
  int first = 0;
  for (size_t o = 0; o < order.size();) {
    own.clear();
    const int here = units(order[o]);
    for (; o < order.size() && units(order[o]) == here; ++o) {
      const int i = order[o];
      const MatDesc& d = mats[i];
      const int a = tiles_of(d.mp, tile), b = tiles_of(d.np, tile);
      const int shares = product_shares(d, k, each);
      constexpr int kBand = 4;  // rows of tiles taken together
      for (int a0 = 0; a0 < a; a0 += kBand)
        for (int y = 0; y < (k.symmetric ? std::min(a, a0 + kBand) : b); ++y)
          for (int x = a0; x < std::min(a, a0 + kBand); ++x) {
            if (k.symmetric && y > x) continue;
            MatTile t = {};
            t.d = d;
            t.i = (uint16_t)x;
            t.j = (uint16_t)y;
            t.shares = (uint16_t)shares;
            t.slot = (uint32_t)*slots;
            if (shares > 1) *slots += shares;
            for (int s = 0; s < shares; ++s) {
              t.share = (uint16_t)s;
              own.push_back(t);
            }
          }
    }
    const int64_t total = (int64_t)own.size(), per = total / 8, more = total % 8;
    int64_t at = 0;
    for (int x = 0; x < 8; ++x) {
      const int64_t count = per + (x < more);
      std::vector<MatTile>& to = die[(first + x) % 8];
      to.insert(to.end(), own.begin() + at, own.begin() + at + count);
      at += count;
    }
    first = (int)((first + more) % 8);
  }
  p->tiles.at = plan->tiles.size();
  size_t longest = 0;
  for (const auto& v : die) longest = std::max(longest, v.size());
  for (size_t r = 0; r < longest; ++r)
    for (const auto& v : die)
      if (r < v.size()) plan->tiles.push_back(v[r]);
  p->tiles.count = (int)(plan->tiles.size() - p->tiles.at);
}

// Threads of a product's block.
int product_threads(int parts, int cls) {
  constexpr int kThreads[2][kTileClasses] = {
      {ProductShape<64, 1>::kThreads, ProductShape<128, 1>::kThreads, ProductShape<192, 1>::kThreads, ProductShape<256, 1>::kThreads,
       ProductShape<64, 1>::kThreads},
      {ProductShape<64, 2>::kThreads, ProductShape<128, 2>::kThreads, ProductShape<192, 2>::kThreads, ProductShape<256, 2>::kThreads,
       ProductShape<64 + kDeep, 2>::kThreads}};
  return kThreads[parts - 1][cls];
}

// Whether a launch holds all blocks of each kind: beyond 2^32 threads it would wrap round, without an error.
bool launches_hold(const std::vector<MatDesc>& mats, const Group& g, const ProductKind& gram, const ProductKind& square,
                   const ProductKind& apply, int each) {
  int64_t begin = 0, of_gram = 0, of_square = 0, of_apply = 0;
  for (const MatDesc& d : mats) {
    begin += (int64_t)(d.mp / 64) * (d.np / 64);
    of_gram += product_tiles(d, gram, kTileOf[g.gram.cls]) * product_shares(d, gram, each);
    of_square += product_tiles(d, square, kTileOf[g.square.cls]);
    of_apply += product_tiles(d, apply, kTileOf[g.apply.cls]);
  }
  return std::max({begin * 256, of_gram * product_threads(g.parts, g.gram.cls), of_square * product_threads(g.parts, g.square.cls),
                   of_apply * product_threads(g.parts, g.apply.cls)}) < (1ll << 32);
}

// Places of a group's matrices in the iterates' memory, and its lists of blocks; its matrices are those of the table from
// group->first on.  False where they are too many for a launch.
bool plan_group(MatPlan* plan, Group* g) {
  const std::vector<MatDesc> bare(plan->mats.begin() + g->first, plan->mats.begin() + g->first + g->count);
  const ProductKind gram = {true, true}, square = {true, false}, apply = {false, false};
  int each = 0;
  const double cost_gram = choose_product(bare, gram, g->parts, &g->gram, &each);
  const double cost_square = choose_product(bare, square, g->parts, &g->square, nullptr);
  const double cost_apply = choose_product(bare, apply, g->parts, &g->apply, nullptr);
  const double cost = cost_gram + cost_square + cost_apply;
  g->pairs = cost_gram + 5.0 * cost_square + cost_apply < 0.9 * 2.0 * cost;  // (not for a little: it rounds more)
  bool small = true;
  size_t lds = 0;
  for (const MatDesc& d : bare) {
    const int64_t bytes = 2 * small_halves(d.m, d.n, g->parts);
    small &= bytes <= kSmallLds && (int64_t)small_pad(d.m) * small_pad(d.n) <= kSmallElems;
    lds = std::max(lds, (size_t)bytes);
  }
  if (small && small_cost(bare, g->parts, lds) < cost) {
    g->small_lds = lds;
    return true;
  }
  if (!launches_hold(bare, *g, gram, square, apply, each)) return false;
  for (int i = g->first; i < g->first + g->count; ++i) {
    MatDesc& d = plan->mats[i];
    const int64_t mn = (int64_t)d.mp * d.np * g->parts, mm = (int64_t)d.mp * d.mp * g->parts;
    d.x[0] = plan->halves;
    d.x[1] = d.x[0] + mn;
    for (int k = 0; k < 3; ++k) d.sq[k] = d.x[1] + mn + k * mm;
    plan->halves = d.sq[2] + mm;
  }
  const std::vector<MatDesc> mats(plan->mats.begin() + g->first, plan->mats.begin() + g->first + g->count);
  g->begin.at = plan->tiles.size();
  for (const MatDesc& d : mats)
    for (int a = 0; a < d.mp / 64; ++a)
      for (int b = 0; b < d.np / 64; ++b) plan->tiles.push_back(MatTile{d, (uint16_t)a, (uint16_t)b, 0, 1, 0});
  g->begin.count = (int)(plan->tiles.size() - g->begin.at);
  int64_t slots = 0;
  list_product(plan, mats, gram, &g->gram, each, &slots);
  g->join.at = plan->tiles.size();
  for (int i = 0; i < g->gram.tiles.count; ++i) {
    const MatTile t = plan->tiles[g->gram.tiles.at + i];
    if (t.shares > 1 && t.share == 0) plan->tiles.push_back(t);
  }
  g->join.count = (int)(plan->tiles.size() - g->join.at);
  g->partial = plan->partial;
  plan->partial += slots * kTileOf[g->gram.cls] * kTileOf[g->gram.cls];
  list_product(plan, mats, square, &g->square, 0, &slots);
  list_product(plan, mats, apply, &g->apply, 0, &slots);
  return true;
}

// `parts`: of each matrix's operands.  ARTOPK_OK, or ARTOPK_EINVAL with the reason in `err`.  Throws std::bad_alloc.
int make_plan(const artopk_matrix* mats, int32_t count, int64_t n, int32_t type, const std::vector<int>& parts, MatPlan* plan,
              char* err) {
  if (n < 1 || n >= (1ll << 31)) return fail_text(err, ARTOPK_EINVAL, "n=%lld outside [1, 2^31)", (long long)n);
  if (type != ARTOPK_G_F32 && type != ARTOPK_G_BF16 && type != ARTOPK_G_F16)
    return fail_text(err, ARTOPK_EINVAL, "unknown element type %d", type);
  std::vector<int32_t> order(count);
  for (int i = 0; i < count; ++i) {
    const artopk_matrix& m = mats[i];
    if (m.rows < 1 || m.rows > kMaxSide || m.cols < 1 || m.cols > kMaxSide)
      return fail_text(err, ARTOPK_EINVAL, "matrix %d is %d x %d; sides have to be in [1, %d]", i, m.rows, m.cols, kMaxSide);
    const int64_t size = (int64_t)m.rows * m.cols;
    if (m.offset < 0 || size > n || m.offset > n - size)
      return fail_text(err, ARTOPK_EINVAL, "matrix %d does not lie within the vector", i);
    if (!std::isfinite(m.scale)) return fail_text(err, ARTOPK_EINVAL, "matrix %d's scale is not finite", i);
    order[i] = i;
  }
  std::sort(order.begin(), order.end(), [&](int a, int b) { return mats[a].offset < mats[b].offset; });
  for (int i = 1; i < count; ++i) {
    const artopk_matrix& m = mats[order[i - 1]];
    if (m.offset + (int64_t)m.rows * m.cols > mats[order[i]].offset)
      return fail_text(err, ARTOPK_EINVAL, "matrices %d and %d overlap", order[i - 1], order[i]);
  }

  std::vector<int> place(count);  // of a matrix in the table
  for (int kind = 1; kind <= 2; ++kind) {
    Group g;
    g.parts = kind;
    g.first = (int)plan->mats.size();
    for (int i = 0; i < count; ++i) {
      if (parts[i] != kind) continue;
      const artopk_matrix& m = mats[i];
      MatDesc d = {};
      d.at = m.offset;
      d.tall = m.rows > m.cols;
      d.m = std::min(m.rows, m.cols);
      d.n = std::max(m.rows, m.cols);
      d.scale = m.scale;
      d.mp = (d.m + 63) / 64 * 64;
      d.np = (d.n + 63) / 64 * 64;
      place[i] = d.id = (int)plan->mats.size();
      plan->mats.push_back(d);
    }
    g.count = (int)plan->mats.size() - g.first;
    if (g.count) plan->groups[plan->ngroups++] = g;
  }

  // pieces of the vector, those of a matrix side by side; at most 512 a matrix, so that every block that needs its norm
  // can add them up
  int64_t done = 0;
  auto loose = [&](int64_t end) {
    for (; done < end; done += 16384) plan->chunks.push_back(MatChunk{done, std::min(end, done + 16384), -1, 0});
    done = end;
  };
  for (int k = 0; k < count; ++k) {
    const int i = place[order[k]];
    MatDesc& d = plan->mats[i];
    loose(d.at);
    const int64_t size = (int64_t)d.m * d.n, end = d.at + size;
    int64_t each = (size + 511) / 512;
    each = (std::max<int64_t>(each, 8192) + 63) / 64 * 64;
    d.part = plan->sums;
    for (; done < end; done += each) plan->chunks.push_back(MatChunk{done, std::min(end, done + each), i, plan->sums++});
    done = end;
    d.parts = plan->sums - d.part;
  }
  loose(n);

  for (int i = 0; i < plan->ngroups; ++i)
    if (!plan_group(plan, &plan->groups[i]))
      return fail_text(err, ARTOPK_EINVAL, "the matrices are more tiles of 64 x 64 than a launch holds");
  return ARTOPK_OK;
}

// What an entry point launches on, with its places in the handle's memory.
struct Route {
  Group groups[2];
  int ngroups = 0;
  int nchunks = 0;
  const MatDesc* mats = nullptr;
  const MatChunk* chunks = nullptr;
  const MatTile* tiles = nullptr;
  double* sums = nullptr;
  float* sizes = nullptr;  // of every matrix, s with ||X_0|| < 2^s
  float* partial = nullptr;
};

// The parts of each matrix's operands, for the entry point that gives a matrix itself or the one that steps weights by it.
// float16's own rounding is 0.2e-3, and HALF would show in it: it takes SPLIT always.  bfloat16's is 1.7e-3.  Against 64 bits
// HALF is 0.9e-3 to 2.3e-3 off from 64 rows on (the worst of Gaussian, low-rank and graded matrices; 3.6e-3 where all singular
// values are the same, so that all roundings go the same way), and of fewer rows up to 9e-3 (4 x 4096), 7e-3 (48 x 4096), 4e-3
// (24 x 384).  So matrices of fewer than 64 rows take SPLIT, whatever lies beside them in the vector: it costs little there,
// where launches and latency count (a second group of launches, 20 us for 16 in one launch).  artopk_orthogonalize, whose
// result is nothing but X, takes it for all matrices where most of the result (its squared norm is its matrices' rows) is of at
// most 256 rows (24 of 256 x 1024 195 us for 120); weights are a sum, of which X is usually the smaller part.
constexpr int32_t kFewRows = 256, kSplitBelow = 64;
std::vector<int> parts_for(const artopk_matrix* mats, int32_t count, int32_t type, int32_t products, bool weights) {
  if (products != ARTOPK_PRODUCTS_DEFAULT) return std::vector<int>(count, products == ARTOPK_PRODUCTS_SPLIT ? 2 : 1);
  if (type != ARTOPK_G_BF16) return std::vector<int>(count, 2);
  std::vector<int> parts(count);
  int64_t all = 0, few = 0;
  for (int32_t i = 0; i < count; ++i) {
    const int32_t rows = std::min(mats[i].rows, mats[i].cols);
    parts[i] = rows < kSplitBelow ? 2 : 1;
    all += rows;
    if (rows <= kFewRows) few += rows;
  }
  if (!weights && 2 * few > all) parts.assign(count, 2);
  return parts;
}

// Both entry points' plans, and the places of their tables; the iterates' memory is used by one call at a time.
struct Plans {
  MatPlan plan[2];
  int count = 1;  // 1: they are the same
  size_t o_mats[2], o_chunks[2], o_tiles[2], o_sums[2], o_sizes[2], o_partial[2], o_mem = 0, total = 0;
};

int make_plans(const artopk_matrix* mats, int32_t count, int64_t n, int32_t type, int32_t products, Plans* p, char* err) {
  if (!mats) return fail_text(err, ARTOPK_EINVAL, "mats is NULL");
  if (count < 1 || count > kMaxMatrices) return fail_text(err, ARTOPK_EINVAL, "count=%d outside [1, %d]", count, kMaxMatrices);
  if (products != ARTOPK_PRODUCTS_HALF && products != ARTOPK_PRODUCTS_SPLIT && products != ARTOPK_PRODUCTS_DEFAULT)
    return fail_text(err, ARTOPK_EINVAL, "unknown kind of products %d", products);
  const std::vector<int> own = parts_for(mats, count, type, products, false), weights = parts_for(mats, count, type, products, true);
  p->count = own == weights ? 1 : 2;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at = align_up(at + bytes, 256);
    return o;
  };
  int64_t halves = 0;
  for (int i = 0; i < p->count; ++i) {
    MatPlan& plan = p->plan[i];
    const int rc = make_plan(mats, count, n, type, i == 0 ? own : weights, &plan, err);
    if (rc) return rc;
    p->o_mats[i] = take(plan.mats.size() * sizeof(MatDesc));
    p->o_chunks[i] = take(plan.chunks.size() * sizeof(MatChunk));
    p->o_tiles[i] = take(plan.tiles.size() * sizeof(MatTile));
    p->o_sums[i] = take((size_t)plan.sums * sizeof(double));
    p->o_sizes[i] = take(plan.mats.size() * sizeof(float));
    p->o_partial[i] = take((size_t)plan.partial * sizeof(float));
    halves = std::max(halves, plan.halves);
  }
  p->o_mem = take((size_t)halves * 2);
  p->total = at;
  return ARTOPK_OK;
}

}  // namespace

struct artopk_matrices {
  hipStream_t stream = nullptr;
  int64_t n = 0;
  int32_t type = 0;
  Route own, weights;  // of artopk_orthogonalize and of artopk_muon_step
  char* slab = nullptr;
  _Float16* mem = nullptr;
  char err[kErrText] = {0};
};

namespace {

#define MAT_TRY(h, expr)                                                                                       \
  do {                                                                                                         \
    hipError_t e_ = (expr);                                                                                    \
    if (e_ != hipSuccess)                                                                                      \
      return fail_text((h)->err, ARTOPK_EHIP, "%s failed: %s (%s:%d)", #expr, hipGetErrorString(e_), __FILE__, \
                       __LINE__);                                                                              \
  } while (0)

struct Steps {
  int count = 0;
  float co[ARTOPK_MAX_POLAR_STEPS][3];
  double factor[ARTOPK_MAX_POLAR_STEPS];  // the largest |a + b s^2 + c s^4|
  float grown[ARTOPK_MAX_POLAR_STEPS + 1];  // log2 of the factors before each step and behind the last, multiplied
};
constexpr double kMostFactor = 15.0;

// The coefficients of every step, or ARTOPK_EINVAL where the iterates could leave the operands' range: with singular
// values of at most `most` before a step, the largest of |s (a + b s^2 + c s^4)| and of |a + b s^2 + c s^4| over
// [0, most] lie at an end or where a derivative is zero.
int take_coefficients(artopk_matrices* h, int32_t steps, const float* coefficients, Steps* st) {
  if (steps < 0 || steps > ARTOPK_MAX_POLAR_STEPS)
    return fail_text(h->err, ARTOPK_EINVAL, "steps=%d outside [0, %d]", steps, ARTOPK_MAX_POLAR_STEPS);
  double most = 1.0, grown = 0.0;
  st->count = steps;
  st->grown[0] = 0.0f;
  for (int k = 0; k < steps; ++k) {
    float* out = st->co[k];
    for (int i = 0; i < 3; ++i) out[i] = coefficients ? coefficients[3 * k + i] : kUsual[i];
    const double a = out[0], b = out[1], c = out[2];
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c))
      return fail_text(h->err, ARTOPK_EINVAL, "coefficients of step %d are not finite", k);
    double next = 0.0, factor = std::fabs(a);
    auto look = [&](double y) {  // y = s^2
      if (!(y >= 0.0 && y <= most * most)) return;
      const double q = a + y * (b + c * y);
      factor = std::max(factor, std::fabs(q));
      next = std::max(next, std::sqrt(y) * std::fabs(q));
    };
    look(most * most);
    if (c != 0.0) {
      look(-b / (2.0 * c));
      const double disc = 9.0 * b * b - 20.0 * a * c;  // of a + 3 b y + 5 c y^2
      if (disc >= 0.0) {
        look((-3.0 * b + std::sqrt(disc)) / (10.0 * c));
        look((-3.0 * b - std::sqrt(disc)) / (10.0 * c));
      }
    }
    if (b != 0.0) look(-a / (3.0 * b));  // (c = 0; an extra point otherwise)
    st->factor[k] = factor;
    grown += std::log2(factor);  // (minus infinity where nothing is left)
    st->grown[k + 1] = (float)grown;
    if (next > 2.0 || factor > kMostFactor)
      return fail_text(h->err, ARTOPK_EINVAL,
                       "step %d would take singular values up to %.4g to %.4g, with a factor of %.4g; at most 2 and 15 are taken", k,
                       most, next, factor);
    most = std::max(next, 1e-30);
  }
  return ARTOPK_OK;
}

template <int TILE, int PARTS, int MODE>
void product(const artopk_matrices* h, const Route& r, const Group& g, const Span& s, const ProductArgs& a, const FinishArgs& f) {
  k_mat_product<TILE, PARTS, MODE><<<s.count, ProductShape<TILE, PARTS>::kThreads, 0, h->stream>>>(r.tiles + s.at, h->mem, a, f,
                                                                                                  r.partial + g.partial, r.sizes);
}

template <int PARTS, int MODE>
void product(const artopk_matrices* h, const Route& r, const Group& g, const Product& p, const ProductArgs& a, const FinishArgs& f) {
  switch (p.cls) {
    case 0: return product<64, PARTS, MODE>(h, r, g, p.tiles, a, f);
    case 1: return product<128, PARTS, MODE>(h, r, g, p.tiles, a, f);
    case 2: return product<192, PARTS, MODE>(h, r, g, p.tiles, a, f);
    case 3: return product<256, PARTS, MODE>(h, r, g, p.tiles, a, f);
    default: return product<64 + (PARTS == 2 ? kDeep : 0), PARTS, MODE>(h, r, g, p.tiles, a, f);
  }
}

template <int TILE, int PARTS>
void join_shares(const artopk_matrices* h, const Route& r, const Group& g) {
  k_mat_join<TILE, PARTS><<<dim3(g.join.count, 2), ProductShape<TILE, PARTS>::kThreads, 0, h->stream>>>(
      r.tiles + g.join.at, h->mem, r.partial + g.partial);
}

// All steps of a group's matrices.
template <int PARTS, class From>
void polar(const artopk_matrices* h, const Route& r, const Group& g, From from, const Steps& st, float eps, const FinishArgs& f) {
  if (g.small_lds) {
    PolarSteps ps = {};
    ps.steps = st.count;
    memcpy(ps.co, st.co, sizeof(float) * 3 * st.count);
    memcpy(ps.grown, st.grown, sizeof(float) * st.count);
    k_mat_small<PARTS, From><<<g.count, kSmallThreads, g.small_lds, h->stream>>>(from, r.mats + g.first, ps, eps, f);
    return;
  }
  k_mat_begin<PARTS, From><<<g.begin.count, 256, 0, h->stream>>>(from, r.tiles + g.begin.at, r.sums, eps, h->mem, r.sizes);
  int x = 0;  // which X
  auto square = [&](int k, int in, int out) {
    product<PARTS, kSquare>(h, r, g, g.square, ProductArgs{x, in, in, out, st.co[k][0], st.co[k][1], st.co[k][2], st.grown[k], 0}, f);
  };
  auto times = [&](int in, int in2, int out, float grown, float then) {
    product<PARTS, kTimes>(h, r, g, g.square, ProductArgs{x, in, in2, out, 0, 0, 0, grown, then}, f);
  };
  for (int k = 0; k < st.count;) {
    const float grown = st.grown[k];
    product<PARTS, kGram>(h, r, g, g.gram, ProductArgs{x, 0, 0, 0, 0, 0, 0, 0, 0}, f);
    if (g.join.count) kTileOf[g.gram.cls] == 64 ? join_shares<64, PARTS>(h, r, g) : join_shares<128, PARTS>(h, r, g);
    square(k, 0, 1);
    int q = 1;
    if (g.pairs && k + 1 < st.count && st.factor[k] * st.factor[k + 1] <= kMostFactor) {
      times(1, 0, 2, 0, 0);                    // Q_1 A_0, as large as A_0 is stored
      times(2, 1, 0, grown, st.grown[k + 1]);  // A_1
      square(k + 1, 0, 2);                     // Q_2
      times(2, 1, 0, 0, 0);                    // Q_2 Q_1
      q = 0;
      ++k;
    }
    ++k;
    const ProductArgs a = {x, q, 0, 0, 0, 0, 0, grown, st.grown[k]};
    if (k < st.count)
      product<PARTS, kApply>(h, r, g, g.apply, a, f);
    else
      product<PARTS, kFinal>(h, r, g, g.apply, a, f);
    x ^= 1;
  }
}

// What the squares' or the momentum's launch leaves to do.
template <class From>
void polar(const artopk_matrices* h, const Route& r, From from, const Steps& st, float eps, const FinishArgs& f) {
  if (st.count == 0) {
    k_mat_scaled<From><<<r.nchunks, 256, 0, h->stream>>>(from, r.mats, r.chunks, r.sums, eps, f);
    return;
  }
  for (int i = 0; i < r.ngroups; ++i) {
    const Group& g = r.groups[i];
    if (g.parts == 2)
      polar<2>(h, r, g, from, st, eps, f);
    else
      polar<1>(h, r, g, from, st, eps, f);
  }
}

// Calls f with a null pointer of the handle's element type.
template <class F>
void with_type(int32_t type, F&& f) {
  if (type == ARTOPK_G_F32) f((float*)nullptr);
  else if (type == ARTOPK_G_BF16) f((__bf16*)nullptr);
  else f((_Float16*)nullptr);
}

size_t elem_size(int32_t type) { return type == ARTOPK_G_F32 ? 4 : 2; }

int check_vector(artopk_matrices* h, const char* name, const void* p, size_t size) {
  if (!p) return fail_text(h->err, ARTOPK_EINVAL, "%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(p) % size) return fail_text(h->err, ARTOPK_EINVAL, "%s is not aligned to its elements", name);
  return ARTOPK_OK;
}

int check_eps(artopk_matrices* h, float eps) {
  if (!(eps > 0.0f) || !std::isfinite(eps)) return fail_text(h->err, ARTOPK_EINVAL, "eps has to be positive and finite");
  return ARTOPK_OK;
}

// Lets the kernels of small matrices have the handle's LDS.
template <int PARTS>
hipError_t allow_small(const artopk_matrices* h) {
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_mat_small<PARTS, FromMomentum>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                     (int)kSmallLds);
  with_type(h->type, [&](auto* tag) {
    using T = std::remove_pointer_t<decltype(tag)>;
    if (e == hipSuccess)
      e = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_mat_small<PARTS, FromVector<T>>), hipFuncAttributeMaxDynamicSharedMemorySize,
                              (int)kSmallLds);
  });
  return e;
}

}  // namespace

int64_t artopk_matrices_scratch_bytes(const artopk_matrix* mats, int32_t count, int64_t n, int32_t type, int32_t products) {
  try {
    Plans plans;
    if (make_plans(mats, count, n, type, products, &plans, g_noctx_err)) return -1;
    return (int64_t)plans.total;
  } catch (const std::exception&) {
    return -1;
  }
}

int artopk_matrices_info(const artopk_matrix* mats, int32_t count, int64_t n, int32_t type, int32_t products, int32_t weights,
                         int32_t* info_out, int32_t info_count) {
  if (!info_out || info_count < ARTOPK_MATRICES_INFO)
    return fail_text(g_noctx_err, ARTOPK_EINVAL, "info_out has fewer than %d places", ARTOPK_MATRICES_INFO);
  try {
    Plans plans;
    const int rc = make_plans(mats, count, n, type, products, &plans, g_noctx_err);
    if (rc) return rc;
    const MatPlan& plan = plans.plan[weights && plans.count == 2];
    int32_t* o = info_out;
    *o++ = plan.ngroups;
    for (int i = 0; i < 2; ++i) {
      const Group g = i < plan.ngroups ? plan.groups[i] : Group();
      const bool tiles = i < plan.ngroups && !g.small_lds;
      *o++ = g.count;
      *o++ = i < plan.ngroups ? g.parts : 0;
      *o++ = g.small_lds != 0;
      *o++ = tiles && g.pairs;
      *o++ = tiles ? kTileOf[g.gram.cls] : 0;
      *o++ = tiles ? kTileOf[g.square.cls] : 0;
      *o++ = tiles ? kTileOf[g.apply.cls] : 0;
      *o++ = g.join.count;
    }
    return ARTOPK_OK;
  } catch (const std::exception&) {
    return fail_text(g_noctx_err, ARTOPK_ENOMEM, "out of host memory");
  }
}

int artopk_matrices_create(artopk_matrices** out, const artopk_matrix* mats, int32_t count, int64_t n, int32_t type,
                           int32_t products, void* hip_stream) {
  if (!out) return fail_text(g_noctx_err, ARTOPK_EINVAL, "out is NULL");
  Plans plans;
  try {
    const int rc = make_plans(mats, count, n, type, products, &plans, g_noctx_err);
    if (rc) return rc;
  } catch (const std::exception&) {
    return fail_text(g_noctx_err, ARTOPK_ENOMEM, "out of host memory");
  }
  artopk_matrices* h = new (std::nothrow) artopk_matrices();
  if (!h) return fail_text(g_noctx_err, ARTOPK_ENOMEM, "out of host memory");
  h->stream = reinterpret_cast<hipStream_t>(hip_stream);
  h->n = n;
  h->type = type;
  void* p = nullptr;
  hipError_t e = hipMalloc(&p, plans.total);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    delete h;
    return fail_text(g_noctx_err, ARTOPK_ENOMEM, "hipMalloc of %lld bytes failed: %s", (long long)plans.total, hipGetErrorString(e));
  }
  h->slab = static_cast<char*>(p);
  h->mem = reinterpret_cast<_Float16*>(h->slab + plans.o_mem);
  for (int i = 0; i < plans.count && e == hipSuccess; ++i) {
    const MatPlan& plan = plans.plan[i];
    Route& r = i == 0 ? h->own : h->weights;
    r.nchunks = (int)plan.chunks.size();
    r.ngroups = plan.ngroups;
    for (int g = 0; g < plan.ngroups; ++g) r.groups[g] = plan.groups[g];
    r.mats = reinterpret_cast<const MatDesc*>(h->slab + plans.o_mats[i]);
    r.chunks = reinterpret_cast<const MatChunk*>(h->slab + plans.o_chunks[i]);
    r.tiles = reinterpret_cast<const MatTile*>(h->slab + plans.o_tiles[i]);
    r.sums = reinterpret_cast<double*>(h->slab + plans.o_sums[i]);
    r.sizes = reinterpret_cast<float*>(h->slab + plans.o_sizes[i]);
    r.partial = reinterpret_cast<float*>(h->slab + plans.o_partial[i]);
    auto fill = [&](size_t to, const void* from, size_t bytes) {
      if (e == hipSuccess && bytes) e = hipMemcpy(h->slab + to, from, bytes, hipMemcpyHostToDevice);
    };
    fill(plans.o_mats[i], plan.mats.data(), plan.mats.size() * sizeof(MatDesc));
    fill(plans.o_chunks[i], plan.chunks.data(), plan.chunks.size() * sizeof(MatChunk));
    fill(plans.o_tiles[i], plan.tiles.data(), plan.tiles.size() * sizeof(MatTile));
    for (int g = 0; g < r.ngroups; ++g)
      if (e == hipSuccess && r.groups[g].small_lds) e = r.groups[g].parts == 2 ? allow_small<2>(h) : allow_small<1>(h);
  }
  if (plans.count == 1) h->weights = h->own;
  if (e != hipSuccess) {
    (void)hipFree(h->slab);
    delete h;
    return fail_text(g_noctx_err, ARTOPK_EHIP, "filling the tables failed: %s", hipGetErrorString(e));
  }
  *out = h;
  return ARTOPK_OK;
}

int artopk_matrices_destroy(artopk_matrices* m) {
  if (!m) return ARTOPK_EINVAL;
  if (m->slab) (void)hipFree(m->slab);
  delete m;
  return ARTOPK_OK;
}

const char* artopk_matrices_last_error(const artopk_matrices* m) { return m ? m->err : g_noctx_err; }

int artopk_orthogonalize(artopk_matrices* m, const void* x, void* out, int32_t steps, const float* coefficients, float eps) {
  if (!m) return fail_text(g_noctx_err, ARTOPK_EINVAL, "artopk_orthogonalize: m is NULL");
  int rc;
  Steps st;
  const size_t size = elem_size(m->type);
  if ((rc = check_vector(m, "x", x, size)) || (rc = check_vector(m, "out", out, size))) return rc;
  if ((rc = take_coefficients(m, steps, coefficients, &st)) || (rc = check_eps(m, eps))) return rc;
  {
    RangeSet rs;
    rs.add(x, (size_t)m->n * size, false, "x");
    rs.add(out, (size_t)m->n * size, true, "out");
    if ((rc = rs.check(m->err))) return rc;
  }
  FinishArgs f = {};
  f.out = out;
  f.type = m->type;
  with_type(m->type, [&](auto* tag) {
    using T = std::remove_pointer_t<decltype(tag)>;
    const Route& r = m->own;
    bool sums = steps == 0;  // (small matrices' blocks sum for themselves)
    for (int i = 0; i < r.ngroups; ++i) sums |= r.groups[i].small_lds == 0;
    if (sums) k_mat_squares<T><<<r.nchunks, 256, 0, m->stream>>>(static_cast<const T*>(x), r.chunks, r.sums);
    polar(m, r, FromVector<T>{static_cast<const T*>(x)}, st, eps, f);
  });
  MAT_TRY(m, hipGetLastError());
  return ARTOPK_OK;
}

int artopk_muon_step(artopk_matrices* m, void* weights, float* momentum, const float* update, float update_scale, float mu,
                     int32_t nesterov, float eta, float decay, float eta_rest, int32_t steps, const float* coefficients,
                     float eps) {
  if (!m) return fail_text(g_noctx_err, ARTOPK_EINVAL, "artopk_muon_step: m is NULL");
  int rc;
  Steps st;
  const size_t size = elem_size(m->type);
  if ((rc = check_vector(m, "weights", weights, size)) || (rc = check_vector(m, "momentum", momentum, 4)) ||
      (rc = check_vector(m, "update", update, 4)))
    return rc;
  if (!std::isfinite(update_scale) || !std::isfinite(mu) || !std::isfinite(eta) || !std::isfinite(decay) ||
      !std::isfinite(eta_rest))
    return fail_text(m->err, ARTOPK_EINVAL, "update_scale, mu, eta, decay or eta_rest is not finite");
  if ((rc = take_coefficients(m, steps, coefficients, &st)) || (rc = check_eps(m, eps))) return rc;
  {
    RangeSet rs;
    rs.add(weights, (size_t)m->n * size, true, "weights");
    rs.add(momentum, (size_t)m->n * 4, true, "momentum");
    rs.add(update, (size_t)m->n * 4, false, "update");
    if ((rc = rs.check(m->err))) return rc;
  }
  FinishArgs f = {};
  f.out = weights;
  f.type = m->type;
  f.muon = 1;
  f.a = MuonArgs{mu, update_scale, nesterov != 0, eta, (float)(1.0 - (double)eta * (double)decay), eta_rest};
  const Route& r = m->weights;
  with_type(m->type, [&](auto* tag) {
    using T = std::remove_pointer_t<decltype(tag)>;
    k_mat_momentum<T><<<r.nchunks, 256, 0, m->stream>>>(static_cast<T*>(weights), momentum, update, f.a, r.chunks, r.sums);
  });
  polar(m, r, FromMomentum{momentum, update, f.a}, st, eps, f);
  MAT_TRY(m, hipGetLastError());
  return ARTOPK_OK;
}
