// C ABI of the orthogonalising call: argument checks, the workspace's layout, the lists of
// workgroups of every phase.  The arithmetic is in slowmo_orth.hip.
#include "slowmo_orth.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <memory>
#include <type_traits>
#include <vector>

#include "../../include/slowmo_operators.h"
#include "slowmo_status.h"

using namespace slowmo;
using namespace slowmo::orth;

namespace {

// One launch's worth of the program that every matrix goes through.
struct Op {
  bool update;
  Symmetric symmetric;
  Update up;
};

// The tiles of the three kinds of products: X X^T, n x n by n x n, and n x n by X.
struct Lists {
  std::vector<Tile> gram, square, update;
};

struct Device {
  const Tile *gram = nullptr, *square = nullptr, *update = nullptr;
  int32_t n_gram = 0, n_square = 0, n_update = 0;
};

}  // namespace

struct slowmo_orth {
  bool split = false, small = false;
  int32_t small_side = 0;
  Steps steps{};
  std::vector<Op> program;
  std::vector<int32_t> index;       // places in the caller's list of the matrices that are not empty
  Call call{};
  const Item *sums = nullptr, *load = nullptr;
  const int32_t *tiny = nullptr;
  int32_t n_tiny = 0, n_sums = 0, n_load = 0;
  Device tiles[kKinds];
};

namespace {

constexpr int64_t kMostSide = 65536;
constexpr size_t kAlign = 256;
const float kDefault[3] = {3.4445f, -4.7750f, 2.0315f};

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// Everything a handle needs, laid out from the configuration and the shapes alone.
struct Plan {
  bool pairs = false;
  bool small = false;         // every matrix goes by one workgroup from load to store
  std::vector<Matrix> matrices;
  std::vector<int32_t> index, tiny;
  std::vector<Item> sums, load;
  Lists lists[kKinds];
  int64_t partial_sums = 0;   // floats
  int32_t tickets = 0;
  size_t matrices_at = 0, addresses_at = 0, sums_at = 0, scales_at = 0, abc_at = 0, tiny_at = 0, sum_items_at = 0, load_at = 0,
         tiles_at[kKinds][3] = {}, tickets_at = 0, partial_at = 0, arena_at = 0, total = 0;
};

const char *check(const slowmo_orth_config *c, int32_t n, const int64_t *rows, const int64_t *cols,
                  const int64_t *ld) {
  if (!c) return "cfg is NULL";
  for (int32_t d : {c->in_dtype, c->out_dtype})
    if (d != SLOWMO_F32 && d != SLOWMO_BF16) return "unknown dtype";
  if (c->steps < 1 || c->steps > SLOWMO_MAX_ORTH_STEPS) return "steps must be in 1..SLOWMO_MAX_ORTH_STEPS";
  if (c->scale != SLOWMO_SCALE_NONE && c->scale != SLOWMO_SCALE_SHAPE && c->scale != SLOWMO_SCALE_RMS)
    return "unknown scale";
  if (!(std::isfinite(c->eps) && c->eps >= 0.f)) return "eps must be finite and >= 0";
  if (c->coefficients)
    for (int32_t i = 0; i < 3 * c->steps; ++i)
      if (!std::isfinite(c->coefficients[i])) return "a coefficient is not finite";
  if (n < 1 || n > (1 << 20)) return "n_matrices must be in 1..2^20";
  if (!rows || !cols) return "rows or cols is NULL";
  for (int32_t i = 0; i < n; ++i) {
    if (rows[i] < 0 || cols[i] < 0 || rows[i] > kMostSide || cols[i] > kMostSide)
      return "sides must be in 0..65536";
    if (ld && (ld[i] < cols[i] || ld[i] > (int64_t(1) << 40))) return "ld must be in cols..2^40";
  }
  return nullptr;
}

// Tiles of a grid in bands of 8 rows, down each column of a band: neighbours share the columns' factor,
// which for P X is the long one.
template <typename F>
void walk(int32_t down, int32_t across, F &&f) {
  for (int32_t a0 = 0; a0 < down; a0 += 8)
    for (int32_t b = 0; b < across; ++b)
      for (int32_t a = a0; a < std::min(down, a0 + 8); ++a) f(a, b);
}

// Workgroups go to the 8 dies in turn, each with an L2 of its own.  The list in bundles -- a matrix's tiles,
// or 32 neighbours of a large one's -- goes to the dies whole, each to the one with the fewest steps so far, so
// that a factor is fetched into one L2 and no die gets all of the longest sums.
std::vector<Tile> spread(const std::vector<Tile> &v) {
  int64_t steps[8] = {};
  std::vector<Tile> queue[8], out;
  for (size_t at = 0; at < v.size();) {
    size_t end = at;
    while (end < v.size() && v[end].matrix == v[at].matrix && v[end].pieces == v[at].pieces) ++end;
    if (end - at > 32 && (end - at) * 16 > v.size()) end = at + 32;
    const auto die = std::min_element(steps, steps + 8) - steps;
    for (; at < end; ++at) {
      queue[die].push_back(v[at]);
      steps[die] += v[at].count;
    }
  }
  // All of them run at once, and a die's CUs take them in turn: where their sums are of very unequal length, long
  // and short ones go together, by three rounds of 32 of which the second runs backwards (ResNet-18's matrices
  // for 8 workers, 4 to 144 steps: 2.48 / 2.45 ms a call without / with this).
  const auto [least, most] = std::minmax_element(v.begin(), v.end(), [](const Tile &a, const Tile &b) { return a.count < b.count; });
  if (!v.empty() && v.size() <= 768 && most->count > 4 * least->count)
    for (auto &q : queue) {
      std::stable_sort(q.begin(), q.end(), [](const Tile &a, const Tile &b) { return a.count > b.count; });
      for (size_t at = 32; at < q.size(); at += 64) std::reverse(q.begin() + at, q.begin() + std::min(q.size(), at + 32));
    }
  size_t next[8] = {};
  while (out.size() < v.size()) {
    size_t die = out.size() % 8;
    if (next[die] == queue[die].size())  // it has run out: the one with the most left gives
      for (size_t d = 0; d < 8; ++d)
        if (queue[d].size() - next[d] > queue[die].size() - next[die]) die = d;
    out.push_back(queue[die][next[die]++]);
  }
  return out;
}

// What is left of the list after whole rounds of `slots` workgroups would leave most of the card idle
// for the length of its longest tile: its tiles are cut along the summed side into shares of about equal
// length, as many as there are slots.  Shares are no shorter than 48 steps and no more than 16 to
// a tile, since the last one adds the others' sums up (no shorter than 32 / 48 / 96 / 128: an encoder block's
// matrices 432 / 405 / 411 / 437 us a call).  The 48 was measured on bf16 results; of pairs of halves a step
// has three products, and other lengths were not measured.
void balance(std::vector<Tile> &v, int kind, Plan &p) {
  const int32_t slots = kSlotsOf[kind];
  const size_t whole = v.size() / slots * slots;
  if (whole == v.size()) return;
  int32_t longest = 0;
  for (size_t i = whole; i < v.size(); ++i) longest = std::max(longest, v[i].count);
  auto shares = [&](int32_t length) {
    int64_t n = 0;
    for (size_t i = whole; i < v.size(); ++i) n += (v[i].count + length - 1) / length;
    return n;
  };
  int32_t lo = std::max(48, (longest + 15) / 16), hi = std::max(longest, lo);
  while (lo < hi) {
    const int32_t mid = (lo + hi) / 2;
    if (shares(mid) <= slots)
      hi = mid;
    else
      lo = mid + 1;
  }
  std::vector<Tile> out(v.begin(), v.begin() + whole);
  int64_t slot = 0;
  int32_t ticket = 0;
  for (size_t i = whole; i < v.size(); ++i) {
    const int32_t pieces = (v[i].count + lo - 1) / lo;
    if (pieces < 2) {
      out.push_back(v[i]);
      continue;
    }
    for (int32_t q = 0; q < pieces; ++q) {
      Tile t = v[i];
      t.first = static_cast<int32_t>(static_cast<int64_t>(v[i].count) * q / pieces);
      t.count = static_cast<int32_t>(static_cast<int64_t>(v[i].count) * (q + 1) / pieces) - t.first;
      t.piece = q;
      t.pieces = pieces;
      t.slot = static_cast<int32_t>(slot);
      t.ticket = ticket;
      out.push_back(t);
    }
    slot += pieces;
    ++ticket;
  }
  p.partial_sums = std::max(p.partial_sums, slot * kRowsOf[kind] * kColsOf[kind]);
  p.tickets = std::max(p.tickets, ticket);
  v.swap(out);
}

// Squares of 256 have half the traffic in shared memory per product but one workgroup per CU, which
// stands still while it writes its results: they pay where sums are long and tiles are many.
// 8192 x 8192, tiles of 256 / 128: 983 / 1190 us a product.  With 256 from n = 1024 on, 32 of 1024 x 1024 and 16 of
// 1024 x 4096 took 2.87 ms for 2.64, six such matrices 764 us for 457.
bool large_tiles(const Matrix &m) {
  return m.n >= 2048 && static_cast<int64_t>(m.n) * m.k >= int64_t(256) * 256 * 256;
}

// Rows of 256 for P X: three quarters of the traffic per product, two workgroups per CU.
bool wide_tiles(const Matrix &m) { return m.n >= 256 && m.kp % 256 == 0; }

// One workgroup in 64 bits: what fits its shared memory, and longer ones that k_small does not take, while
// the products' launches take longer (one workgroup / products: 604 x 17 72 / 123 us, 32 x 512 148 / 115 us).
bool tiny(const Matrix &m) {
  const int64_t n = m.n, k = m.k;
  return n <= kTinySide && (n * k <= kTinyElements || (k > kSmallLength && n * n * k <= kTinyWork));
}

float factor(const slowmo_orth_config &c, int64_t rows, int64_t cols) {
  const double r = static_cast<double>(rows), k = static_cast<double>(cols);
  return static_cast<float>(c.scale == SLOWMO_SCALE_NONE    ? 1.
                            : c.scale == SLOWMO_SCALE_SHAPE ? std::sqrt(std::max(1., r / k))
                                                            : 0.2 * std::sqrt(std::max(r, k)));
}

Steps steps_of(const slowmo_orth_config &c) {
  Steps s{};
  s.count = c.steps;
  for (int32_t t = 0; t < c.steps; ++t)
    for (int i = 0; i < 3; ++i) s.abc[t][i] = c.coefficients ? c.coefficients[3 * t + i] : kDefault[i];
  return s;
}

Plan plan(const slowmo_orth_config &c, int32_t n_matrices, const int64_t *rows, const int64_t *cols,
          const int64_t *ld) {
  Plan p;
  const bool split = c.out_dtype == SLOWMO_F32;
  double one_by_one = 0., by_pairs = 0.;
  std::vector<int32_t> of[2];  // matrices in small and in large tiles
  for (int32_t i = 0; i < n_matrices; ++i) {
    if (!rows[i] || !cols[i]) continue;
    Matrix m{};
    m.tall = rows[i] > cols[i];
    m.n = static_cast<int32_t>(std::min(rows[i], cols[i]));
    m.k = static_cast<int32_t>(std::max(rows[i], cols[i]));
    m.ld = ld ? ld[i] : cols[i];
    m.scale = factor(c, rows[i], cols[i]);
    const int32_t at = static_cast<int32_t>(p.matrices.size());
    if (tiny(m)) {
      p.tiny.push_back(at);
      m.tiny = 1;
    } else {
      const int which = large_tiles(m);
      of[which].push_back(at);
      m.np = static_cast<int32_t>(up(m.n, kRowsOf[which]));
      m.kp = static_cast<int32_t>(up(m.k, kRowsOf[which]));
      const double n = m.np, k = m.kp;
      one_by_one += 6. * n * n * k + 2. * n * n * n;
      by_pairs += 3. * n * n * k + 5. * n * n * n;
    }
    p.matrices.push_back(m);
    p.index.push_back(i);
  }
  // Small matrices alone (beside tiny ones): one workgroup each.
  int32_t side = split ? kSmallSideSplit : kSmallSide, small = 0;
  for (const Matrix &m : p.matrices) small += m.tiny || (m.n <= side && m.k <= kSmallLength);
  p.small = p.tiny.size() < p.matrices.size() && small == static_cast<int32_t>(p.matrices.size());
  if (p.small)
    for (auto &list : of) list.clear();
  // The first two steps as one, on n x n matrices: see program().  8 matrices of n x k, as one / one by one, us:
  // n = 1024, k / n = 1.25 375 / 372, 1.5 395 / 396, 2 491 / 518, 4 759 / 842; n = 512 165 / 157, 169 / 163, 177 / 174,
  // 231 / 242; fp32 results, n = 1024 807 / 778, 871 / 856, 1021 / 1043, 1583 / 1743.  The bound below takes one from
  // k / n = 1.25 on, up to 8 % too early.
  p.pairs = !p.small && c.steps >= 3 && by_pairs < 0.93 * one_by_one;

  int64_t halves = 0;
  auto take = [&](int64_t count) {
    const int64_t at = halves;
    halves += up(count, kAlign / sizeof(uint16_t));
    return at;
  };
  int32_t sums = 0;
  for (auto &list : of) {
    for (int32_t at : list) {
      Matrix &m = p.matrices[at];
      m.at = take(Places(m.np, m.kp, p.pairs ? kSquares : 2).total(split));
      m.first_sum = sums;
      m.sums = static_cast<int32_t>(std::min<int64_t>(kMostSums, (static_cast<int64_t>(m.n) * m.k + 16383) / 16384));
      sums += m.sums;
      for (int32_t q = 0; q < m.sums; ++q) p.sums.push_back({at, q, m.sums, 0});
      const int32_t down = (m.tall ? m.kp : m.np) / kPatch, across = (m.tall ? m.np : m.kp) / kPatch;
      for (int32_t a = 0; a < down; ++a)
        for (int32_t b = 0; b < across; b += kPatches) p.load.push_back({at, a, b, 0});
    }
  }
  for (int which : {kSmall, kLarge}) {
    auto grams = of[which], updates = of[which];
    auto by = [&](auto side) {
      return [&p, side](int32_t a, int32_t b) { return p.matrices[a].*side > p.matrices[b].*side; };
    };
    std::stable_sort(grams.begin(), grams.end(), by(&Matrix::kp));  // long sums first
    std::stable_sort(updates.begin(), updates.end(), by(&Matrix::np));
    const int32_t side = kRowsOf[which];
    auto put = [&](std::vector<Tile> &v, int32_t at, int32_t i, int32_t j, int32_t depth) {
      const Matrix &m = p.matrices[at];
      v.push_back({m.at, m.np, m.kp, i, j, 0, depth / kDeep, 0, 1, 0, 0, at, {}});
    };
    auto put_half = [&](std::vector<Tile> &v, int32_t at, int32_t i, int32_t j, int32_t depth) {
      if (j > i) return;
      put(v, at, i, j, depth);
      if (j == i && !split) v.back().count /= 2;  // the diagonal's steps go two by two; depth is a multiple of 128
    };
    Lists &to = p.lists[which];
    for (int32_t at : grams) {
      const Matrix &m = p.matrices[at];
      walk(m.np / side, m.np / side, [&](int32_t i, int32_t j) {
        put_half(to.gram, at, i, j, m.kp);
      });
    }
    for (int32_t at : updates) {
      const Matrix &m = p.matrices[at];
      walk(m.np / side, m.np / side, [&](int32_t i, int32_t j) {
        put_half(to.square, at, i, j, m.np);
      });
      const int kind = which == kSmall && wide_tiles(m) ? kWide : which;
      walk(m.np / side, m.kp / kColsOf[kind], [&](int32_t i, int32_t j) { put(p.lists[kind].update, at, i, j, m.np); });
    }
  }
  // Too few to fill the card, or beside small ones, whose launch would come on top: as small ones.  Matrices of 1024 x
  // 4096, wide / small, us: 256 wide tiles 318 / 315, 384 419 / 414, 512 459 / 465, 1024 760 / 777, 4096 2712 / 2827;
  // with two of 128 x 512 beside them 384 444 / 413, 512 486 / 475, 768 647 / 652, 2048 1309 / 1313, 4096 2866 / 2829
  // (fp32 results 384 786 / 752, 512 890 / 904, 2048 2925 / 2969).
  if (p.lists[kWide].update.size() < (p.lists[kSmall].update.empty() ? 512u : 2048u)) {
    for (const Tile &t : p.lists[kWide].update)
      for (int32_t half : {0, 1}) {
        Tile s = t;
        s.j = 2 * t.j + half;
        p.lists[kSmall].update.push_back(s);
      }
    p.lists[kWide].update.clear();
    std::stable_sort(p.lists[kSmall].update.begin(), p.lists[kSmall].update.end(),
                     [](const Tile &a, const Tile &b) { return a.count > b.count; });
  }
  for (int kind = 0; kind < kKinds; ++kind) {
    Lists &l = p.lists[kind];
    for (std::vector<Tile> *v : {&l.gram, &l.square, &l.update}) {
      balance(*v, kind, p);
      *v = spread(*v);
    }
  }
  size_t off = 0;
  auto section = [&](size_t bytes) {
    const size_t at = off;
    off += static_cast<size_t>(up(static_cast<int64_t>(std::max<size_t>(bytes, 1)), kAlign));
    return at;
  };
  p.matrices_at = section(p.matrices.size() * sizeof(Matrix));
  p.addresses_at = section(p.matrices.size() * sizeof(Addresses));
  p.sums_at = section(p.sums.size() * sizeof(double));
  p.scales_at = section(p.matrices.size() * kScales * sizeof(float));
  p.abc_at = section(sizeof(Steps::abc));
  p.tiny_at = section(p.tiny.size() * sizeof(int32_t));
  p.sum_items_at = section(p.sums.size() * sizeof(Item));
  p.load_at = section(p.load.size() * sizeof(Item));
  for (int which = 0; which < kKinds; ++which) {
    const Lists &l = p.lists[which];
    p.tiles_at[which][0] = section(l.gram.size() * sizeof(Tile));
    p.tiles_at[which][1] = section(l.square.size() * sizeof(Tile));
    p.tiles_at[which][2] = section(l.update.size() * sizeof(Tile));
  }
  p.tickets_at = section(p.tickets * sizeof(uint32_t));
  p.partial_at = section(static_cast<size_t>(p.partial_sums) * sizeof(float));
  p.arena_at = section(static_cast<size_t>(halves) * sizeof(uint16_t));
  p.total = off;
  return p;
}

// The largest of |f(s)| for singular values s up to `most`, with 2 % for what rounding adds.
template <typename F>
double largest(double most, F &&f) {
  double v = 0.;
  for (int i = 0; i <= 2048; ++i) v = std::max(v, std::fabs(f(most * i / 2048.)));
  return 1.02 * v;
}

// The power of two that a half array of spectral norm `most` is held times.
float power(double most) {
  return static_cast<float>(std::min(8192., std::exp2(std::floor(std::log2(32768. / std::max(most, 1e-30))))));
}

// The largest singular value of X in front of each step and after the last, and whether all stay under 7.5 (halves
// times 2^kPowerX reach 8).  Followed in 4096 pieces of 0..1, each as the interval that a step's polynomial takes it
// to, widened for rounding by kRounding of |a| s + |b| s^3 + |c| s^5.  One interval, or 2 % of each value for
// rounding, refuses schedules of steps that are steep past the values that arrive there, as fast ones are:
// quintics that are each the best approximation of 1 on what the one before leaves of 1e-3..1 reach 1.99 and, divided by
// a safety factor of 1.01, stay at 2.00 here.  Without the factor they are refused, rightly: roundings at the steep end
// grow 12-fold a step, and matrices of equal elements came to infinity (halves) and 249 (pairs) on the CPU.
constexpr double kMostValue = 7.5, kRounding = 1. / 1024;

bool follow(const Steps &steps, double (&most)[SLOWMO_MAX_ORTH_STEPS + 1]) {
  constexpr int kPieces = 4096;
  struct Interval {
    double lo, hi;
  };
  std::vector<Interval> v(kPieces);
  for (int i = 0; i < kPieces; ++i) v[i] = {i / double(kPieces), (i + 1) / double(kPieces)};
  most[0] = 1.;
  for (int32_t t = 0; t < steps.count; ++t) {
    const double a = steps.abc[t][0], b = steps.abc[t][1], c = steps.abc[t][2];
    auto f = [=](double s) { return s * (a + s * s * (b + c * s * s)); };
    // where the slope a + 3 b s^2 + 5 c s^4 is zero
    double turns[4], square[2] = {-1., -1.};
    const double root = 9. * b * b - 20. * a * c;
    if (root >= 0.) {
      const double q = -0.5 * (3. * b + std::copysign(std::sqrt(root), b));
      if (c != 0.) square[0] = q / (5. * c);
      if (q != 0.) square[1] = a / q;
    }
    for (int i = 0; i < 2; ++i) {
      turns[2 * i] = square[i] > 0. ? std::sqrt(square[i]) : 0.;
      turns[2 * i + 1] = -turns[2 * i];
    }
    double largest = 0.;
    for (Interval &p : v) {
      const double at = std::max(std::fabs(p.lo), std::fabs(p.hi)), square = at * at;
      const double wide = kRounding * at * (std::fabs(a) + square * (std::fabs(b) + square * std::fabs(c)));
      double lo = std::min(f(p.lo), f(p.hi)), hi = std::max(f(p.lo), f(p.hi));
      for (double s : turns)
        if (s > p.lo && s < p.hi) lo = std::min(lo, f(s)), hi = std::max(hi, f(s));
      p = {lo - wide, hi + wide};
      largest = std::max({largest, -p.lo, p.hi});
    }
    if (!(largest < kMostValue)) return false;
    most[t + 1] = std::max(largest, 1e-3);
  }
  return true;
}

// The steps as launches.  One step is A = X X^T, P = b A + c A A, X <- a X + P X.  Where X is much
// longer than wide, the first two steps are one: with P0 from A0, the second step's A is
// (a0 + P0)^2 A0, a product of n x n matrices too, and X <- a0 a1 X + Q X with
// Q = (a0 + P0)(a1 + P1) - a0 a1: 3 n n k + 5 n n n for 6 n n k + 2 n n n, and X is read and written once
// less.  (All n x n factors are polynomials of the same A, so that each product of two is symmetric
// again.)  Only the first two: A's roundings reach the second step's A a0^2 = 12 times as large, which shows
// once singular values are near 1.  512 x 2048 against 64 bits, products of halves / of pairs: one by
// one 0.8e-3 / 2.2e-6, first two 0.8e-3 / 1.8e-6, the next two as well 3.3e-3 / 3.8e-6.
// Leaves the powers of two with the steps.  Returns an empty program if the coefficients let X outgrow a half (follow()).
std::vector<Op> program(Steps &steps, bool pairs, bool split) {
  std::vector<Op> ops;
  enum { kA, kP, kW, kQ };
  auto symmetric = [&](Symmetric s) {
    Op op{};
    op.symmetric = s;
    ops.push_back(op);
  };
  double bounds[SLOWMO_MAX_ORTH_STEPS + 1];
  if (!follow(steps, bounds)) return {};
  int32_t from = 0;
  for (int32_t t = 0; t < steps.count;) {
    const bool two = pairs && t == 0;
    const double most = bounds[t];
    const double a0 = steps.abc[t][0], b0 = steps.abc[t][1], c0 = steps.abc[t][2];
    auto p0 = [=](double s) { return b0 * s * s + c0 * s * s * s * s; };
    // Of single halves the last two steps' a goes to P's diagonal; the others' X enters as hi + lo.
    // Pairs of halves have bits enough.
    const bool carry = !split && (two || t < steps.count - 2);
    const double keep0 = carry ? 0. : a0;
    const float sa = power(largest(most, [&](double s) { return s * s; }));
    const float sp = power(largest(most, [&](double s) { return p0(s) + (two ? 0. : keep0); }));
    steps.a_power[t] = sa;
    steps.p_power[t] = sp;
    steps.carry[t] = carry;
    symmetric({from, -1, -1, -1, -1, kA, sa / (kScaleX * kScaleX), 0.f, 0.f, 0.f, t == 0, t});
    symmetric({from, kA, kA, kA, -1, kP, static_cast<float>(c0 * sp / (double(sa) * sa)),
               static_cast<float>(b0 * sp / sa), 0.f, static_cast<float>(two ? 0. : keep0 * sp), 0, -1});
    Op op{};
    op.update = true;
    op.up = {from, kP, carry, 0, 0, 1.f / sp, static_cast<float>(a0), t == 0, kScales / 2 + t};
    if (two) {
      const double a1 = steps.abc[t + 1][0], b1 = steps.abc[t + 1][1], c1 = steps.abc[t + 1][2];
      auto x1 = [=](double s) { return s * (a0 + p0(s)); };
      auto p1 = [=](double s) { return b1 * x1(s) * x1(s) + c1 * std::pow(x1(s), 4.); };
      const double keep = carry ? 0. : a0 * a1;
      const float sw = power(largest(most, [&](double s) { return s * x1(s); }));
      const float sa1 = power(largest(most, [&](double s) { return x1(s) * x1(s); }));
      const float sp1 = power(largest(most, p1));
      const float sq = power(largest(most, [&](double s) { return (a0 + p0(s)) * (a1 + p1(s)) - a0 * a1 + keep; }));
      symmetric({from, kP, kA, kA, -1, kW, sw / (sp * sa), static_cast<float>(a0 * sw / sa), 0.f, 0.f, 0, -1});
      symmetric({from, kW, kP, kW, -1, kA, sa1 / (sw * sp), static_cast<float>(a0 * sa1 / sw), 0.f, 0.f, 0, -1});
      symmetric({from, kA, kA, kA, -1, kW, static_cast<float>(c1 * sp1 / (double(sa1) * sa1)),
                 static_cast<float>(b1 * sp1 / sa1), 0.f, 0.f, 0, -1});
      symmetric({from, kW, kP, kP, kW, kQ, sq / (sp1 * sp), static_cast<float>(a1 * sq / sp),
                 static_cast<float>(a0 * sq / sp1), static_cast<float>(keep * sq), 0, -1});
      op.up.by = kQ;
      op.up.alpha = 1.f / sq;
      op.up.beta = static_cast<float>(a0 * a1);
    }
    ops.push_back(op);
    from = 1 - from;
    t += two ? 2 : 1;
  }
  Update *next = nullptr;
  for (auto op = ops.rbegin(); op != ops.rend(); ++op) {
    if (!op->update) continue;
    op->up.last = next == nullptr;
    op->up.carry_next = next && next->carry;
    next = &op->up;
  }
  return ops;
}

slowmo_status run(slowmo_orth *h, const void *const *in, float *const *momentum, void *const *out, float mu,
                  int32_t nesterov, void *stream_) {
  const bool with_momentum = momentum != nullptr;
  const size_t in_size = h->call.in_bf16 ? 2 : 4, out_size = h->call.out_bf16 ? 2 : 4;
  const int32_t count = static_cast<int32_t>(h->index.size());
  for (int32_t i = 0; i < count; ++i) {
    const int32_t at = h->index[i];
    if (!in[at] || !out[at] || (with_momentum && !momentum[at]))
      return fail_thread(SLOWMO_ERR_ARG, "a matrix pointer is NULL");
    if (reinterpret_cast<uintptr_t>(in[at]) % in_size || reinterpret_cast<uintptr_t>(out[at]) % out_size ||
        (with_momentum && reinterpret_cast<uintptr_t>(momentum[at]) % 4))
      return fail_thread(SLOWMO_ERR_ALIGN, "a matrix pointer is not aligned to its element size");
  }
  if (!count) return SLOWMO_OK;
  hipStream_t s = static_cast<hipStream_t>(stream_);
  Call c = h->call;
  c.mu = mu;
  c.nesterov = nesterov;
  c.momentum = with_momentum;
  c.exact = c.in_bf16 && !with_momentum && !h->split;
  hipError_t e = hipSuccess;
  auto ok = [&](hipError_t got) { return (e = got) == hipSuccess; };
  auto refused = [&] { return fail_thread_hip(e, "slowmo_orthogonalize (results may be partly written)"); };
  for (int32_t first = 0; first < count; first += kInline) {
    Few few{};  // travels with the launch
    const int32_t some = std::min(kInline, count - first);
    for (int32_t i = 0; i < some; ++i) {
      const int32_t at = h->index[first + i];
      few.at[i] = {in[at], with_momentum ? momentum[at] : nullptr, out[at]};
    }
    if (h->small && !ok(launch_small(c, h->steps, few, first, some, h->small_side, h->split, s))) return refused();
    if ((!h->small || h->n_tiny) && !ok(launch_addresses(c, few, first, some, s))) return refused();
  }
  if (h->n_tiny && !ok(launch_tiny(c, h->steps, h->tiny, h->n_tiny, s))) return refused();
  if (h->small || h->n_tiny == count) return SLOWMO_OK;
  if (!ok(launch_sums(c, h->sums, h->n_sums, s)) || !ok(launch_load(c, h->load, h->n_load, s))) return refused();
  for (const Op &op : h->program) {
    for (int which = 0; which < kKinds; ++which) {
      const Device &d = h->tiles[which];
      const bool gram = op.symmetric.left < 0;
      const int32_t tiles = op.update ? d.n_update : gram ? d.n_gram : d.n_square;
      if (!tiles) continue;
      if (!ok(op.update ? launch_update(c, which, op.up, d.update, tiles, h->split, s)
                        : launch_symmetric(c, which, op.symmetric, gram ? d.gram : d.square, tiles, h->split, s)))
        return refused();
    }
  }
  return SLOWMO_OK;
}

}  // namespace

extern "C" {

// Reasons to refuse that both calls share.
static const char *refusal(const slowmo_orth_config *cfg, int32_t n_matrices, const int64_t *rows,
                           const int64_t *cols, const int64_t *ld) {
  if (const char *bad = check(cfg, n_matrices, rows, cols, ld)) return bad;
  Steps steps = steps_of(*cfg);
  if (program(steps, false, false).empty()) return "the coefficients let singular values grow to 7.5";
  return nullptr;
}

size_t slowmo_orth_bytes(const slowmo_orth_config *cfg, int32_t n_matrices, const int64_t *rows,
                         const int64_t *cols, const int64_t *ld) {
  size_t bytes = 0;
  walled([&]() -> slowmo_status {
    if (const char *bad = refusal(cfg, n_matrices, rows, cols, ld)) return fail_thread(SLOWMO_ERR_ARG, bad);
    bytes = plan(*cfg, n_matrices, rows, cols, ld).total;
    return SLOWMO_OK;
  });
  return bytes;
}

slowmo_status slowmo_orth_create(slowmo_orth **out, const slowmo_orth_config *cfg, int32_t n_matrices,
                                 const int64_t *rows, const int64_t *cols, const int64_t *ld,
                                 void *workspace, size_t workspace_bytes, void *stream) {
  if (!out) return fail_thread(SLOWMO_ERR_ARG, "out is NULL");
  *out = nullptr;
  return walled([&]() -> slowmo_status {
    if (const char *bad = refusal(cfg, n_matrices, rows, cols, ld)) return fail_thread(SLOWMO_ERR_ARG, bad);
    if (!workspace) return fail_thread(SLOWMO_ERR_ARG, "workspace is NULL");
    if (reinterpret_cast<uintptr_t>(workspace) % kAlign)
      return fail_thread(SLOWMO_ERR_ALIGN, "workspace must be 256-byte aligned");
    Plan p = plan(*cfg, n_matrices, rows, cols, ld);
    if (workspace_bytes < p.total)
      return fail_thread(SLOWMO_ERR_NOMEM, "workspace is smaller than slowmo_orth_bytes()");
    if (slowmo_status st = slowmo_check_device_range(workspace, p.total); st != SLOWMO_OK) return st;
    std::unique_ptr<slowmo_orth> h(new slowmo_orth);
    h->split = cfg->out_dtype == SLOWMO_F32;
    h->steps = steps_of(*cfg);
    h->small = p.small;
    for (const Matrix &m : p.matrices) h->small_side = std::max(h->small_side, m.n);
    h->program = program(h->steps, p.pairs, h->split);
    h->index = p.index;
    char *base = static_cast<char *>(workspace);
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = hipSuccess;
    auto put = [&](size_t at, const auto &v, auto *&to, int32_t &count) {
      if (!v.empty() && e == hipSuccess)
        e = hipMemcpyAsync(base + at, v.data(), v.size() * sizeof(v[0]), hipMemcpyHostToDevice, s);
      to = reinterpret_cast<std::remove_reference_t<decltype(to)>>(base + at);
      count = static_cast<int32_t>(v.size());
    };
    int32_t n_matrices_here = 0;
    put(p.matrices_at, p.matrices, h->call.matrices, n_matrices_here);
    put(p.tiny_at, p.tiny, h->tiny, h->n_tiny);
    put(p.sum_items_at, p.sums, h->sums, h->n_sums);
    put(p.load_at, p.load, h->load, h->n_load);
    for (int which = 0; which < kKinds; ++which) {
      Device &d = h->tiles[which];
      put(p.tiles_at[which][0], p.lists[which].gram, d.gram, d.n_gram);
      put(p.tiles_at[which][1], p.lists[which].square, d.square, d.n_square);
      put(p.tiles_at[which][2], p.lists[which].update, d.update, d.n_update);
    }
    if (e == hipSuccess)
      e = hipMemcpyAsync(base + p.abc_at, h->steps.abc, sizeof(Steps::abc), hipMemcpyHostToDevice, s);
    if (e == hipSuccess) e = h->small ? prepare_small() : prepare_products(h->split);
    if (p.tickets && e == hipSuccess) e = hipMemsetAsync(base + p.tickets_at, 0, p.tickets * sizeof(uint32_t), s);
    const hipError_t waited = hipStreamSynchronize(s);  // the tables are in ordinary memory that ends here
    if (e == hipSuccess) e = waited;
    if (e != hipSuccess) return fail_thread_hip(e, "slowmo_orth_create");
    h->call.addresses = reinterpret_cast<Addresses *>(base + p.addresses_at);
    h->call.sums = reinterpret_cast<double *>(base + p.sums_at);
    h->call.scales = reinterpret_cast<float *>(base + p.scales_at);
    h->call.abc = reinterpret_cast<const float *>(base + p.abc_at);
    h->call.steps = h->steps.count;
    h->call.tickets = reinterpret_cast<uint32_t *>(base + p.tickets_at);
    h->call.partial = reinterpret_cast<float *>(base + p.partial_at);
    h->call.arena = reinterpret_cast<_Float16 *>(base + p.arena_at);
    h->call.buffers = p.pairs ? kSquares : 2;
    h->call.eps = cfg->eps;
    h->call.in_bf16 = cfg->in_dtype == SLOWMO_BF16;
    h->call.out_bf16 = cfg->out_dtype == SLOWMO_BF16;
    *out = h.release();
    return SLOWMO_OK;
  });
}

slowmo_status slowmo_orthogonalize(slowmo_orth *h, const void *const *in, void *const *out, void *stream) {
  return walled([&]() -> slowmo_status {
    if (!h || !in || !out) return fail_thread(SLOWMO_ERR_ARG, "the handle, in or out is NULL");
    return run(h, in, nullptr, out, 0.f, 0, stream);
  });
}

slowmo_status slowmo_momentum_orthogonalize(slowmo_orth *h, const void *const *grads, float *const *momentum,
                                            void *const *out, float mu, int32_t nesterov, void *stream) {
  return walled([&]() -> slowmo_status {
    if (!h || !grads || !momentum || !out)
      return fail_thread(SLOWMO_ERR_ARG, "the handle, grads, momentum or out is NULL");
    if (!(std::isfinite(mu) && mu >= 0.f && mu < 1.f))
      return fail_thread(SLOWMO_ERR_ARG, "mu must satisfy 0 <= mu < 1");
    if (nesterov != 0 && nesterov != 1) return fail_thread(SLOWMO_ERR_ARG, "nesterov must be 0 or 1");
    return run(h, grads, momentum, out, mu, nesterov, stream);
  });
}

slowmo_status slowmo_orth_destroy(slowmo_orth *h) {
  delete h;
  return SLOWMO_OK;
}

}  // extern "C"
