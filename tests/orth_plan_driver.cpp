// The orthogonalising call's lists of workgroups, on random lists of matrices: every tile
// of every product is there once, its shares cover its summed side once, and nothing
// reaches past a matrix, the partial sums or the tickets.  The kernels' side is left out.
#include "slowmo_orth.cpp"

#include <array>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>

namespace slowmo {
slowmo_status fail_thread(slowmo_status s, const char *) noexcept { return s; }
slowmo_status fail_thread_hip(hipError_t, const char *) noexcept { return SLOWMO_ERR_HIP; }
namespace orth {
hipError_t launch_tiny(const Call &, const Steps &, const int32_t *, int32_t, hipStream_t) { return hipSuccess; }
hipError_t launch_small(const Call &, const Steps &, const Few &, int32_t, int32_t, int32_t, bool, hipStream_t) { return hipSuccess; }
hipError_t prepare_small() { return hipSuccess; }
hipError_t launch_addresses(const Call &, const Few &, int32_t, int32_t, hipStream_t) { return hipSuccess; }
hipError_t launch_sums(const Call &, const Item *, int32_t, hipStream_t) { return hipSuccess; }
hipError_t launch_load(const Call &, const Item *, int32_t, hipStream_t) { return hipSuccess; }
hipError_t prepare_products(bool) { return hipSuccess; }
hipError_t launch_symmetric(const Call &, int, const Symmetric &, const Tile *, int32_t, bool, hipStream_t) { return hipSuccess; }
hipError_t launch_update(const Call &, int, const Update &, const Tile *, int32_t, bool, hipStream_t) { return hipSuccess; }
}  // namespace orth
}  // namespace slowmo
extern "C" slowmo_status slowmo_check_device_range(const void *, size_t) { return SLOWMO_OK; }
extern "C" hipError_t hipMemcpyAsync(void *, const void *, size_t, hipMemcpyKind, hipStream_t) { return hipSuccess; }
extern "C" hipError_t hipMemsetAsync(void *, int, size_t, hipStream_t) { return hipSuccess; }
extern "C" hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }

static void check(bool ok, const char *what) {
  if (ok) return;
  std::printf("FAILED: %s\n", what);
  std::exit(1);
}

// Squares of 128 that each matrix's products cover: [matrix, product].
using Cover = std::map<std::array<int, 2>, std::set<std::pair<int, int>>>;

static void check_list(const Plan &p, int kind, const std::vector<Tile> &list, int product, bool split, Cover &cover) {
  std::map<std::array<int, 3>, std::vector<Tile>> tiles;
  for (const Tile &t : list) tiles[{t.matrix, t.i, t.j}].push_back(t);
  const int rows = kRowsOf[kind], cols = product == 2 ? kColsOf[kind] : rows;
  std::set<int> slots;
  for (const auto &[key, shares] : tiles) {
    const Matrix &m = p.matrices[key[0]];
    const bool diagonal = !split && product != 2 && key[1] == key[2];  // counted in twos
    const int depth = (product == 0 ? m.kp : m.np) / kDeep / (diagonal ? 2 : 1);
    check((key[1] + 1) * rows <= m.np && (key[2] + 1) * cols <= (product == 2 ? m.kp : m.np), "a tile is inside");
    std::vector<char> seen(depth, 0);
    std::set<int> pieces;
    for (const Tile &t : shares) {
      check(t.at == m.at && t.np == m.np && t.kp == m.kp, "a tile has its matrix's places");
      check(t.pieces == static_cast<int>(shares.size()) && t.count >= 1 && t.piece >= 0 && t.piece < t.pieces, "shares");
      check(pieces.insert(t.piece).second, "a share is there once");
      if (t.pieces > 1) {
        check((t.slot + int64_t(t.pieces)) * rows * kColsOf[kind] <= p.partial_sums && t.slot == shares[0].slot, "its partial sums");
        check(t.ticket >= 0 && t.ticket < p.tickets && t.ticket == shares[0].ticket, "its ticket");
        check(slots.insert(t.slot + t.piece).second, "a place of partial sums has one share");
      }
      for (int q = t.first; q < t.first + t.count; ++q) {
        check(q >= 0 && q < depth && !seen[q], "a step is taken once");
        seen[q] = 1;
      }
    }
    for (char s : seen) check(s, "every step is taken");
    for (int a = 0; a < rows / 128; ++a)
      for (int b = 0; b < cols / 128; ++b)
        check(cover[{key[0], product}].insert({key[1] * rows / 128 + a, key[2] * cols / 128 + b}).second, "tiles are apart");
  }
}

int main() {
  std::mt19937 random(1);
  auto side = [&](int most) { return static_cast<int64_t>(1 + random() % (1 << (1 + random() % most))); };
  int small = 0, pairs = 0, wide = 0, large = 0, cut = 0;
  for (int round = 0; round < 440; ++round) {
    int n = 1 + random() % 6;
    const int most = round % 4 ? 13 : 8;
    std::vector<int64_t> rows(n), cols(n);
    for (int i = 0; i < n; ++i) rows[i] = side(most), cols[i] = side(most);
    if (round >= 400) {  // alike: small alone, in large tiles, wide
      n = round < 420 ? 3 : 40;
      const int64_t r = round < 410 ? 40 + random() % 24 : round < 420 ? 2048 + random() % 1000 : 512 + random() % 512;
      const int64_t c = round < 410 ? 30 + random() % 220 : (round < 420 ? 8192 : 4096) + random() % 4096;
      rows.assign(n, r), cols.assign(n, c);
    }
    slowmo_orth_config cfg{};
    cfg.steps = 1 + random() % 7;
    cfg.out_dtype = random() % 2;
    Plan p = plan(cfg, n, rows.data(), cols.data(), nullptr);
    check(p.total == plan(cfg, n, rows.data(), cols.data(), nullptr).total, "the same workspace each time");
    const bool split = cfg.out_dtype == SLOWMO_F32;
    Cover cover;
    for (int kind = 0; kind < kKinds; ++kind) {
      const Lists &l = p.lists[kind];
      const std::vector<Tile> *of[] = {&l.gram, &l.square, &l.update};
      for (int product = 0; product < 3; ++product) check_list(p, kind, *of[product], product, split, cover);
    }
    for (size_t i = 0; i < p.matrices.size(); ++i) {
      const Matrix &m = p.matrices[i];
      if (m.tiny || p.small) continue;
      const int at = static_cast<int>(i);
      const size_t a = m.np / 128, b = m.kp / 128;
      const size_t half = large_tiles(m) ? a / 2 * (a / 2 + 1) * 2 : a * (a + 1) / 2;
      check(cover[{at, 0}].size() == half && cover[{at, 1}].size() == half, "the lower half of a symmetric product");
      check(cover[{at, 2}].size() == a * b, "all of P X");
      std::set<std::pair<int, int>> patches;
      const int down = (m.tall ? m.kp : m.np) / kPatch, across = (m.tall ? m.np : m.kp) / kPatch;
      for (const Item &t : p.load)
        if (t.matrix == at)
          for (int q = t.j; q < t.j + kPatches && q < across; ++q)
            check(t.i < down && patches.insert({t.i, q}).second, "a patch is loaded once");
      check(patches.size() == static_cast<size_t>(down) * across, "every patch is loaded");
    }
    Steps steps = steps_of(cfg);
    const std::vector<Op> ops = program(steps, p.pairs, split);
    check(!ops.empty() && ops.back().update && ops.back().up.last, "the last launch writes the results");
    int updates = 0, from = 0;
    for (const Op &op : ops) {
      check((op.update ? op.up.from : op.symmetric.from) == from, "products read the X that was written");
      if (op.update) ++updates, from = 1 - from;
      if (!op.update) check(op.symmetric.out < (p.pairs ? kSquares : 2), "a buffer that is there");
    }
    check(updates == cfg.steps - (p.pairs ? 1 : 0), "as many steps as asked for");
    small += p.small, pairs += p.pairs, wide += !p.lists[kWide].update.empty();
    large += !p.lists[kLarge].gram.empty(), cut += p.tickets > 0;
  }
  std::printf("%d small, %d by pairs, %d wide, %d large, %d cut\n", small, pairs, wide, large, cut);
  check(small > 10 && pairs > 10 && wide > 0 && large > 10 && cut > 10, "every way was taken");
  std::puts("ok");
}
