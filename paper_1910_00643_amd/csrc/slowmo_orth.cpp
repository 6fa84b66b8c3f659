// C ABI of the orthogonalising call: argument checks, the workspace's layout, the lists of
// workgroups of every phase.  The arithmetic is in slowmo_orth.hip.
#include "slowmo_orth.h"

#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <cstring>
#include <memory>
#include <vector>

#include "../../include/slowmo_operators.h"
#include "slowmo_status.h"

using namespace slowmo;
using namespace slowmo::orth;

struct slowmo_orth {
  slowmo_orth_config cfg;
  Steps steps{};
  std::vector<Matrix> matrices;     // those that are not empty
  std::vector<int32_t> index;       // their places in the caller's list
  int32_t n_matrices = 0, tile = 0;
  Call call{};
  const Item *patches = nullptr, *padded = nullptr, *gram = nullptr, *square = nullptr, *update = nullptr;
  const int32_t *tiny = nullptr;
  int32_t n_tiny = 0, n_patches = 0, n_padded = 0, n_gram = 0, n_square = 0, n_update = 0;
};

namespace {

constexpr int64_t kMostSide = 65536;
constexpr size_t kAlign = 256;
const float kDefault[3] = {3.4445f, -4.7750f, 2.0315f};

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// Everything a handle needs, laid out from the configuration and the shapes alone.
struct Plan {
  int32_t tile = 128;
  std::vector<Matrix> matrices;
  std::vector<int32_t> index;
  std::vector<Item> patches, padded, gram, square, update;
  std::vector<int32_t> tiny;
  size_t tiny_at = 0, matrices_at = 0, addresses_at = 0, squares_at = 0, inverse_at = 0, patches_at = 0, padded_at = 0,
         gram_at = 0, square_at = 0, update_at = 0, arena_at = 0, total = 0;
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

float factor(const slowmo_orth_config &c, int64_t rows, int64_t cols) {
  const double r = static_cast<double>(rows), k = static_cast<double>(cols);
  return static_cast<float>(c.scale == SLOWMO_SCALE_NONE    ? 1.
                            : c.scale == SLOWMO_SCALE_SHAPE ? std::sqrt(std::max(1., r / k))
                                                            : 0.2 * std::sqrt(std::max(r, k)));
}

// Tiles of a grid in blocks of 4 x 8, which 32 neighbouring workgroups share factors in.
template <typename F>
void walk(int32_t down, int32_t across, F &&f) {
  for (int32_t a0 = 0; a0 < down; a0 += 4)
    for (int32_t b0 = 0; b0 < across; b0 += 8)
      for (int32_t a = a0; a < std::min(down, a0 + 4); ++a)
        for (int32_t b = b0; b < std::min(across, b0 + 8); ++b) f(a, b);
}

// Workgroups go to the 8 dies in turn: of every 256, each die gets 32 neighbours of the list.
std::vector<Item> spread(const std::vector<Item> &v) {
  std::vector<Item> out(v.size());
  for (size_t base = 0; base < v.size(); base += 256) {
    const size_t count = std::min<size_t>(256, v.size() - base), each = count / 8, more = count % 8;
    for (size_t b = 0; b < count; ++b) {
      const size_t die = b % 8;
      out[base + b] = v[base + die * each + std::min(die, more) + b / 8];
    }
  }
  return out;
}

// The products' workgroups, those of long sums first.
void order(Plan &p) {
  std::vector<int32_t> by(p.matrices.size());
  for (size_t i = 0; i < by.size(); ++i) by[i] = static_cast<int32_t>(i);
  auto grams = by, updates = by;
  std::stable_sort(grams.begin(), grams.end(), [&](int32_t a, int32_t b) { return p.matrices[a].kp > p.matrices[b].kp; });
  std::stable_sort(updates.begin(), updates.end(), [&](int32_t a, int32_t b) { return p.matrices[a].np > p.matrices[b].np; });
  std::vector<Item> gram, square, update;
  for (int32_t at : grams) {
    const int32_t n = p.matrices[at].np / p.tile;
    walk(n, n, [&](int32_t i, int32_t j) {
      if (j <= i) gram.push_back({at, i, j, 0});
    });
  }
  for (int32_t at : updates) {
    const int32_t n = p.matrices[at].np / p.tile, k = p.matrices[at].kp / p.tile;
    walk(n, n, [&](int32_t i, int32_t j) {
      if (j <= i) square.push_back({at, i, j, 0});
    });
    walk(n, k, [&](int32_t i, int32_t j) { update.push_back({at, i, j, 0}); });
  }
  p.gram = spread(gram);
  p.square = spread(square);
  p.update = spread(update);
}

Plan plan(const slowmo_orth_config &c, int32_t n_matrices, const int64_t *rows, const int64_t *cols,
          const int64_t *ld) {
  Plan p;
  const bool split = c.out_dtype == SLOWMO_F32;
  if (const char *force = std::getenv("SLOWMO_ORTH_TILE")) p.tile = std::atoi(force);
  int64_t halves = 0;
  auto take = [&](int64_t count) {
    const int64_t at = halves;
    halves += up(count, kAlign / sizeof(uint16_t));
    return at;
  };
  for (int32_t i = 0; i < n_matrices; ++i) {
    if (!rows[i] || !cols[i]) continue;
    Matrix m{};
    m.tall = rows[i] > cols[i];
    m.n = static_cast<int32_t>(std::min(rows[i], cols[i]));
    m.k = static_cast<int32_t>(std::max(rows[i], cols[i]));
    const int32_t at = static_cast<int32_t>(p.matrices.size());
    if (m.n <= kTinySide && static_cast<int64_t>(m.n) * m.k <= kTinyElements) {
      m.ld = ld ? ld[i] : cols[i];
      m.scale = factor(c, rows[i], cols[i]);
      p.tiny.push_back(at);
      p.matrices.push_back(m);
      p.index.push_back(i);
      continue;
    }
    m.np = static_cast<int32_t>(up(m.n, p.tile));
    m.kp = static_cast<int32_t>(up(m.k, p.tile));
    m.ld = ld ? ld[i] : cols[i];
    m.scale = factor(c, rows[i], cols[i]);
    const int64_t wide = static_cast<int64_t>(m.np) * m.kp, square = static_cast<int64_t>(m.np) * m.np;
    for (int64_t &to : m.x) to = take(wide);
    m.a = take(square);
    m.p = take(square);
    m.x_lo[0] = take(wide);
    if (split) {
      m.x_lo[1] = take(wide);
      m.a_lo = take(square);
      m.p_lo = take(square);
    }
    m.first_patch = static_cast<int32_t>(p.patches.size());
    auto cover = [&](std::vector<Item> &to, int64_t down, int64_t across) {
      for (int64_t a = 0; a < down; a += kPatch)
        for (int64_t b = 0; b < across; b += kPatch)
          to.push_back({at, static_cast<int32_t>(a / kPatch), static_cast<int32_t>(b / kPatch), 0});
    };
    cover(p.patches, rows[i], cols[i]);
    cover(p.padded, m.tall ? m.kp : m.np, m.tall ? m.np : m.kp);
    m.patches = static_cast<int32_t>(p.patches.size()) - m.first_patch;
    p.matrices.push_back(m);
    p.index.push_back(i);
  }
  order(p);
  size_t off = 0;
  auto section = [&](size_t bytes) {
    const size_t at = off;
    off += static_cast<size_t>(up(static_cast<int64_t>(std::max<size_t>(bytes, 1)), kAlign));
    return at;
  };
  p.matrices_at = section(p.matrices.size() * sizeof(Matrix));
  p.addresses_at = section(p.matrices.size() * sizeof(Addresses));
  p.squares_at = section(p.patches.size() * sizeof(double));
  p.inverse_at = section(p.matrices.size() * sizeof(float));
  p.tiny_at = section(p.tiny.size() * sizeof(int32_t));
  p.patches_at = section(p.patches.size() * sizeof(Item));
  p.padded_at = section(p.padded.size() * sizeof(Item));
  p.gram_at = section(p.gram.size() * sizeof(Item));
  p.square_at = section(p.square.size() * sizeof(Item));
  p.update_at = section(p.update.size() * sizeof(Item));
  p.arena_at = section(static_cast<size_t>(halves) * sizeof(uint16_t));
  p.total = off;
  return p;
}

slowmo_status run(slowmo_orth *h, const void *const *in, float *const *momentum, void *const *out, float mu,
                  int32_t nesterov, void *stream_) {
  const bool with_momentum = momentum != nullptr;
  const size_t in_size = h->cfg.in_dtype == SLOWMO_BF16 ? 2 : 4, out_size = h->cfg.out_dtype == SLOWMO_BF16 ? 2 : 4;
  const int32_t count = static_cast<int32_t>(h->matrices.size());
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
  const bool split = h->cfg.out_dtype == SLOWMO_F32;
  hipError_t e = hipSuccess;
  auto ok = [&](hipError_t got) { return (e = got) == hipSuccess; };
  for (int32_t first = 0; first < count; first += kInline) {
    Few few{};
    const int32_t some = std::min(kInline, count - first);
    for (int32_t i = 0; i < some; ++i) {
      const int32_t at = h->index[first + i];
      few.at[i] = {in[at], with_momentum ? momentum[at] : nullptr, out[at]};
    }
    if (!ok(launch_addresses(c, few, first, some, s))) return fail_thread_hip(e, "slowmo_orthogonalize");
  }
  if (h->n_tiny && !ok(launch_tiny(c, h->steps, h->tiny, h->n_tiny, s)))
    return fail_thread_hip(e, "slowmo_orthogonalize");
  if (h->n_tiny == count) return SLOWMO_OK;
  if (!ok(launch_squares(c, h->patches, h->n_patches, s)) || !ok(launch_norms(c, count, s)) ||
      !ok(launch_load(c, h->padded, h->n_padded, s)))
    return fail_thread_hip(e, "slowmo_orthogonalize");
  for (int32_t t = 0; t < h->steps.count; ++t) {
    const float *k = h->steps.abc[t];
    // Pairs of halves have bits enough; of single ones the last two steps, whose roundings grow no more.
    auto carries = [&](int32_t step) { return !split && step < h->steps.count - 2; };
    const Step st{k[0], k[1], k[2], t & 1, t + 1 == h->steps.count, carries(t), carries(t + 1)};
    if (!ok(launch_products(c, h->tile, kGram, st, h->gram, h->n_gram, split, s)) ||
        !ok(launch_products(c, h->tile, kPolynomial, st, h->square, h->n_square, split, s)) ||
        !ok(launch_products(c, h->tile, kUpdate, st, h->update, h->n_update, split, s)))
      return fail_thread_hip(e, "slowmo_orthogonalize");
  }
  return SLOWMO_OK;
}

}  // namespace

extern "C" {

size_t slowmo_orth_bytes(const slowmo_orth_config *cfg, int32_t n_matrices, const int64_t *rows,
                         const int64_t *cols, const int64_t *ld) {
  size_t bytes = 0;
  walled([&]() -> slowmo_status {
    if (const char *bad = check(cfg, n_matrices, rows, cols, ld)) return fail_thread(SLOWMO_ERR_ARG, bad);
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
    if (const char *bad = check(cfg, n_matrices, rows, cols, ld)) return fail_thread(SLOWMO_ERR_ARG, bad);
    if (!workspace) return fail_thread(SLOWMO_ERR_ARG, "workspace is NULL");
    if (reinterpret_cast<uintptr_t>(workspace) % kAlign)
      return fail_thread(SLOWMO_ERR_ALIGN, "workspace must be 256-byte aligned");
    Plan p = plan(*cfg, n_matrices, rows, cols, ld);
    if (workspace_bytes < p.total)
      return fail_thread(SLOWMO_ERR_NOMEM, "workspace is smaller than slowmo_orth_bytes()");
    if (slowmo_status st = slowmo_check_device_range(workspace, p.total); st != SLOWMO_OK) return st;
    std::unique_ptr<slowmo_orth> h(new slowmo_orth);
    h->cfg = *cfg;
    h->cfg.coefficients = nullptr;
    h->steps.count = cfg->steps;
    for (int32_t t = 0; t < cfg->steps; ++t)
      for (int i = 0; i < 3; ++i)
        h->steps.abc[t][i] = cfg->coefficients ? cfg->coefficients[3 * t + i] : kDefault[i];
    h->n_matrices = n_matrices;
    h->tile = p.tile;
    if (hipError_t e = prepare_products(p.tile, cfg->out_dtype == SLOWMO_F32); e != hipSuccess)
      return fail_thread_hip(e, "slowmo_orth_create");
    h->matrices = p.matrices;
    h->index = p.index;
    char *base = static_cast<char *>(workspace);
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = hipSuccess;
    auto put = [&](size_t at, const void *from, size_t bytes) {
      if (bytes && e == hipSuccess) e = hipMemcpyAsync(base + at, from, bytes, hipMemcpyHostToDevice, s);
    };
    put(p.matrices_at, p.matrices.data(), p.matrices.size() * sizeof(Matrix));
    auto items = [&](size_t at, const std::vector<Item> &v, const Item *&to, int32_t &count) {
      put(at, v.data(), v.size() * sizeof(Item));
      to = reinterpret_cast<const Item *>(base + at);
      count = static_cast<int32_t>(v.size());
    };
    put(p.tiny_at, p.tiny.data(), p.tiny.size() * sizeof(int32_t));
    h->tiny = reinterpret_cast<const int32_t *>(base + p.tiny_at);
    h->n_tiny = static_cast<int32_t>(p.tiny.size());
    items(p.patches_at, p.patches, h->patches, h->n_patches);
    items(p.padded_at, p.padded, h->padded, h->n_padded);
    items(p.gram_at, p.gram, h->gram, h->n_gram);
    items(p.square_at, p.square, h->square, h->n_square);
    items(p.update_at, p.update, h->update, h->n_update);
    hipError_t waited = hipStreamSynchronize(s);  // the tables are in ordinary memory that ends here
    if (e == hipSuccess) e = waited;
    if (e != hipSuccess) return fail_thread_hip(e, "slowmo_orth_create");
    h->call.matrices = reinterpret_cast<const Matrix *>(base + p.matrices_at);
    h->call.addresses = reinterpret_cast<Addresses *>(base + p.addresses_at);
    h->call.squares = reinterpret_cast<double *>(base + p.squares_at);
    h->call.inverse = reinterpret_cast<float *>(base + p.inverse_at);
    h->call.arena = reinterpret_cast<_Float16 *>(base + p.arena_at);
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
