// New keys and values to their places in a paged cache, keys and queries turned by their positions on the way
// (include/slowmo_attention.h).
//
// Memory bounds it: every element is read once and written once.  A lane takes 16 bytes of a row, or, where it
// turns halves, 16 bytes of each, so that no lane needs another's elements.  Measured: 25 393 tokens of 32 + 8 + 8 heads of
// 128, bf16, 625 MB in 128 us, 4.9 TB/s; a large copy reaches 4.6 to 4.8.  48 single tokens: 6.4 us of a call's 13, the rest its
// launch and its checks.
#include "slowmo_attention.h"

namespace slowmo {
namespace attention {
namespace {

constexpr int kHeads = 4;  // heads of a lane: they share their angles, which are twice as many bytes as a head's elements

struct Args {
  Rows side[3], out[3];  // keys, values, queries; where they go (queries: by token)
  int64_t page_stride[2];
  int32_t heads[3], groups[3];  // groups of kHeads
  const int64_t *offsets, *lengths;
  const int32_t *pages;
  const float *table;
  int64_t table_rows, pages_stride, tokens, first;
  int32_t columns, n_pages[2], page_log2, batch, dim, rot;
  int32_t turned, plain;  // pieces of a row that is turned, and of one that is not
  int32_t every;          // lanes of a token: a piece of kHeads heads each
  bool clear;
};

template <typename T, int V, bool WIDE>
struct alignas(WIDE ? V * sizeof(T) : sizeof(T)) Piece {
  T e[V];
};

// INTER: pairs lie beside each other.  A piece is V elements, of a turned stretch in halves V of each half; not
// WIDE: one pair, and one element of what is not turned, at any alignment.
template <typename T, int V, bool INTER, bool WIDE>
__global__ __launch_bounds__(256) void k_append(Args a) {
  using P = Piece<T, V, WIDE>;
  constexpr int C = WIDE ? V : 1;
  using Copy = Piece<T, C, WIDE>;
  const int64_t base = (a.first + blockIdx.x) * 256;
  const int64_t t0 = base >> 32 ? base / a.every : static_cast<u32>(base) / static_cast<u32>(a.every);
  const u32 in = static_cast<u32>(base - t0 * a.every) + threadIdx.x;
  const int64_t t = t0 + in / a.every;
  int piece = static_cast<int>(in % a.every);
  // which rows, which piece of them
  int which = 0, per = a.turned;
  const int keys = a.groups[0] * a.turned, values = a.groups[1] * a.plain;
  if (piece >= keys + values) which = 2, piece -= keys + values;
  else if (piece >= keys) which = 1, piece -= keys, per = a.plain;
  const int head = piece / per * kHeads, heads = min(kHeads, a.heads[which] - head);
  piece %= per;
  const int half = a.rot / 2, pieces = INTER ? a.rot / V : half / V;  // that turn
  const bool turns = which != 1 && piece < pieces;
  const int d = turns ? piece * V : which == 1 ? piece * C : a.rot + (piece - pieces) * C;
  // The elements are asked for beside the token's place, which takes several trips to memory one after the other; those of
  // rows behind the last sequence, which may not be there yet, are not (no difference for 48 or 25 393 tokens).
  P x[kHeads], y[kHeads];
  if (t < min(a.tokens, a.offsets[a.batch])) {
    const T *from = static_cast<const T *>(a.side[which].data) + t * a.side[which].token + head * a.side[which].head + d;
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
      if (h >= heads) continue;
      if (turns) {
        x[h] = *reinterpret_cast<const P *>(from + h * a.side[which].head);
        if constexpr (!INTER) y[h] = *reinterpret_cast<const P *>(from + h * a.side[which].head + half);
      } else {
        __builtin_memcpy(&x[h], reinterpret_cast<const Copy *>(from + h * a.side[which].head), sizeof(Copy));
      }
    }
  }
  // the first token's sequence by all lanes, then on from there
  const int lane = threadIdx.x & 63;
  // (the copy of the pointer keeps the arguments out of scratch memory: 306 us for 131 with a captured)
  const int64_t *offsets = a.offsets;
  int b = stretch_of(a.batch, [=](int i) { return offsets[i] <= t0; }) - 1;
  for (int first = b + 1; first <= a.batch; first += 64) {
    const int got = __popcll(__ballot(first + lane <= a.batch && a.offsets[min(first + lane, a.batch)] <= t0));
    b += got;
    if (got < 64) break;
  }
  if (t >= a.tokens || b < 0) return;
  for (int steps = 0; steps < 4 && b < a.batch && a.offsets[b + 1] <= t; ++steps) ++b;
  if (b < a.batch && a.offsets[b + 1] <= t) {
    int lo = b + 1, hi = a.batch;  // the last entry that is not past t
    while (lo < hi) {
      const int mid = lo + (hi - lo + 1) / 2;
      if (a.offsets[mid] <= t) lo = mid;
      else hi = mid - 1;
    }
    b = lo;
  }
  const bool rest = b >= a.batch;  // behind the last sequence
  if (rest && (!a.clear || which != 2)) return;
  const int64_t begin = rest ? 0 : a.offsets[b], end = rest ? 0 : a.offsets[b + 1], position = rest ? 0 : a.lengths[b] - (end - t);
  T *to = static_cast<T *>(a.out[which].data) + head * a.out[which].head + d;
  if (which == 2) {
    to += t * a.out[2].token;
  } else {
    const int64_t column = position >> a.page_log2;
    if (t < begin || position < 0 || column >= a.columns) return;
    const int page = a.pages[b * a.pages_stride + column];
    if (static_cast<u32>(page) >= static_cast<u32>(a.n_pages[which])) return;
    to += page * a.page_stride[which] + (position & ((int64_t(1) << a.page_log2) - 1)) * a.out[which].token;
  }
  const int64_t next = a.out[which].head;
  if (!turns || rest) {
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
      if (h >= heads) continue;
      if (rest) x[h] = y[h] = P{};
      Copy copy;
      __builtin_memcpy(&copy, &x[h], sizeof(Copy));
      if (!turns) *reinterpret_cast<Copy *>(to + h * next) = copy;
      if (turns) *reinterpret_cast<P *>(to + h * next) = x[h];
      if constexpr (!INTER)
        if (turns) *reinterpret_cast<P *>(to + h * next + half) = y[h];
    }
    return;
  }
  const bool known = position >= 0 && position < a.table_rows;
  const float *cos = a.table + (known ? position : 0) * a.rot, *sin = cos + half;
  constexpr int N = INTER ? V / 2 : V;
  const int pair = piece * N;
  float c[N], s[N];
#pragma unroll
  for (int i = 0; i < N; ++i) c[i] = s[i] = __builtin_nanf("");
  if (known) {
    __builtin_memcpy(c, __builtin_assume_aligned(cos + pair, 4), sizeof(c));
    __builtin_memcpy(s, __builtin_assume_aligned(sin + pair, 4), sizeof(s));
  }
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    if (h >= heads) continue;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      T &first = INTER ? x[h].e[2 * i] : x[h].e[i], &second = INTER ? x[h].e[2 * i + 1] : y[h].e[i];
      const float u = static_cast<float>(first), v = static_cast<float>(second);
      first = static_cast<T>(u * c[i] - v * s[i]);
      second = static_cast<T>(u * s[i] + v * c[i]);
    }
    *reinterpret_cast<P *>(to + h * next) = x[h];
    if constexpr (!INTER) *reinterpret_cast<P *>(to + h * next + half) = y[h];
  }
}

template <typename T>
hipError_t launch(Args a, bool wide, bool inter, hipStream_t stream) {
  constexpr int W = 16 / sizeof(T);
  // narrow: single elements, pairs beside each other two at a time
  const int v = wide ? W : inter ? 2 : 1, rest = wide ? W : 1;
  hipError_t e = hipSuccess;
  const int turning = inter ? a.rot / v : a.rot / 2 / v;
  a.turned = turning + (a.dim - a.rot) / rest;
  a.plain = a.dim / rest;
  for (int i = 0; i < 3; ++i) a.groups[i] = (a.heads[i] + kHeads - 1) / kHeads;
  a.every = (a.groups[0] + a.groups[2]) * a.turned + a.groups[1] * a.plain;
  const int64_t blocks = (a.tokens * a.every + 255) / 256;
  for (a.first = 0; a.first < blocks && e == hipSuccess; a.first += kMostBlocks) {
    const u32 n = static_cast<u32>(std::min(kMostBlocks, blocks - a.first));
    if (wide && inter) k_append<T, W, true, true><<<n, 256, 0, stream>>>(a);
    else if (wide) k_append<T, W, false, true><<<n, 256, 0, stream>>>(a);
    else if (inter) k_append<T, 2, true, false><<<n, 256, 0, stream>>>(a);
    else k_append<T, 1, false, false><<<n, 256, 0, stream>>>(a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace
}  // namespace attention
}  // namespace slowmo

using namespace slowmo;
using namespace slowmo::attention;

extern "C" {

slowmo_status slowmo_cache_append(const slowmo_append_config *cfg, const slowmo_pages *pages, int64_t tokens,
                                  const slowmo_heads *k, const slowmo_heads *v, const slowmo_cache *k_cache,
                                  const slowmo_cache *v_cache, const slowmo_heads *q, const slowmo_heads *q_out,
                                  void *stream) {
  return walled([&]() -> slowmo_status {
    auto bad = [](const char *msg) { return fail_thread(SLOWMO_ERR_ARG, msg); };
    if (!cfg) return bad("cfg is NULL");
    if (cfg->dtype != SLOWMO_F32 && cfg->dtype != SLOWMO_BF16) return bad("unknown dtype");
    if (cfg->head_dim < 1 || cfg->head_dim > SLOWMO_MAX_HEAD_DIM) return bad("head_dim must be in 1..SLOWMO_MAX_HEAD_DIM");
    if (cfg->rotary_dim < 0 || cfg->rotary_dim > cfg->head_dim || cfg->rotary_dim % 2)
      return bad("rotary_dim must be even and in 0..head_dim");
    if (cfg->interleaved != 0 && cfg->interleaved != 1) return bad("interleaved must be 0 or 1");
    if (cfg->clear_rest != 0 && cfg->clear_rest != 1) return bad("clear_rest must be 0 or 1");
    if (const slowmo_status s = check_pages(pages, tokens)) return s;
    if (cfg->rotary_dim) {
      if (cfg->table_rows < 0 || cfg->table_rows > (int64_t(1) << 40)) return bad("table_rows must be in 0..2^40");
      if (tokens && cfg->table_rows && !cfg->table) return bad("table is NULL");
      if (!aligned(cfg->table, 4)) return fail_thread(SLOWMO_ERR_ALIGN, "the table is not 4-byte aligned");
    }
    if (!q != !q_out) return bad("q and q_out go together");
    const int32_t d = cfg->head_dim, dt = cfg->dtype;
    const slowmo_heads *rows[] = {k, v, q, q_out};
    for (int i = 0; i < (q ? 4 : 2); ++i)
      if (const slowmo_status s = check_rows(rows[i], tokens, d, dt, i == 3)) return s;
    const slowmo_cache *caches[] = {k_cache, v_cache};
    for (const slowmo_cache *c : caches)
      if (const slowmo_status s = check_cache(c, d, dt, true)) return s;
    if (k_cache->heads != k->heads || v_cache->heads != v->heads) return bad("a cache has other heads than what is appended");
    if (k_cache->page != v_cache->page) return bad("the caches have the same page");
    if (q && q->heads != q_out->heads) return bad("q_out has q's heads");
    const Extent out[] = {extent(*k_cache, d, dt), extent(*v_cache, d, dt), q ? extent(*q_out, tokens, d, dt) : Extent{}};
    const Extent in[] = {extent(*k, tokens, d, dt), extent(*v, tokens, d, dt), q ? extent(*q, tokens, d, dt) : Extent{}};
    const bool same = q && q->data == q_out->data && q->token_stride == q_out->token_stride && q->head_stride == q_out->head_stride;
    for (int i = 0; i < 3; ++i)
      for (int j = 0; j < 3; ++j) {
        if (overlap(out[i], in[j]) && !(i == 2 && j == 2 && same)) return bad("an output overlaps an input");
        if (i < j && overlap(out[i], out[j])) return bad("the outputs overlap");
      }
    if (!tokens || (!pages->batch && !(q && cfg->clear_rest))) return SLOWMO_OK;
    Args a{};
    a.clear = q && cfg->clear_rest;
    const slowmo_heads *sides[] = {k, v, q};
    for (int i = 0; i < 3; ++i)
      if (sides[i]) a.side[i] = rows_of(*sides[i]), a.heads[i] = sides[i]->heads;
    for (int i = 0; i < 2; ++i) {
      a.out[i] = {caches[i]->data, caches[i]->token_stride, caches[i]->head_stride};
      a.page_stride[i] = caches[i]->page_stride;
      a.n_pages[i] = static_cast<int32_t>(caches[i]->pages);
    }
    if (q) a.out[2] = rows_of(*q_out);
    a.offsets = pages->offsets, a.lengths = pages->lengths, a.pages = pages->pages, a.pages_stride = pages->stride;
    a.table = cfg->table, a.table_rows = cfg->table_rows, a.tokens = tokens;
    a.columns = pages->columns, a.batch = pages->batch, a.dim = d, a.rot = cfg->rotary_dim;
    while ((1 << a.page_log2) < k_cache->page) ++a.page_log2;
    const int w = 16 / static_cast<int>(size_of(dt));
    bool wide = d % w == 0 && cfg->rotary_dim % (cfg->interleaved ? w : 2 * w) == 0;
    for (int i = 0; i < (q ? 4 : 2); ++i) wide = wide && wide_rows(*rows[i], d, dt);
    for (const slowmo_cache *c : caches) wide = wide && wide_rows(*c, d, dt);
    const hipError_t e = dt == SLOWMO_BF16 ? launch<__bf16>(a, wide, cfg->interleaved, static_cast<hipStream_t>(stream))
                                           : launch<float>(a, wide, cfg->interleaved, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? SLOWMO_OK : fail_thread_hip(e, "slowmo_cache_append");
  });
}

}  // extern "C"
