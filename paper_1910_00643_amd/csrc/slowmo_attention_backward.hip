// The gradient of attention over packed sequences (include/slowmo_attention.h has the formulas).
//
// Two passes over the visible pairs, each the owner of what it sums, so that nothing is added by atomics: k_queries
// has 32 queries to a wave and goes over the keys (dQ; it also leaves each row's g . out and its statistics for the other
// pass), k_keys has 32 keys to a wave and goes over the rows of the query heads that share them (dK, dV).
// That is seven products of a pair for five: the scores and g V^T are computed twice.  bf16: nine, they are computed once more
// for an exact g . out.
//
// 8192 tokens of 16 heads of 128 on 4 key heads, bf16: k_queries 775 us, 887 TFLOP/s of its five products, 46 % of the matrix
// units' cycles and 51 % of the vector units', which take turns; k_keys 892 us, 616 of its four, 33 % and 37 %, half of its
// waves' time a wait; 30 us to add the pieces.
//
// bf16: P and dS are rounded to bf16 where they meet bf16 factors, and nothing else is: dQ, dK and dV are off by what these
// roundings and their own make, 2.4e-3 of their norm against 64 bits for normal inputs, where their own is 1.7e-3.  Keys with a
// vector in common, which dS, whose sum is 0, takes out of dQ but its rounding does not: 2.8e-3 (of deviation 1), 8.1e-3 (5).
#include "slowmo_attention.h"

namespace slowmo {
namespace attention {
namespace {

struct Args {
  Rows q, k, v, g, out, dq, dk, dv;
  const float *lse;
  const int64_t *q_offsets, *k_offsets;
  int32_t batch, heads, group, dim;
  u32 by_group;  // 2^32 / group, rounded up
  int64_t tokens, keys, first, slots;
  float scale, scale2;  // of scores; of scores to powers of two
  Mask mask;
  bool wide, clear;
  bool apart;  // the keys' rows are not the queries': another list of offsets, or the same one over another number of rows
  int32_t parts, stretch;  // stretches of a sequence's rows, and rows of one: a tile of keys has a workgroup for each
  float *lse2, *delta;  // [tokens][query heads]: lse in powers of two; g . out
  float *sums;          // [parts][keys][key heads][2][padded head]: dK and dV of a piece
};

template <typename T, int DP>
constexpr bool kTwoWaves = DP <= (sizeof(T) == 2 ? 128 : 64);  // 256 registers a lane are enough for two waves of a SIMD

template <typename T, int DP>
__global__ __launch_bounds__(256, (kTwoWaves<T, DP> ? 2 : 1)) void k_queries(Args a) {
  using L = Tile<T, DP>;
  using frag = typename Kind<T>::frag;
  constexpr int NB = DP / 32, KB = L::rows / 32;
  extern __shared__ __align__(1024) char smem[];
  const int lane = threadIdx.x & 63, low = lane & 31, high = lane >> 5;
  const int wave = uniform(static_cast<int>(threadIdx.x >> 6)), waves = blockDim.x >> 6, height = waves * 32;
  int head;
  int64_t slot;
  if (!head_slot(a.first + blockIdx.x, a.heads, a.slots, head, slot)) return;
  slot = a.slots - 1 - slot;
  const Place at = place_of(a.q_offsets, a.batch, a.tokens, a.group, height, slot);
  const int64_t rows = static_cast<int64_t>(at.n) * a.group, row0 = static_cast<int64_t>(at.tile) * height;
  if (at.b < 0 || row0 >= rows) return;
  const int row = wave * 32 + low, last_row = static_cast<int>(min(rows - row0, static_cast<int64_t>(height))) - 1;
  const bool mine = row <= last_row, idle = wave * 32 > last_row;
  const Split split(row0, a.group, a.by_group);
  const int token = split.token(min(row, last_row)), of = split.head(min(row, last_row), token);
  const int64_t qt = at.begin + token;
  const int qh = head * a.group + of;
  T *dq = static_cast<T *>(a.dq.data) + qt * a.dq.token + qh * a.dq.head;
  f32x16 acc[NB];
  if (at.b == a.batch) {
    if (!a.clear) return;
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[b] = f32x16{};
    store_columns<T, NB>(dq, acc, 0.f, a.dim, high, a.wide, mine);
    return;
  }
  int64_t k_begin = at.begin;
  int keys = at.n;
  if (a.apart) {
    k_begin = clamped(uniform(a.k_offsets[at.b]), 0, a.keys);
    keys = static_cast<int>(clamped(uniform(a.k_offsets[at.b + 1]), k_begin, a.keys) - k_begin);
  }
  const int far = keys - at.n;
  const Walk walk = walk_of(a.mask, split.t0 + far, split.token(last_row) + far, keys, L::rows);
  const Sight sight = sight_of(a.mask, token + far, keys);
  const Sight first = sight_of(a.mask, split.token(min(wave * 32, last_row)) + far, keys),
              last = sight_of(a.mask, split.token(min(wave * 32 + 31, last_row)) + far, keys);
  if (a.dim != DP) {
    for (int i = threadIdx.x; i < 4 * L::bytes / 16; i += blockDim.x) reinterpret_cast<u32x4 *>(smem)[i] = u32x4{0, 0, 0, 0};
    __syncthreads();
  }
  const T *k = static_cast<const T *>(a.k.data) + k_begin * a.k.token + head * a.k.head;
  const T *v = static_cast<const T *>(a.v.data) + k_begin * a.v.token + head * a.v.head;
  auto bring = [&](int u) SLOWMO_INLINE {
    char *to = smem + (u & 1) * 2 * L::bytes;
    const int j0 = walk.at(u) * L::rows, end = keys - 1 - j0;
    bring_rows<T, DP>(to, L::rows, k + j0 * a.k.token, a.dim, a.wide, [&](int r) { return min(r, end) * a.k.token; });
    bring_rows<T, DP>(to + L::bytes, L::rows, v + j0 * a.v.token, a.dim, a.wide, [&](int r) { return min(r, end) * a.v.token; });
  };
  if (walk.count) bring(0);  // beside the queries
  frag qf[DP / 16], gf[DP / 16];
  float delta = 0.f;
  {
    const T *q = static_cast<const T *>(a.q.data) + qt * a.q.token + qh * a.q.head;
    const T *g = static_cast<const T *>(a.g.data) + qt * a.g.token + qh * a.g.head;
    const T *o = static_cast<const T *>(a.out.data) + qt * a.out.token + qh * a.out.head;
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
      qf[s] = load_frag<T>(q, 16 * s + 8 * high, a.dim, a.wide);
      gf[s] = load_frag<T>(g, 16 * s + 8 * high, a.dim, a.wide);
      const frag of_out = load_frag<T>(o, 16 * s + 8 * high, a.dim, a.wide);
#pragma unroll
      for (int i = 0; i < 8; ++i) delta += static_cast<float>(gf[s][i]) * static_cast<float>(of_out[i]);
    }
  }
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) settle(qf[s]), settle(gf[s]);
  delta = both_sum(delta);
  const int64_t at_row = qt * (static_cast<int64_t>(a.heads) * a.group) + qh;
  float lse2 = a.lse[at_row] * kLog2E;
  settle(lse2);
  // g . out is off by what `out` was rounded by, and where keys or values have something in common, or few keys have a row's
  // weight, that is far from little beside dS, which is what is left when dP and g . out all but cancel.  A row's dS sums to 0, so
  // the sum of P (dP - g . out) is what g . out is off by.  bf16: a first pass, of the two products that dS takes, is for that
  // sum alone (2048 causal tokens, D = 128, keys and values around a vector of deviation 1 each: dQ off by 2.8e-3 of
  // its norm, which is the rounding of dS alone; 1.5e-2 where only rows are mended that it is 2^-8 of the sum of |dS| off in).
  // Five products for three: a step of 8192 tokens of 16 heads of 128 takes 1967 us for 1677.  fp32: the pass that
  // forms dQ sums it too, and is made again where it is more than 2^-21 of the sum of |dS|: dQ is then nearer 64 bits than
  // that of elementary fp32 operations is.
  constexpr bool kMends = sizeof(T) == 4;
  float off, size;
  bool forms = kMends;  // whether the pass forms dQ
  for (bool careful = false, mended = false, again = false;; again = true) {
    const bool there = again && !careful && walk.count <= 2;  // both tiles are in shared memory still
    if (again && walk.count && !there && !careful) bring(0);
    off = size = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[b] = f32x16{};
    for (int u = 0; u < walk.count; ++u) {
      if (careful) __syncthreads();
      else arrive();
      const int next = careful ? u : u + 1;
      if (next < walk.count && !there) bring(next);
      char *k_tile = smem + (u & 1) * 2 * L::bytes, *v_tile = k_tile + L::bytes, *column_tile = k_tile;
      const int j0 = walk.at(u) * L::rows, j1 = j0 + L::rows - 1;
      if (careful) {
        // The scores want the keys as they are: a wild one that a row of finite lse sees has -infinity there, and no weight.
        // The product with dS takes them from the next tile's place, which comes after this one here.
        arrive();
        // A row that sees one, and is not NaN anyway, sees it times 0.
        column_tile = smem + (~u & 1) * 2 * L::bytes;
        if (any_wild<T, DP, L::rows>(k_tile)) add_wild<T, DP, L::rows>(k_tile, acc, 0.f, [&](int r) { return sees(sight, j0 + r); });
        tame<T, DP, L::rows>(column_tile, k_tile);
      }
      if (idle || ((j0 > last.hi || j1 < first.lo) && j0 >= last.sinks)) continue;
      const bool all = (j0 >= last.lo && j1 <= first.hi) || j1 < first.sinks;
      // wide heads: addresses worked out anew for each tile; kept, they would be spilled to scratch
      int row_lane = low, column_lane = lane;
      if constexpr (DP * sizeof(T) >= 384) settle(row_lane), settle(column_lane);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        f32x16 s{}, dp{};
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int st = 0; st < DP / 16; ++st) {
          s = mma(row_frag<T, DP>(k_tile, 32 * kb + row_lane, st, high), qf[st], s);
          dp = mma(row_frag<T, DP>(v_tile, 32 * kb + row_lane, st, high), gf[st], dp);
        }
        read_ahead<T, DP / 8, 1, 1, 6>();
#pragma unroll
        for (int i = 0; i < 16; ++i)
          s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.scale2, -lse2)) * (dp[i] - delta);
        if (!all) {
          branch();
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!sees(sight, j0 + 32 * kb + 8 * (i / 4) + 4 * high + i % 4)) s[i] = 0.f;
        }
        if (kMends || !forms) {
#pragma unroll
          for (int i = 0; i < 16; ++i) off += s[i], size += fabsf(s[i]);
        }
        if (!forms) continue;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const frag ds = as_frag<T>(s, half);
#pragma unroll
          for (int b = 0; b < NB; ++b) acc[b] = mma(column_frag<T, DP>(column_tile, b, 2 * kb + half, column_lane), ds, acc[b]);
        }
        read_ahead<T, 2 * NB, 1, 2, 3>();
      }
    }
    off = both_sum(off);
    if (!forms) {
      delta += off, forms = true;
      __syncthreads();  // this pass's reads of shared memory are done
      continue;
    }
    if (!careful) {
      int any = 0;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) any |= wild(acc[b][i]);
      careful = __syncthreads_or(any);
      if (careful) continue;
    }
    if (!kMends) {
      off = 0.f;
      break;
    }
    const bool far_off = fabsf(off) > both_sum(size) * (1.f / (1 << 21));
    if (mended || !__syncthreads_or(far_off)) break;
    mended = true;
    if (far_off) delta += off;  // the other rows come out as they were
  }
  if (mine && !high) a.lse2[at_row] = lse2, a.delta[at_row] = delta + off;
  store_columns<T, NB>(dq, acc, a.scale, a.dim, high, a.wide, mine);
}

// Rows of a tile as the keys see them.
constexpr int kRows = 32;
struct Stats {
  float lse2[kRows], delta[kRows];
  int position[kRows];
};
constexpr int kNowhere = INT32_MIN + 1;  // of rows past the last one

// k_keys holds in shared memory its keys (their values are in registers: both would leave room for one wave of a SIMD,
// 1152 us for 16 heads on 8192 tokens of 128) and two tiles of 32 rows, or, where rows are 1 KB, one.
template <typename T, int DP>
struct Keys {
  using L = Tile<T, DP>;
  static constexpr int stages = L::row_bytes <= 512 ? 2 : 1, waves = L::row_bytes <= 512 ? 4 : 2;
  static constexpr int tile = kRows * L::row_bytes;
  static constexpr int bytes(int w) { return w * tile + stages * (2 * tile + static_cast<int>(sizeof(Stats))); }
};

// The rows, (token, head) by (token, head), whose queries see some key of j0..j_end, and the positions that see a key.
struct Seen {
  int64_t lo, hi;
};
// Their pieces z0 .. z0 + count - 1: without a window the stretches of a sequence's rows that they lie in, with one
// pieces of like length.
struct Pieces {
  int z0, count;
  int64_t lo, hi, per, base;
  __device__ __forceinline__ int64_t begin(int z) const { return max(lo, base + z * per); }
  __device__ __forceinline__ int64_t end(int z) const { return z == z0 + count - 1 ? hi : min(hi, base + (z + 1) * per); }
};
__device__ __forceinline__ Pieces pieces_of(const Seen &s, int window, int stretch, int parts) {
  Pieces p{0, 1, s.lo, s.hi, stretch, 0};
  if (s.hi <= s.lo) return p;
  if (window) {
    p.count = static_cast<int>(min(static_cast<int64_t>(parts), (s.hi - s.lo + stretch - 1) / stretch));
    p.per = ((s.hi - s.lo + p.count - 1) / p.count + kRows - 1) / kRows * kRows;
    p.base = s.lo;
  } else {
    p.z0 = static_cast<int>(min(s.lo / stretch, static_cast<int64_t>(parts - 1)));  // the last one has no end
    p.count = static_cast<int>(min((s.hi - 1) / stretch, static_cast<int64_t>(parts - 1))) - p.z0 + 1;
  }
  return p;
}
__device__ __forceinline__ int from_of(const Mask &m, int key) {
  return m.causal ? key : m.window && key >= m.sinks ? key - m.window + 1 : kNowhere + 1;
}
__device__ __forceinline__ int to_of(const Mask &m, int key) {
  return m.window && key >= m.sinks ? key + m.window - 1 : INT32_MAX;
}
__device__ __forceinline__ Seen seen_of(const Mask &m, int group, int j0, int j_end, int far, int n) {
  const int p_lo = from_of(m, j0), p_hi = j0 < m.sinks ? INT32_MAX : to_of(m, j_end);
  const int64_t lo = clamped(static_cast<int64_t>(p_lo) - far, 0, n), hi = clamped(static_cast<int64_t>(p_hi) - far + 1, lo, n);
  return {lo * group, hi * group};
}

__device__ __forceinline__ void word_to_shared(u32 shared, u32 offset, const float *base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(shared), "v"(offset), "s"(base) : "memory");
}

// WHAT: 1 dV, 2 dK, 3 both.
template <typename T, int DP, int WHAT>
__global__ __launch_bounds__((64 * Keys<T, DP>::waves), (kTwoWaves<T, DP> ? 2 : 1)) void k_keys(Args a) {
  using frag = typename Kind<T>::frag;
  constexpr int NB = DP / 32, S = Keys<T, DP>::stages, B = Keys<T, DP>::tile;
  extern __shared__ __align__(1024) char smem[];
  const int lane = threadIdx.x & 63, low = lane & 31, high = lane >> 5;
  const int wave = uniform(static_cast<int>(threadIdx.x >> 6)), waves = blockDim.x >> 6, width = waves * 32;
  int head;
  int64_t slot;
  if (!head_slot(a.first + blockIdx.x, a.heads, a.slots * a.parts, head, slot)) return;
  // the last rows, which the most keys are seen by, first, all tiles of keys over the same stretch of rows side by side
  const int part = a.parts - 1 - static_cast<int>(slot / a.slots);
  slot %= a.slots;
  const Place at = place_of(a.k_offsets, a.batch, a.keys, 1, width, slot);
  const int keys = at.n;
  const int j0 = at.tile * width;
  if (at.b < 0 || static_cast<int64_t>(at.tile) * width >= keys) return;
  const int j = j0 + wave * 32 + low;
  const bool mine = j < keys;
  const int jc = mine ? j : keys - 1;
  // this lane's row of dK, dV: worked out where it is written, for want of registers in between
  auto row_of = [&](const Rows &x) SLOWMO_INLINE { return static_cast<T *>(x.data) + (at.begin + jc) * x.token + head * x.head; };
  constexpr bool kV = WHAT & 1, kK = WHAT & 2;
  constexpr int NK = kK ? NB : 1, NV = kV ? NB : 1;
  f32x16 acck[NK], accv[NV];
  auto clear = [&]() SLOWMO_INLINE {
#pragma unroll
    for (int b = 0; b < NK; ++b) acck[b] = f32x16{};
#pragma unroll
    for (int b = 0; b < NV; ++b) accv[b] = f32x16{};
  };
  clear();
  if (at.b == a.batch) {
    if (!a.clear || part) return;
    if constexpr (kK) store_columns<T, NB>(row_of(a.dk), acck, 0.f, a.dim, high, a.wide, mine);
    if constexpr (kV) store_columns<T, NB>(row_of(a.dv), accv, 0.f, a.dim, high, a.wide, mine);
    return;
  }
  int64_t q_begin = at.begin;
  int n = keys;
  if (a.apart) {
    q_begin = clamped(uniform(a.q_offsets[at.b]), 0, a.tokens);
    n = static_cast<int>(clamped(uniform(a.q_offsets[at.b + 1]), q_begin, a.tokens) - q_begin);
  }
  const int far = keys - n;
  const Seen seen = seen_of(a.mask, a.group, j0, min(j0 + width, keys) - 1, far, n);
  const Pieces pieces = pieces_of(seen, a.mask.window, a.stretch, a.parts);
  if (part < pieces.z0 || part >= pieces.z0 + pieces.count) return;
  const int64_t r_lo = pieces.begin(part), r_hi = pieces.end(part);
  const int my_lo = mine ? from_of(a.mask, j) : 1, my_hi = mine ? to_of(a.mask, j) : 0;
  const int wj0 = j0 + wave * 32, wj1 = min(wj0 + 31, keys - 1);
  const bool whole = wj0 + 31 < keys;

  char *k_tile = smem, *ring = smem + waves * B;
  if (a.dim != DP) {
    for (int i = threadIdx.x; i < (waves + 2 * S) * B / 16; i += blockDim.x) reinterpret_cast<u32x4 *>(smem)[i] = u32x4{0, 0, 0, 0};
    __syncthreads();
  }
  bring_rows<T, DP>(k_tile, width, static_cast<const T *>(a.k.data) + (at.begin + j0) * a.k.token + head * a.k.head, a.dim, a.wide,
                    [&](int r) { return min(r, keys - 1 - j0) * a.k.token; });
  const T *q = static_cast<const T *>(a.q.data) + static_cast<int64_t>(head) * a.group * a.q.head;
  const T *g = static_cast<const T *>(a.g.data) + static_cast<int64_t>(head) * a.group * a.g.head;
  const int64_t stat0 = static_cast<int64_t>(head) * a.group, per_token = static_cast<int64_t>(a.heads) * a.group;
  const Split split(r_lo, a.group, a.by_group);
  const int step_t = kRows / a.group, step_o = kRows % a.group;
  Stats *stats = reinterpret_cast<Stats *>(ring + 2 * S * B);
  // The next tile's first row is the head o0 of token t0; `left` rows are left.
  int t0 = split.t0, o0 = split.o0;
  int64_t left = r_hi - r_lo;
  auto bring = [&](int u) SLOWMO_INLINE {
    char *to = ring + (u % S) * 2 * B;
    Stats *st = stats + u % S;
    const int end = static_cast<int>(min(left, static_cast<int64_t>(kRows))) - 1;  // rows past it take its place
    auto part_row = [&](int r, u32 &t, u32 &o) SLOWMO_INLINE {
      o = o0 + min(r, end);
      t = a.group > 1 ? __umulhi(o, a.by_group) : o;
      o -= t * a.group;
    };
    const int64_t qt = q_begin + t0;
    bring_rows<T, DP>(to, kRows, q + qt * a.q.token, a.dim, a.wide, [&](int r) {
      u32 t, o;
      part_row(r, t, o);
      return t * a.q.token + o * a.q.head;
    });
    bring_rows<T, DP>(to + B, kRows, g + qt * a.g.token, a.dim, a.wide, [&](int r) {
      u32 t, o;
      part_row(r, t, o);
      return t * a.g.token + o * a.g.head;
    });
    if (lane < kRows && (wave == 0 || wave == waves - 1)) {
      u32 t, o;
      part_row(lane, t, o);
      const u32 at = (t * static_cast<u32>(a.heads * a.group) + o) * 4;
      const int64_t s = qt * per_token + stat0;
      if (wave == 0) word_to_shared(uniform(offset_of(st->lse2)), at, uniform(a.lse2 + s));
      if (wave == waves - 1) word_to_shared(uniform(offset_of(st->delta)), at, uniform(a.delta + s));
      st->position[lane] = lane <= end ? t0 + static_cast<int>(t) + far : kNowhere;
    }
    left -= kRows;
    t0 += step_t, o0 += step_o;
    if (o0 >= a.group) o0 -= a.group, ++t0;
  };
  const int turns = r_hi > r_lo ? static_cast<int>((r_hi - r_lo + kRows - 1) / kRows) : 0;
  if (S == 2 && turns) bring(0);
  frag vf[DP / 16];
  {
    const T *v = row_of(a.v);
#pragma unroll
    for (int s = 0; s < (kK ? DP / 16 : 0); ++s) vf[s] = load_frag<T>(v, 16 * s + 8 * high, a.dim, a.wide);
#pragma unroll
    for (int s = 0; s < (kK ? DP / 16 : 0); ++s) settle(vf[s]);
  }
  for (bool careful = false;; careful = true) {
    if (careful) {
      t0 = split.t0, o0 = split.o0, left = r_hi - r_lo;
      if (S == 2 && turns) bring(0);
    }
    for (int u = 0; u < turns; ++u) {
      if (S == 1) {
        __syncthreads();
        bring(u);
      }
      arrive();
      if (S == 2 && u + 1 < turns) bring(u + 1);
      char *q_tile = ring + (u % S) * 2 * B, *g_tile = q_tile + B;
      const Stats *st = stats + u % S;
      auto sees_row = [&](int r) SLOWMO_INLINE {
        const int p = st->position[r];
        return p >= my_lo && p <= my_hi && p != kNowhere;
      };
      if (careful) {
        if (kK && any_wild<T, DP, kRows>(q_tile)) {
          if constexpr (kK) add_wild<T, DP, kRows>(q_tile, acck, 1.f, sees_row);
          __syncthreads();
          tame<T, DP, kRows>(q_tile, q_tile);
        }
        if (kV && any_wild<T, DP, kRows>(g_tile)) {
          if constexpr (kV) add_wild<T, DP, kRows>(g_tile, accv, 1.f, sees_row);
          __syncthreads();
          tame<T, DP, kRows>(g_tile, g_tile);
        }
      }
      const int pa = uniform(st->position[0]), pb = uniform(st->position[kRows - 1]);
      // every row sees every key of the wave, or (rows in order, none missing) none does
      bool all = whole && pb != kNowhere && (!a.mask.causal || wj1 <= pa);
      bool none = pa == kNowhere || wj0 >= keys || (pb != kNowhere && a.mask.causal && wj0 > pb);
      if (a.mask.window) {
        all = all && (wj1 < a.mask.sinks || (pb - wj0 < a.mask.window && wj1 - pa < a.mask.window));
        none = none || (wj0 >= a.mask.sinks && ((pa - wj1 >= a.mask.window) || (pb != kNowhere && wj0 - pb >= a.mask.window)));
      }
      if (none) continue;
      f32x16 s{}, dp{};
      // worked out anew each time: kept, the addresses would not fit the registers
      int k_row = wave * 32 + low, row_lane = low, column_lane = lane;
      settle(k_row);
      if constexpr (DP * sizeof(T) >= 256) settle(row_lane), settle(column_lane);
#pragma unroll
      for (int e = 0; e < DP / 16; ++e) {
        s = mma(row_frag<T, DP>(q_tile, row_lane, e, high), row_frag<T, DP>(k_tile, k_row, e, high), s);
        if constexpr (kK) dp = mma(row_frag<T, DP>(g_tile, row_lane, e, high), vf[e], dp);
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int r = 8 * c + 4 * high;
        const f32x4 l = *reinterpret_cast<const f32x4 *>(st->lse2 + r), d = *reinterpret_cast<const f32x4 *>(st->delta + r);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[4 * c + i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[4 * c + i], a.scale2, -l[i]));
          if constexpr (kK) dp[4 * c + i] = s[4 * c + i] * (dp[4 * c + i] - d[i]);
        }
      }
      if (!all) {
        branch();
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (!sees_row(8 * (i / 4) + 4 * high + i % 4)) s[i] = dp[i] = 0.f;
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const frag pf = as_frag<T>(s, half), df = as_frag<T>(dp, half);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          if constexpr (kV) accv[b] = mma(column_frag<T, DP>(g_tile, b, half, column_lane), pf, accv[b]);
          if constexpr (kK) acck[b] = mma(column_frag<T, DP>(q_tile, b, half, column_lane), df, acck[b]);
        }
      }
    }
    if (careful) break;
    int any = 0;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if constexpr (kK) any |= wild(acck[b][i]);
        if constexpr (kV) any |= wild(accv[b][i]);
      }
    if (!__syncthreads_or(any)) break;
    clear();
  }
  if (pieces.count == 1) {
    if constexpr (kK) store_columns<T, NB>(row_of(a.dk), acck, a.scale, a.dim, high, a.wide, mine);
    if constexpr (kV) store_columns<T, NB>(row_of(a.dv), accv, 1.f, a.dim, high, a.wide, mine);
  } else {
    float *to = a.sums + ((part * a.keys + at.begin + jc) * a.heads + head) * (2 * DP);
    if constexpr (kK) store_columns<float, NB>(to, acck, a.scale, DP, high, true, mine);
    if constexpr (kV) store_columns<float, NB>(to + DP, accv, 1.f, DP, high, true, mine);
  }
}

// The pieces of a key's sums added in their order: a workgroup a key of 32 keys' tile, 4 elements to a lane.
template <typename T, int DP>
__global__ __launch_bounds__(256) void k_add(Args a, int width) {
  constexpr int N = 2 * DP / 4, R = 256 / N;  // lanes of a key and head; such rows of a workgroup
  int head;
  int64_t slot;
  // a slot of 32 rows: those of a sequence's tile of keys, so that all have the same pieces
  if (!head_slot(a.first + blockIdx.x, a.heads, a.slots, head, slot)) return;
  const Place at = place_of(a.k_offsets, a.batch, a.keys, 1, 32, slot);
  const int keys = at.n, first = at.tile * 32;
  if (at.b < 0 || at.b == a.batch || static_cast<int64_t>(at.tile) * 32 >= keys) return;
  int64_t q_begin = at.begin;
  int n = keys;
  if (a.apart) {
    q_begin = clamped(uniform(a.q_offsets[at.b]), 0, a.tokens);
    n = static_cast<int>(clamped(uniform(a.q_offsets[at.b + 1]), q_begin, a.tokens) - q_begin);
  }
  const int j0 = first / width * width;
  const Pieces pieces =
      pieces_of(seen_of(a.mask, a.group, j0, min(j0 + width, keys) - 1, keys - n, n), a.mask.window, a.stretch, a.parts);
  if (pieces.count == 1) return;
  const int e = static_cast<int>(threadIdx.x % N) * 4, d = e % DP;
  if (threadIdx.x >= R * N || d >= a.dim) return;
  const Rows &to = e < DP ? a.dk : a.dv;
  for (int j = first + threadIdx.x / N; j < min(first + 32, keys); j += R) {
    const int64_t row = (at.begin + j) * a.heads + head;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    const int last = pieces.z0 + pieces.count;
#pragma unroll 4
    for (int p = pieces.z0; p < last; ++p) {
      const f32x4 more = *reinterpret_cast<const f32x4 *>(a.sums + (p * a.keys * a.heads + row) * (2 * DP) + e);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] += more[i];
    }
    T *x = static_cast<T *>(to.data) + (at.begin + j) * to.token + head * to.head + d;
    for (int i = 0; i < 4; ++i)
      if (d + i < a.dim) x[i] = static_cast<T>(sum[i]);
  }
}

struct Plan {
  int q_waves, k_waves, parts, stretch;
};
// A sequence's rows go by stretches, a workgroup for each and each tile of keys that some row of it sees: with a causal
// mask the first keys are seen by all queries, and the sinks of a window by all but a few, and tiles of keys that
// go over the same stretch side by side find it in their L2 (8192 tokens of 16 heads of 128, each tile of keys cut into
// pieces of its own: 67 % of reads missed the L2, 1318 us).  How long the sequences are is not known here, and each stretch
// too many is workgroups that find nothing to do: stretches are for twice the average, and the last one has no end.
Plan plan_for(const Mask &m, int64_t tokens, int64_t keys, int64_t group, int64_t heads, int64_t batch, int row_bytes) {
  Plan p;
  p.q_waves = waves_of(tokens, group, batch, 4);
  p.k_waves = waves_of(keys, 1, batch, row_bytes > 512 ? 2 : 4);
  const int64_t sequences = std::max<int64_t>(1, std::min(batch, keys)), width = p.k_waves * 32, n = tokens / sequences;
  const int64_t seen = m.window ? std::min<int64_t>(n, width + (m.causal ? 1 : 2) * static_cast<int64_t>(m.window)) : m.causal ? n / 2 : n;
  const int64_t turns = (keys / width + sequences) * heads * (seen * group / kRows + 1);
  // pieces short enough that a round of the card's 512 workgroups is not the whole of it
  int64_t stretch = std::clamp<int64_t>(turns / 1024, 24, 1 << 20) * kRows;
  // no more than a gigabyte of sums
  const int64_t layer = keys * heads * 2 * SLOWMO_MAX_ATTENTION_DIM * 4;
  const int64_t most = std::clamp<int64_t>((int64_t(1) << 30) / std::max<int64_t>(layer, 1), 1, 16);
  // rows that a tile is gone over by, where no sequence is longer than twice the average
  const int64_t rows = m.window && !m.sinks ? (width + 2 * static_cast<int64_t>(m.window)) * group
                                            : std::max<int64_t>(1, std::min(tokens, 2 * n) * group);
  if (!m.window) stretch = std::max(stretch, ((rows + most - 1) / most + kRows - 1) / kRows * kRows);
  p.parts = static_cast<int>(std::clamp<int64_t>((rows + stretch - 1) / stretch, 1, most));
  p.stretch = static_cast<int>(std::min<int64_t>(stretch, INT32_MAX / kRows * kRows));
  return p;
}
int row_bytes(int dim, int32_t dtype) { return padded(dim) * static_cast<int>(size_of(dtype)); }

hipError_t run(Args a, int32_t dtype, const Plan &p, hipStream_t stream) {
  hipError_t e = hipSuccess;
  auto room = [&](auto kernel, int bytes) {
    if (bytes > 64 * 1024)
      e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  };
  dispatch(dtype, a.dim, [&](auto kind, auto dp) {
    using T = decltype(kind);
    constexpr int DP = dp();
    using L = Tile<T, DP>;
    if (a.tokens) {
      room(k_queries<T, DP>, 4 * L::bytes);
      a.slots = slots_of(a.tokens, a.group, p.q_waves * 32, a.batch);
      const int64_t items = items_of(a.heads, a.slots);
      for (a.first = 0; a.first < items && e == hipSuccess; a.first += kMostBlocks) {
        k_queries<T, DP><<<static_cast<u32>(std::min(kMostBlocks, items - a.first)), 64 * p.q_waves, 4 * L::bytes, stream>>>(a);
        e = hipGetLastError();
      }
    }
    if (a.keys && e == hipSuccess) {
      const int bytes = Keys<T, DP>::bytes(p.k_waves);
      const auto go = [&](auto kernel) {
        room(kernel, bytes);
        a.slots = slots_of(a.keys, 1, p.k_waves * 32, a.batch);
        const int64_t items = items_of(a.heads, a.slots * a.parts);
        for (a.first = 0; a.first < items && e == hipSuccess; a.first += kMostBlocks) {
          kernel<<<static_cast<u32>(std::min(kMostBlocks, items - a.first)), 64 * p.k_waves, bytes, stream>>>(a);
          e = hipGetLastError();
        }
      };
      // Both sums of heads of 256 do not fit the registers: dV and dK by a pass each, five products for four without
      // scratch in the loop (4096 tokens of 8 heads of 256 on 2, bf16, the whole gradient 1670 -> 1068 us).  A fifth product
      // of fp32 takes longer than the scratch (5937 -> 6891).
      if constexpr (DP == 256 && sizeof(T) == 2) {
        go(k_keys<T, DP, 1>);
        if (e == hipSuccess) go(k_keys<T, DP, 2>);
      } else {
        go(k_keys<T, DP, 3>);
      }
      if (a.parts > 1) {
        a.slots = slots_of(a.keys, 1, 32, a.batch);
        const int64_t blocks = items_of(a.heads, a.slots);
        for (a.first = 0; a.first < blocks && e == hipSuccess; a.first += kMostBlocks) {
          k_add<T, DP><<<static_cast<u32>(std::min(kMostBlocks, blocks - a.first)), 256, 0, stream>>>(a, p.k_waves * 32);
          e = hipGetLastError();
        }
      }
    }
  });
  return e;
}

size_t stat_bytes(int64_t tokens, int64_t q_heads) { return (static_cast<size_t>(tokens) * q_heads * 4 + 15) / 16 * 16; }

}  // namespace
}  // namespace attention
}  // namespace slowmo

using namespace slowmo;
using namespace slowmo::attention;

extern "C" {

size_t slowmo_attention_backward_bytes(const slowmo_attention_config *cfg, int32_t batch, int64_t tokens, int64_t keys,
                                       int32_t q_heads, int32_t k_heads) {
  if (check_config(cfg) || batch < 0 || tokens < 0 || keys < 0 || tokens > kLongest || keys > kLongest || q_heads < 1 ||
      k_heads < 1 || q_heads > (1 << 20) || q_heads % k_heads)
    return 0;
  const Plan p = plan_for(mask_of(*cfg), tokens, keys, q_heads / k_heads, k_heads, batch, row_bytes(cfg->head_dim, cfg->dtype));
  return 2 * stat_bytes(tokens, q_heads) +
         (p.parts > 1 ? static_cast<size_t>(p.parts) * keys * k_heads * 2 * padded(cfg->head_dim) * sizeof(float) : 0);
}

slowmo_status slowmo_attention_backward(const slowmo_attention_config *cfg, int32_t batch, const int64_t *q_offsets,
                                        const int64_t *k_offsets, int64_t tokens, int64_t keys, const slowmo_heads *g,
                                        const slowmo_heads *q, const slowmo_heads *k, const slowmo_heads *v,
                                        const slowmo_heads *out, const float *lse, const slowmo_heads *dq,
                                        const slowmo_heads *dk, const slowmo_heads *dv, void *workspace,
                                        size_t workspace_bytes, void *stream) {
  return walled([&]() -> slowmo_status {
    auto bad = [](const char *msg) { return fail_thread(SLOWMO_ERR_ARG, msg); };
    if (const slowmo_status s = check_call(cfg, batch, q_offsets, k_offsets, tokens, keys)) return s;
    const slowmo_heads *in[] = {g, q, out, k, v}, *written[] = {dq, dk, dv};
    const int32_t d = cfg->head_dim, dt = cfg->dtype;
    for (int i = 0; i < 5; ++i)
      if (const slowmo_status s = check_rows(in[i], i < 3 ? tokens : keys, d, dt, false)) return s;
    for (int i = 0; i < 3; ++i)
      if (const slowmo_status s = check_rows(written[i], i < 1 ? tokens : keys, d, dt, true)) return s;
    if (q->heads != g->heads || q->heads != out->heads || q->heads != dq->heads || k->heads != v->heads ||
        k->heads != dk->heads || k->heads != dv->heads)
      return bad("g, out and dq have q's heads, v, dk and dv have k's");
    if (const slowmo_status s = check_group(tokens, q->heads, k->heads)) return s;
    if (tokens && !lse) return bad("lse is NULL");
    if (!aligned(lse, 4)) return fail_thread(SLOWMO_ERR_ALIGN, "lse must be 4-byte aligned");
    const size_t need = slowmo_attention_backward_bytes(cfg, batch, tokens, keys, q->heads, k->heads);
    if (need && !workspace) return bad("workspace is NULL");
    if (need && !aligned(workspace, 16)) return fail_thread(SLOWMO_ERR_ALIGN, "workspace must be 16-byte aligned");
    if (workspace_bytes < need) return fail_thread(SLOWMO_ERR_NOMEM, "workspace is smaller than slowmo_attention_backward_bytes()");
    Extent from[6], to[4];
    for (int i = 0; i < 5; ++i) from[i] = extent(*in[i], i < 3 ? tokens : keys, d, dt);
    from[5] = extent(lse, tokens * q->heads * sizeof(float));
    for (int i = 0; i < 3; ++i) to[i] = extent(*written[i], i < 1 ? tokens : keys, d, dt);
    to[3] = extent(workspace, need);
    for (int i = 0; i < 4; ++i) {
      for (const Extent &x : from)
        if (overlap(to[i], x)) return bad("an output or the workspace overlaps an input");
      for (int j = 0; j < i; ++j)
        if (overlap(to[i], to[j])) return bad("outputs, or one and the workspace, overlap");
    }
    if (!tokens && !keys) return SLOWMO_OK;
    Args a{};
    a.q = rows_of(*q), a.k = rows_of(*k), a.v = rows_of(*v), a.g = rows_of(*g), a.out = rows_of(*out);
    a.dq = rows_of(*dq), a.dk = rows_of(*dk), a.dv = rows_of(*dv);
    a.lse = lse, a.q_offsets = q_offsets, a.k_offsets = k_offsets ? k_offsets : q_offsets;
    a.apart = a.k_offsets != q_offsets || keys != tokens;
    a.batch = batch, a.heads = k->heads, a.group = q->heads / k->heads, a.dim = d;
    a.by_group = by_group(a.group);
    a.tokens = tokens, a.keys = keys;
    a.scale = cfg->scale, a.scale2 = cfg->scale * kLog2E;
    a.mask = mask_of(*cfg);
    a.clear = cfg->clear_rest != 0;
    a.wide = true;
    for (const slowmo_heads *h : in) a.wide = a.wide && wide_rows(*h, d, dt);
    for (const slowmo_heads *h : written) a.wide = a.wide && wide_rows(*h, d, dt);
    const Plan p = plan_for(a.mask, tokens, keys, a.group, a.heads, batch, row_bytes(d, dt));
    a.parts = p.parts, a.stretch = p.stretch;
    a.lse2 = static_cast<float *>(workspace);
    a.delta = a.lse2 + stat_bytes(tokens, q->heads) / 4;
    a.sums = a.delta + stat_bytes(tokens, q->heads) / 4;
    const hipError_t e = run(a, dt, p, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? SLOWMO_OK : fail_thread_hip(e, "slowmo_attention_backward");
  });
}

}  // extern "C"
