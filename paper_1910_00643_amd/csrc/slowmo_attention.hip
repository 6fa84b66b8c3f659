// Attention over packed sequences and over a paged cache (include/slowmo_attention.h has the formulas).
//
// One pass over the keys with the running maximum and sum of the softmax.  A workgroup has the rows of one key
// head's query heads (token by token, its heads within), 32 to a wave; the keys and values go by tiles of 64
// through shared memory, the next tile's on their way while the current one is used.  Scores, probabilities and the
// result's sums stay in a wave's registers.  Where rows are few the key axis is cut into pieces, which a second kernel joins.
//
// Long prompts are bound by the matrix and the vector units of a SIMD, which take turns (43 % and 51 % of the cycles), at the
// clock that their power leaves (1.8 GHz): 8192 tokens of 32 heads of 128, bf16, 607 us, 906 TFLOP/s of the 1123 of a large
// matrix product; with a window of 2048, 16 384 tokens of 8 heads, 172 us, 751.  Single tokens are bound by memory: 48 over
// caches of up to 16 000 positions 364 us, 4.3 TB/s of a large copy's 4.6; one over 131 070 136 us, of which 14 join 256
// pieces.  fp32 (61 x 197 tokens of 16 heads of 72) 211 us, 51 TFLOP/s of the 154 of a large product: 72 elements and 197 keys are
// padded to 96 and 224, the last 69 rows of a sequence to 96.
//
// P is rounded to bf16 where it meets bf16 values, to the nearest: that, and the result's own rounding, are 2.2e-3 of a
// result's norm against 64 bits where the result's rounding alone is 1.6e-3.
#include "slowmo_attention.h"

namespace slowmo {
namespace attention {
namespace {

constexpr int kMostPieces = 256;  // of a row's keys: a thread each where they are joined

struct Args {
  Rows q, k, v, out;
  float *lse;
  const int64_t *q_offsets, *k_offsets;  // paged: k_offsets are the lengths
  const int32_t *pages;
  int64_t pages_stride, k_page, v_page;  // elements from one page to the next
  int32_t columns, n_pages, page_log2, held;  // held: positions that the table has pages for
  int32_t batch, heads, group, dim;
  u32 by_group;
  int64_t tokens, keys, first, slots;
  float scale;  // of scores to powers of two
  Mask mask;
  bool wide, clear;
  bool apart;  // the keys' rows are not the queries': another list of offsets, or the same one over another number of rows
  int32_t splits, least;  // pieces of the key axis at most; tiles of a piece at least
  float *part, *part_lse;
};

__device__ const u32x4 kNothing[1] = {{0, 0, 0, 0}};

// A tile's way from memory to shared memory.  j0: its first position; rows past `keys` take the last one's place
// and are masked.  Positions without a page are zeros: a row that sees one is marked by its sum.
template <typename T, int DP, bool PAGED>
struct Stage {
  using L = Tile<T, DP>;
  const Args &a;
  int keys, lane, wave, waves;
  // the page of position j0 + lane
  __device__ __forceinline__ int page_at(int b, int j0) const {
    const int column = min(j0 + (lane & (L::rows - 1)), keys - 1) >> a.page_log2;
    return column < a.columns ? a.pages[static_cast<int64_t>(b) * a.pages_stride + column] : -1;
  }
  // the rows of a tile, a bit each (twice, where they are 32), that have no page
  __device__ __forceinline__ uint64_t without(int page) const {
    return __ballot(static_cast<u32>(page) >= static_cast<u32>(a.n_pages));
  }
  __device__ __forceinline__ void load(char *tile, const Rows &x, int64_t page_stride, int64_t begin, int head, int j0,
                                       int page) const {
    const T *base = static_cast<const T *>(x.data) + head * x.head;
    if constexpr (!PAGED) {
      bring_rows<T, DP>(tile, L::rows, base + (begin + j0) * x.token, a.dim, a.wide,
                        [&](int r) { return min(r, keys - 1 - j0) * x.token; });
      return;
    }
    if (!a.wide) {
      for (int i = threadIdx.x; i < L::rows * L::used; i += blockDim.x) {
        const int row = i / L::used, c = i % L::used, j = min(j0 + row, keys - 1);
        const int id = __shfl(page, row);  // the turns are a multiple of 64, so that a wave's lanes are all here
        const bool there = static_cast<u32>(id) < static_cast<u32>(a.n_pages);
        const T *from = base + (there ? id : 0) * page_stride + (j & ((1 << a.page_log2) - 1)) * x.token;
        T *to = reinterpret_cast<T *>(tile + row * L::row_bytes + ((c ^ L::turn(row)) << 4));
#pragma unroll
        for (int e = 0; e < L::E; ++e)
          to[e] = c * L::E + e >= a.dim ? static_cast<T>(0.f)
                  : there               ? from[c * L::E + e]
                                        : static_cast<T>(0.f);
      }
      return;
    }
    const u32 shared = uniform(offset_of(tile));
    constexpr int R = L::C < 64 ? 64 / L::C : 1;  // rows of a piece
    // Whole tiles whose pieces each lie in one page: every lane works out one row's address, and a piece takes that of
    // its first row (48 single tokens over 16 000: 667 -> 452 us with an address for each lane and piece; this way 365, 4.3 TB/s).
    if ((1 << a.page_log2) >= R && j0 + L::rows <= keys &&
        __all(static_cast<u32>(page) < static_cast<u32>(a.n_pages))) {
      const u32 step = static_cast<u32>(x.token) * sizeof(T);
      const int j = j0 + (lane & (L::rows - 1));
      const u32x2 mine = __builtin_bit_cast(
          u32x2, base + static_cast<int64_t>(page) * page_stride + (j & ((1 << a.page_log2) - 1)) * x.token);
      auto piece = [&](int n) SLOWMO_INLINE {
        const int row0 = n * R, c = (lane & (L::C - 1)) ^ L::turn(row0 + lane / L::C);
        const u32x2 from = {static_cast<u32>(__builtin_amdgcn_readlane(mine[0], row0)),
                            static_cast<u32>(__builtin_amdgcn_readlane(mine[1], row0))};
        if (c * L::E < a.dim)
          to_shared(uniform(shared + n * 1024), (lane / L::C) * step + c * 16, __builtin_bit_cast(const T *, from));
      };
      if (waves == 1) {
#pragma unroll
        for (int n = 0; n < L::bytes / 1024; ++n) piece(n);
      } else {
        for (int n = wave; n < L::bytes / 1024; n += waves) piece(n);
      }
      return;
    }
    for (int n = wave; n < L::bytes / 1024; n += waves) {
      const int at = n * 64 + lane, row = at / L::C, c = (at & (L::C - 1)) ^ L::turn(row);
      const int r = min(row, keys - 1 - j0);
      const u32 to = uniform(shared + n * 1024);
      const int id = __shfl(page, row);
      const char *p = reinterpret_cast<const char *>(base + static_cast<int64_t>(id) * page_stride +
                                                     ((j0 + r) & ((1 << a.page_log2) - 1)) * x.token + c * L::E);
      if (static_cast<u32>(id) >= static_cast<u32>(a.n_pages))
        p = reinterpret_cast<const char *>(kNothing);
      if (c * L::E < a.dim) to_shared(to, p);
    }
  }
};

// 256 registers a lane let two waves share a SIMD; wider heads take up to 512.

template <typename T, int DP, bool PAGED>
__global__ __launch_bounds__(256, (DP <= 128 ? 2 : 1)) void k_attention(Args a) {
  using L = Tile<T, DP>;
  using frag = typename Kind<T>::frag;
  constexpr int NB = DP / 32, KB = L::rows / 32;
  extern __shared__ __align__(1024) char smem[];
  const int lane = threadIdx.x & 63, low = lane & 31, high = lane >> 5;
  const int wave = uniform(static_cast<int>(threadIdx.x >> 6)), waves = blockDim.x >> 6, height = waves * 32;

  int head;
  int64_t slot;
  if (!head_slot(a.first + blockIdx.x, a.heads, a.slots * a.splits, head, slot)) return;
  const int split = static_cast<int>(slot % a.splits);
  slot = a.slots - 1 - slot / a.splits;  // the last tiles, which see the most keys, first
  const Place at = place_of(a.q_offsets, a.batch, a.tokens, a.group, height, slot);
  const int64_t rows = static_cast<int64_t>(at.n) * a.group;
  const int64_t row0 = static_cast<int64_t>(at.tile) * height;
  if (at.b < 0 || row0 >= rows) return;
  // this lane's row
  const int row = wave * 32 + low, last_row = static_cast<int>(min(rows - row0, static_cast<int64_t>(height))) - 1;
  const bool mine = row <= last_row, idle = wave * 32 > last_row;
  const Split split_row(row0, a.group, a.by_group);
  const int token = split_row.token(min(row, last_row)), of = split_row.head(min(row, last_row), token);
  const int64_t qt = at.begin + token;
  const int qh = head * a.group + of;
  T *out = static_cast<T *>(a.out.data) + qt * a.out.token + qh * a.out.head;
  float *lse = a.lse ? a.lse + qt * (static_cast<int64_t>(a.heads) * a.group) + qh : nullptr;
  f32x16 acc[NB];
  if (at.b == a.batch) {  // behind the last sequence
    if (!a.clear || split) return;
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[b] = f32x16{};
    store_columns<T, NB>(out, acc, 0.f, a.dim, high, a.wide, mine);
    if (lse && mine && !high) *lse = -INFINITY;
    return;
  }
  int64_t k_begin = at.begin;
  int keys = at.n;
  if constexpr (PAGED) {
    keys = static_cast<int>(clamped(uniform(a.k_offsets[at.b]), 0, kLongest));
  } else if (a.apart) {
    k_begin = clamped(uniform(a.k_offsets[at.b]), 0, a.keys);
    keys = static_cast<int>(clamped(uniform(a.k_offsets[at.b + 1]), k_begin, a.keys) - k_begin);
  }
  const int far = keys - at.n;
  const int p_lo = split_row.t0 + far, p_hi = split_row.token(last_row) + far;
  const Walk walk = walk_of(a.mask, p_lo, p_hi, keys, L::rows, a.held);
  int per;
  const int pieces = pieces_of(walk.count, a.splits, a.least, per);
  if (split >= pieces) return;
  const int u0 = split * per, u1 = min(walk.count, u0 + per);
  const Sight sight = sight_of(a.mask, token + far, keys);
  // what the whole wave sees of every row: between the bounds of its first and last row
  const Sight first = sight_of(a.mask, split_row.token(min(wave * 32, last_row)) + far, keys),
              last = sight_of(a.mask, split_row.token(min(wave * 32 + 31, last_row)) + far, keys);
  if (a.dim != DP) {  // the rows' ends that no load writes
    for (int i = threadIdx.x; i < 4 * L::bytes / 16; i += blockDim.x) reinterpret_cast<u32x4 *>(smem)[i] = u32x4{0, 0, 0, 0};
    __syncthreads();
  }
  const Stage<T, DP, PAGED> stage{a, keys, lane, wave, waves};
  int page = 0;
  bool gone = false;  // some position of a tile has no page
  auto bring = [&](int u) SLOWMO_INLINE {
    char *to = smem + (u & 1) * 2 * L::bytes;
    const int j0 = walk.at(u) * L::rows;
    if constexpr (PAGED) {
      settle(page);
      gone = gone || stage.without(page);
    }
    stage.load(to, a.k, a.k_page, k_begin, head, j0, page);
    stage.load(to + L::bytes, a.v, a.v_page, k_begin, head, j0, page);
    if constexpr (PAGED)
      if (u + 1 < u1) page = stage.page_at(at.b, walk.at(u + 1) * L::rows);
  };
  auto start = [&]() SLOWMO_INLINE {
    if (u0 >= u1) return;
    if constexpr (PAGED) page = stage.page_at(at.b, walk.at(u0) * L::rows);
    bring(u0);
  };
  start();  // beside the queries
  frag qf[DP / 16];
  {
    const T *q = static_cast<const T *>(a.q.data) + qt * a.q.token + qh * a.q.head;
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) qf[s] = load_frag<T>(q, 16 * s + 8 * high, a.dim, a.wide);
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) settle(qf[s]);
  }
  float m, l;
  for (bool careful = false;; careful = true) {
    if (careful) start();
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[b] = f32x16{};
    m = -INFINITY, l = 0.f;
    for (int u = u0; u < u1; ++u) {
      arrive();
      if (u + 1 < u1) bring(u + 1);
      char *k_tile = smem + (u & 1) * 2 * L::bytes, *v_tile = k_tile + L::bytes;
      const int j0 = walk.at(u) * L::rows, j1 = j0 + L::rows - 1;
      if (careful && any_wild<T, DP, L::rows>(v_tile)) tame<T, DP, L::rows>(v_tile, v_tile);
      // the wave has no row, or none that sees a key of the tile
      if (idle || ((j0 > last.hi || j1 < first.lo) && j0 >= last.sinks)) continue;
      // Wide heads: addresses are worked out anew for each tile; kept, they would be spilled to scratch, and reading them
      // back would wait for the tiles under way.
      int row_lane = low, column_lane = lane;
      if constexpr (DP * sizeof(T) >= 384) settle(row_lane), settle(column_lane);
      f32x16 s[KB];
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) s[kb] = f32x16{};
      // Products of fp32 are 16 times as long: those of keys past the last one, and of elements past the head's end, are
      // left out.
      constexpr bool kLong = sizeof(T) == 4;
#pragma unroll
      for (int st = 0; st < DP / 16; ++st) {
        if (kLong && 16 * st >= a.dim) continue;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          if (kLong && j0 + 32 * kb >= keys) continue;
          s[kb] = mma(row_frag<T, DP>(k_tile, 32 * kb + row_lane, st, high), qf[st], s[kb]);
        }
      }
      read_ahead<T, KB * DP / 16, 1, 1, 6>();
      if (!((j0 >= last.lo && j1 <= first.hi) || j1 < first.sinks)) {
        branch();
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!sees(sight, j0 + 32 * kb + 8 * (i / 4) + 4 * high + i % 4)) s[kb][i] = -INFINITY;
      }
      float top = s[0][0];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kb][i]);
      top = both_max(top) * a.scale;
      // The sums are held against a maximum that may be up to 2^8 too low, so that most tiles change no sums.
      if (__any(top > m + 8.f)) {
        const float now = fmaxf(m, top);
        const float by = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - now);
        l *= by;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[b][i] *= by;
        m = now;
      }
      const float under = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[kb][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][i], a.scale, -under));
          l += s[kb][i];
        }
#pragma unroll
      for (int st = 0; st < L::rows / 16; ++st) {
        if (kLong && j0 + 16 * st >= keys) continue;
        const frag p = as_frag<T>(s[st / 2], st % 2);
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[b] = mma(column_frag<T, DP>(v_tile, b, st, column_lane), p, acc[b]);
      }
      read_ahead<T, NB * L::rows / 16, 1, 2, 3>();
    }
    if (careful) {
      // what is wild comes to the sums that are no longer brought down, by 0 at times, to a higher maximum
      __syncthreads();
      start();
      for (int u = u0; u < u1; ++u) {
        arrive();
        if (u + 1 < u1) bring(u + 1);
        char *v_tile = smem + (u & 1) * 2 * L::bytes + L::bytes;
        const int j0 = walk.at(u) * L::rows;
        if (any_wild<T, DP, L::rows>(v_tile)) add_wild<T, DP, L::rows>(v_tile, acc, 1.f, [&](int r) { return sees(sight, j0 + r); });
      }
      break;
    }
    int any = 0;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) any |= wild(acc[b][i]);
    // also ends this pass's reads of shared memory
    if (!__syncthreads_or(any)) break;
  }
  if constexpr (PAGED)
    // NaN in a row's sum is NaN in its result and lse, and survives pieces whose weight underflows
    for (int u = u0; gone && u < u1; ++u) {
      const int j0 = walk.at(u) * L::rows;
      for (uint64_t left = stage.without(stage.page_at(at.b, j0)); left; left &= left - 1)
        if (sees(sight, j0 + __builtin_ctzll(left) % L::rows)) l = __builtin_nanf("");
    }
  l = both_sum(l);
  const float by = l == 0.f ? 0.f : 1.f / l;
  const float log2_sum = l == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(l);
  if (pieces == 1) {
    store_columns<T, NB>(out, acc, by, a.dim, high, a.wide, mine);
    if (lse && mine && !high) *lse = log2_sum * kLn2;
  } else {
    const int64_t every = a.tokens * a.heads * a.group, at_row = qt * (static_cast<int64_t>(a.heads) * a.group) + qh;
    store_columns<float, NB>(a.part + (split * every + at_row) * DP, acc, by, DP, high, true, mine);
    if (mine && !high) a.part_lse[split * every + at_row] = log2_sum;
  }
}

// The pieces of a row joined in their order.  What is wild in one, a key's value that the row sees, stays so if its weight
// underflows.  WAVES = 1: a wave a row, for up to 32 pieces; 4: a workgroup a row, every fourth piece to a wave.  4 elements
// to a lane.
template <typename T, int DP, int WAVES>
__global__ __launch_bounds__(256) void k_join(Args a, int height, int tile) {
  __shared__ float weights[4][64], of_wave[4];
  __shared__ f32x4 sums[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t every = a.tokens * a.heads * a.group;
  const int64_t at_row = (blockIdx.x + a.first) * (4 / WAVES) + (WAVES == 1 ? uniform(wave) : 0);
  if (at_row >= every) return;
  const int64_t qt = at_row / (a.heads * a.group);
  const int qh = static_cast<int>(at_row - qt * (a.heads * a.group));
  // the token's sequence: the last one that starts at or before it
  int count = stretch_of(a.batch, [&](int b) { return clamped(uniform(a.q_offsets[b]), 0, a.tokens) <= qt; });
  for (int first = count; first <= a.batch; first += 64) {
    const int b = first + lane;
    const int got = __popcll(__ballot(b <= a.batch && clamped(a.q_offsets[min(b, a.batch)], 0, a.tokens) <= qt));
    count += got;
    if (got < 64) break;
  }
  const int b = uniform(count - 1);
  if (b < 0 || b >= a.batch) return;
  const int64_t begin = clamped(uniform(a.q_offsets[b]), 0, a.tokens), end = clamped(uniform(a.q_offsets[b + 1]), begin, a.tokens);
  const int n = static_cast<int>(end - begin), keys = static_cast<int>(clamped(uniform(a.k_offsets[b]), 0, kLongest));
  const int64_t rows = static_cast<int64_t>(n) * a.group, row = (qt - begin) * a.group + qh % a.group;
  const int64_t row0 = row / height * height, row_last = min(row0 + height, rows) - 1;
  if (row >= rows) return;
  const Walk walk = walk_of(a.mask, static_cast<int>(row0 / a.group) + keys - n, static_cast<int>(row_last / a.group) + keys - n,
                            keys, tile, a.held);
  int per;
  const int pieces = pieces_of(walk.count, a.splits, a.least, per);
  if (pieces == 1) return;
  // one piece a lane: the largest, then the weights
  const int z = WAVES == 1 ? lane : threadIdx.x;
  const float mine = z < pieces ? a.part_lse[z * every + at_row] : -INFINITY;
  float m = mine;
#pragma unroll
  for (int by = 1; by < 64; by *= 2) m = fmaxf(m, __shfl_xor(m, by));
  bool none = __any(mine != mine);
  if constexpr (WAVES > 1) {
    none = __syncthreads_or(none);
    if (lane == 0) of_wave[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(of_wave[0], of_wave[1]), fmaxf(of_wave[2], of_wave[3]));
  }
  const float weight = __builtin_amdgcn_exp2f(mine - (m == -INFINITY ? 0.f : m));
  if constexpr (WAVES > 1) {
    weights[wave][lane] = weight;
    __syncthreads();
  }
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int y0 = WAVES == 1 ? 0 : wave; y0 < pieces; y0 += 8 * WAVES) {  // eight are asked for at once
    f32x4 v[8];
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int y = min(y0 + WAVES * e, pieces - 1);
      w[e] = WAVES == 1 ? __shfl(weight, y) : weights[y / 64][y % 64];
      if (y0 + WAVES * e >= pieces) w[e] = 0.f;
      v[e] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (4 * lane < DP && y0 + WAVES * e < pieces) v[e] = *reinterpret_cast<const f32x4 *>(a.part + (y * every + at_row) * DP + 4 * lane);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] += wild(v[e][i]) ? v[e][i] : w[e] * v[e][i];
  }
  float total = weight;
  if constexpr (WAVES > 1) {
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave) return;
    total = weights[0][lane] + weights[1][lane] + weights[2][lane] + weights[3][lane];
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] = sums[0][lane][i] + sums[1][lane][i] + sums[2][lane][i] + sums[3][lane][i];
  }
#pragma unroll
  for (int by = 1; by < 64; by *= 2) total += __shfl_xor(total, by);
  const float by = total == 0.f ? 0.f : 1.f / total;
  T *out = static_cast<T *>(a.out.data) + qt * a.out.token + qh * a.out.head;
  for (int i = 0; i < 4; ++i)
    if (4 * lane + i < a.dim)
      out[4 * lane + i] = static_cast<T>(
          none ? __builtin_nanf("") : sum[i] * by);
  if (a.lse && lane == 0) a.lse[at_row] = none ? __builtin_nanf("") : total == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(total)) * kLn2;
}

struct Pieces {
  int splits, least, waves;
};
// Pieces of the key axis, of like length for long and short sequences: some thousand where rows are few, one of 4 waves
// for at least 16 tiles, since its sums are 64 KB.  How long the sequences are is not known here: the table's width is taken.
Pieces pieces_for(const slowmo_attention_config &c, int64_t tokens, int64_t group, int64_t heads, int64_t batch, int64_t positions,
                  int rows_of_tile) {
  Pieces p;
  p.waves = waves_of(tokens, group, batch, 4);
  const int64_t height = p.waves * 32;
  int64_t seen = std::min<int64_t>(positions, kLongest);
  if (c.window) seen = std::min(seen, std::min<int64_t>(c.window, kLongest) + height / group + std::min<int64_t>(c.sinks, kLongest) + 2 * rows_of_tile);
  const int64_t tiles = (seen + rows_of_tile - 1) / rows_of_tile;
  const int64_t groups = std::max<int64_t>(1, std::min(batch, tokens) + tokens * group / height) * heads;
  p.least = static_cast<int>(std::clamp<int64_t>(groups * tiles / (p.waves == 1 ? 8192 : 2048), p.waves == 1 ? 8 : 16, kLongest));
  // no more than a gigabyte of sums
  const int64_t row_bytes = tokens * heads * group * (SLOWMO_MAX_ATTENTION_DIM + 1) * 4;
  const int64_t most = std::clamp<int64_t>((int64_t(1) << 30) / std::max<int64_t>(row_bytes, 1), 1, kMostPieces);
  p.splits = static_cast<int>(std::clamp<int64_t>((tiles + p.least - 1) / p.least, 1, most));
  return p;
}

template <bool PAGED>
hipError_t launch(Args a, int32_t dtype, int waves, hipStream_t stream) {
  hipError_t e = hipSuccess;
  dispatch(dtype, a.dim, [&](auto kind, auto dp) {
    using T = decltype(kind);
    using L = Tile<T, dp()>;
    constexpr int DP = dp();
    const int bytes = 4 * L::bytes;
    const auto kernel = k_attention<T, DP, PAGED>;
    if (bytes > 64 * 1024)
      e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    a.slots = slots_of(a.tokens, a.group, waves * 32, a.batch);
    const int64_t items = items_of(a.heads, a.slots * a.splits);
    for (a.first = 0; a.first < items && e == hipSuccess; a.first += kMostBlocks) {
      kernel<<<static_cast<u32>(std::min(kMostBlocks, items - a.first)), 64 * waves, bytes, stream>>>(a);
      e = hipGetLastError();
    }
    if (a.splits > 1) {
      const int64_t every = a.tokens * a.heads * a.group;
      const int64_t blocks = a.splits <= 32 ? (every + 3) / 4 : every;
      for (a.first = 0; a.first < blocks && e == hipSuccess; a.first += kMostBlocks) {
        const u32 n = static_cast<u32>(std::min(kMostBlocks, blocks - a.first));
        if (a.splits <= 32) k_join<T, DP, 1><<<n, 256, 0, stream>>>(a, waves * 32, L::rows);
        else k_join<T, DP, 4><<<n, 256, 0, stream>>>(a, waves * 32, L::rows);
        e = hipGetLastError();
      }
    }
  });
  return e;
}

void fill(Args &a, const slowmo_attention_config &c, int64_t tokens, const slowmo_heads &q, const slowmo_heads &out, int heads) {
  a.q = rows_of(q), a.out = rows_of(out);
  a.heads = heads, a.group = q.heads / heads, a.by_group = by_group(a.group), a.dim = c.head_dim, a.tokens = tokens;
  a.scale = c.scale * kLog2E;
  a.mask = mask_of(c);
  a.clear = c.clear_rest != 0;
  a.splits = 1, a.least = 1, a.held = kLongest;
}

}  // namespace

// ---- checks ----

const char *check_config(const slowmo_attention_config *c) {
  if (!c) return "cfg is NULL";
  if (c->dtype != SLOWMO_F32 && c->dtype != SLOWMO_BF16) return "unknown dtype";
  if (c->head_dim < 1 || c->head_dim > SLOWMO_MAX_ATTENTION_DIM) return "head_dim must be in 1..SLOWMO_MAX_ATTENTION_DIM";
  if (c->causal != 0 && c->causal != 1) return "causal must be 0 or 1";
  if (c->clear_rest != 0 && c->clear_rest != 1) return "clear_rest must be 0 or 1";
  if (!(std::isfinite(c->scale) && c->scale > 0.f && std::isfinite(c->scale * kLog2E))) return "scale must be finite and > 0";
  if (c->window < 0 || c->sinks < 0) return "window and sinks must be >= 0";
  return nullptr;
}

slowmo_status check_call(const slowmo_attention_config *cfg, int32_t batch, const int64_t *q_offsets, const int64_t *k_offsets,
                         int64_t tokens, int64_t keys) {
  auto bad = [](const char *msg) { return fail_thread(SLOWMO_ERR_ARG, msg); };
  if (const char *msg = check_config(cfg)) return bad(msg);
  if (batch < 0 || batch > (1 << 20)) return bad("batch must be in 0..2^20");
  if (tokens < 0 || tokens > kLongest || keys < 0 || keys > kLongest) return bad("tokens and keys must be in 0..2^30");
  if (!q_offsets) return bad("q_offsets is NULL");
  if (!aligned(q_offsets, 8) || !aligned(k_offsets, 8)) return fail_thread(SLOWMO_ERR_ALIGN, "offsets must be 8-byte aligned");
  if (!k_offsets && keys != tokens) return bad("without k_offsets there are as many keys as tokens");
  return SLOWMO_OK;
}
slowmo_status check_group(int64_t tokens, int32_t q_heads, int32_t k_heads) {
  if (tokens * q_heads > int64_t(1) << 36) return fail_thread(SLOWMO_ERR_ARG, "at most 2^36 rows of queries");
  if (q_heads % k_heads) return fail_thread(SLOWMO_ERR_ARG, "query heads must be a multiple of key heads");
  if (q_heads / k_heads > kMostShared) return fail_thread(SLOWMO_ERR_ARG, "at most 2^12 query heads share a key head");
  return SLOWMO_OK;
}
Mask mask_of(const slowmo_attention_config &c) {
  return {c.causal, static_cast<int32_t>(std::min<int64_t>(c.window, kLongest)),
          c.window ? static_cast<int32_t>(std::min<int64_t>(c.sinks, kLongest)) : 0};
}

slowmo_status check_rows(const slowmo_heads *h, int64_t rows, int32_t dim, int32_t dtype, bool written) {
  auto bad = [](const char *msg) { return fail_thread(SLOWMO_ERR_ARG, msg); };
  if (!h) return bad("a slowmo_heads is NULL");
  if (h->heads < 1 || h->heads > (1 << 20)) return bad("heads must be in 1..2^20");
  if (h->token_stride < 0 || h->head_stride < 0 || h->token_stride > (int64_t(1) << 40) || h->head_stride > (int64_t(1) << 40))
    return bad("strides must be in 0..2^40");
  if (static_cast<double>(h->token_stride) * static_cast<double>(std::max<int64_t>(rows - 1, 0)) +
          static_cast<double>(h->head_stride) * (h->heads - 1) > std::exp2(50.))
    return bad("an array reaches past 2^50 elements");
  if (rows && !h->data) return bad("data is NULL");
  if (!aligned(h->data, size_of(dtype))) return fail_thread(SLOWMO_ERR_ALIGN, "data is not aligned to its element size");
  if (written && rows) {
    const int64_t across = h->head_stride * (h->heads - 1) + dim, down = h->token_stride * (rows - 1) + dim;
    if ((h->heads > 1 && h->head_stride < dim) || (rows > 1 && h->token_stride < dim) ||
        (rows > 1 && h->heads > 1 && h->token_stride < across && h->head_stride < down))
      return bad("rows of an output overlap each other");
  }
  return SLOWMO_OK;
}

slowmo_status check_cache(const slowmo_cache *c, int32_t dim, int32_t dtype, bool written) {
  auto bad = [](const char *msg) { return fail_thread(SLOWMO_ERR_ARG, msg); };
  if (!c) return bad("a slowmo_cache is NULL");
  if (c->heads < 1 || c->heads > (1 << 20)) return bad("a cache's heads must be in 1..2^20");
  if (c->page < 1 || c->page > SLOWMO_MAX_PAGE || (c->page & (c->page - 1))) return bad("page must be a power of two in 1..SLOWMO_MAX_PAGE");
  if (c->pages < 0 || c->pages > INT32_MAX) return bad("pages must be in 0..2^31-1");
  const int64_t most = int64_t(1) << 40;
  if (c->page_stride < 0 || c->token_stride < 0 || c->head_stride < 0 || c->page_stride > most || c->token_stride > most ||
      c->head_stride > most)
    return bad("a cache's strides must be in 0..2^40");
  if (static_cast<double>(c->page_stride) * static_cast<double>(std::max<int64_t>(c->pages - 1, 0)) +
          static_cast<double>(c->token_stride) * (c->page - 1) + static_cast<double>(c->head_stride) * (c->heads - 1) >
      std::exp2(50.))
    return bad("a cache reaches past 2^50 elements");
  if (c->pages && !c->data) return bad("a cache's data is NULL");
  if (!aligned(c->data, size_of(dtype))) return fail_thread(SLOWMO_ERR_ALIGN, "a cache is not aligned to its element size");
  if (written && c->pages) {
    // in the order of their strides every axis steps past what the ones below it cover
    int64_t stride[3] = {c->head_stride, c->token_stride, c->page_stride}, count[3] = {c->heads, c->page, c->pages};
    for (int i = 0; i < 3; ++i)
      for (int j = i + 1; j < 3; ++j)
        if (stride[j] < stride[i]) std::swap(stride[i], stride[j]), std::swap(count[i], count[j]);
    int64_t covered = dim;
    for (int i = 0; i < 3; ++i) {
      if (count[i] < 2) continue;
      if (stride[i] < covered) return bad("rows of a cache overlap each other");
      covered += stride[i] * (count[i] - 1);
    }
  }
  return SLOWMO_OK;
}

slowmo_status check_pages(const slowmo_pages *p, int64_t tokens) {
  auto bad = [](const char *msg) { return fail_thread(SLOWMO_ERR_ARG, msg); };
  if (!p) return bad("pages is NULL");
  if (p->batch < 0 || p->batch > (1 << 20)) return bad("batch must be in 0..2^20");
  if (p->columns < 0 || p->columns > kLongest) return bad("columns must be in 0..2^30");
  if (p->stride < p->columns || p->stride > (int64_t(1) << 40)) return bad("a table's stride must be in columns..2^40");
  if (tokens < 0 || tokens > kLongest) return bad("tokens must be in 0..2^30");
  if (!p->offsets || (p->batch && (!p->lengths || (p->columns && !p->pages)))) return bad("pages, lengths or offsets is NULL");
  if (!aligned(p->pages, 4) || !aligned(p->lengths, 8) || !aligned(p->offsets, 8))
    return fail_thread(SLOWMO_ERR_ALIGN, "pages must be 4-byte aligned, lengths and offsets 8-byte aligned");
  return SLOWMO_OK;
}

Extent extent(const slowmo_heads &h, int64_t rows, int32_t dim, int32_t dtype) {
  Extent e;
  if (!rows) return e;
  const int64_t size = size_of(dtype);
  e.lo = reinterpret_cast<uintptr_t>(h.data);
  e.hi = e.lo + (h.token_stride * (rows - 1) + h.head_stride * (h.heads - 1) + dim) * size;
  e.period[0] = h.token_stride * size, e.width[0] = (h.head_stride * (h.heads - 1) + dim) * size;
  return e;
}
Extent extent(const slowmo_cache &c, int32_t dim, int32_t dtype) {
  Extent e;
  if (!c.pages) return e;
  const int64_t size = size_of(dtype), inside = c.token_stride * (c.page - 1) + c.head_stride * (c.heads - 1) + dim;
  e.lo = reinterpret_cast<uintptr_t>(c.data);
  e.hi = e.lo + (c.page_stride * (c.pages - 1) + inside) * size;
  // keys and values may lie beside each other in every page, or in every row
  e.period[0] = c.page_stride * size, e.width[0] = inside * size;
  if (c.token_stride && c.page_stride % c.token_stride == 0)
    e.period[1] = c.token_stride * size, e.width[1] = (c.head_stride * (c.heads - 1) + dim) * size;
  return e;
}
Extent extent(const void *p, size_t bytes) {
  Extent e;
  if (!bytes || !p) return e;
  e.lo = reinterpret_cast<uintptr_t>(p), e.hi = e.lo + bytes;
  return e;
}
bool overlap(const Extent &x, const Extent &y) {
  if (x.lo == x.hi || y.lo == y.hi || x.hi <= y.lo || y.hi <= x.lo) return false;
  for (int i = 0; i < 2; ++i) {
    const int64_t period = x.period[i];
    if (period <= 0 || period != y.period[i] || x.width[i] > period || y.width[i] > period) continue;
    int64_t d = (static_cast<int64_t>(y.lo) - static_cast<int64_t>(x.lo)) % period;
    if (d < 0) d += period;
    if (x.width[i] <= d && d + y.width[i] <= period) return false;  // side by side within every period
  }
  return true;
}

bool wide_rows(const slowmo_heads &h, int32_t dim, int32_t dtype) {
  const int64_t size = size_of(dtype);
  return dim * size % 16 == 0 && aligned(h.data, 16) && h.token_stride * size % 16 == 0 && h.head_stride * size % 16 == 0 &&
         h.token_stride * size < (1 << 25) && h.head_stride * size * h.heads < (1 << 30);
}
bool wide_rows(const slowmo_cache &c, int32_t dim, int32_t dtype) {
  const int64_t size = size_of(dtype);
  return dim * size % 16 == 0 && aligned(c.data, 16) && c.page_stride * size % 16 == 0 && c.token_stride * size % 16 == 0 &&
         c.head_stride * size % 16 == 0 && c.token_stride * size < (1 << 25);
}

}  // namespace attention
}  // namespace slowmo

using namespace slowmo;
using namespace slowmo::attention;

extern "C" {

slowmo_status slowmo_attention(const slowmo_attention_config *cfg, int32_t batch, const int64_t *q_offsets,
                               const int64_t *k_offsets, int64_t tokens, int64_t keys, const slowmo_heads *q,
                               const slowmo_heads *k, const slowmo_heads *v, const slowmo_heads *out, float *lse,
                               void *stream) {
  return walled([&]() -> slowmo_status {
    auto bad = [](const char *msg) { return fail_thread(SLOWMO_ERR_ARG, msg); };
    if (const slowmo_status s = check_call(cfg, batch, q_offsets, k_offsets, tokens, keys)) return s;
    const slowmo_heads *every[] = {q, k, v, out};
    for (int i = 0; i < 4; ++i)
      if (const slowmo_status s = check_rows(every[i], i == 1 || i == 2 ? keys : tokens, cfg->head_dim, cfg->dtype, i == 3)) return s;
    if (k->heads != v->heads || q->heads != out->heads) return bad("v has k's heads, out has q's");
    if (const slowmo_status s = check_group(tokens, q->heads, k->heads)) return s;
    if (!aligned(lse, 4)) return fail_thread(SLOWMO_ERR_ALIGN, "lse must be 4-byte aligned");
    const Extent eo = extent(*out, tokens, cfg->head_dim, cfg->dtype), el = extent(lse, tokens * q->heads * sizeof(float));
    for (int i = 0; i < 3; ++i) {
      const Extent ei = extent(*every[i], i ? keys : tokens, cfg->head_dim, cfg->dtype);
      if (overlap(eo, ei) || overlap(el, ei)) return bad("an output overlaps an input");
    }
    if (overlap(eo, el)) return bad("out and lse overlap");
    if (!tokens) return SLOWMO_OK;
    Args a{};
    fill(a, *cfg, tokens, *q, *out, k->heads);
    a.k = rows_of(*k), a.v = rows_of(*v), a.lse = lse, a.keys = keys, a.batch = batch;
    a.q_offsets = q_offsets, a.k_offsets = k_offsets ? k_offsets : q_offsets;
    a.apart = a.k_offsets != q_offsets || keys != tokens;
    a.wide = true;
    for (const slowmo_heads *h : every) a.wide = a.wide && wide_rows(*h, cfg->head_dim, cfg->dtype);
    const hipError_t e = launch<false>(a, cfg->dtype, waves_of(tokens, a.group, batch, 4), static_cast<hipStream_t>(stream));
    return e == hipSuccess ? SLOWMO_OK : fail_thread_hip(e, "slowmo_attention");
  });
}

size_t slowmo_paged_attention_bytes(const slowmo_attention_config *cfg, const slowmo_pages *pages, int64_t tokens, int32_t q_heads,
                                    const slowmo_cache *k_cache) {
  if (check_config(cfg) || !pages || !k_cache || tokens <= 0 || tokens > kLongest || q_heads <= 0 || q_heads > (1 << 20) ||
      k_cache->heads <= 0 || q_heads % k_cache->heads || pages->batch <= 0 || pages->columns < 0 || k_cache->page <= 0)
    return 0;
  const int dp = padded(cfg->head_dim);
  const int rows = rows_of_tile(cfg->head_dim, cfg->dtype);
  const Pieces p = pieces_for(*cfg, tokens, q_heads / k_cache->heads, k_cache->heads, pages->batch,
                              static_cast<int64_t>(pages->columns) * k_cache->page, rows);
  return p.splits == 1 ? 0 : static_cast<size_t>(p.splits) * tokens * q_heads * (dp + 1) * sizeof(float);
}

slowmo_status slowmo_paged_attention(const slowmo_attention_config *cfg, const slowmo_pages *pages, int64_t tokens,
                                     const slowmo_heads *q, const slowmo_cache *k_cache, const slowmo_cache *v_cache,
                                     const slowmo_heads *out, float *lse, void *workspace, size_t workspace_bytes,
                                     void *stream) {
  return walled([&]() -> slowmo_status {
    auto bad = [](const char *msg) { return fail_thread(SLOWMO_ERR_ARG, msg); };
    if (const char *msg = check_config(cfg)) return bad(msg);
    if (const slowmo_status s = check_pages(pages, tokens)) return s;
    const slowmo_heads *every[] = {q, out};
    for (int i = 0; i < 2; ++i)
      if (const slowmo_status s = check_rows(every[i], tokens, cfg->head_dim, cfg->dtype, i == 1)) return s;
    const slowmo_cache *caches[] = {k_cache, v_cache};
    for (const slowmo_cache *c : caches)
      if (const slowmo_status s = check_cache(c, cfg->head_dim, cfg->dtype, false)) return s;
    if (k_cache->heads != v_cache->heads || k_cache->page != v_cache->page || k_cache->pages != v_cache->pages)
      return bad("the caches have the same heads, page and pages");
    if (q->heads != out->heads) return bad("out has q's heads");
    if (const slowmo_status s = check_group(tokens, q->heads, k_cache->heads)) return s;
    if (!aligned(lse, 4)) return fail_thread(SLOWMO_ERR_ALIGN, "lse must be 4-byte aligned");
    const Extent eo = extent(*out, tokens, cfg->head_dim, cfg->dtype), el = extent(lse, tokens * q->heads * sizeof(float));
    const size_t need = slowmo_paged_attention_bytes(cfg, pages, tokens, q->heads, k_cache);
    if (need && !workspace) return bad("workspace is NULL");
    if (need && !aligned(workspace, 16)) return fail_thread(SLOWMO_ERR_ALIGN, "workspace must be 16-byte aligned");
    if (workspace_bytes < need) return fail_thread(SLOWMO_ERR_NOMEM, "workspace is smaller than slowmo_paged_attention_bytes()");
    const Extent ew = extent(workspace, need);
    const Extent in[] = {extent(*q, tokens, cfg->head_dim, cfg->dtype), extent(*k_cache, cfg->head_dim, cfg->dtype),
                         extent(*v_cache, cfg->head_dim, cfg->dtype)};
    for (const Extent &i : in)
      if (overlap(eo, i) || overlap(el, i) || overlap(ew, i)) return bad("an output or the workspace overlaps an input");
    if (overlap(eo, el) || overlap(eo, ew) || overlap(el, ew)) return bad("out, lse and the workspace overlap");
    if (!tokens) return SLOWMO_OK;
    Args a{};
    fill(a, *cfg, tokens, *q, *out, k_cache->heads);
    a.k = {k_cache->data, k_cache->token_stride, k_cache->head_stride}, a.k_page = k_cache->page_stride;
    a.v = {v_cache->data, v_cache->token_stride, v_cache->head_stride}, a.v_page = v_cache->page_stride;
    a.lse = lse, a.batch = pages->batch;
    a.q_offsets = pages->offsets, a.k_offsets = pages->lengths;
    a.pages = pages->pages, a.pages_stride = pages->stride, a.columns = pages->columns;
    a.n_pages = static_cast<int32_t>(k_cache->pages);
    while ((1 << a.page_log2) < k_cache->page) ++a.page_log2;
    a.held = static_cast<int32_t>(std::min<int64_t>(static_cast<int64_t>(a.columns) << a.page_log2, kLongest));
    a.wide = wide_rows(*q, cfg->head_dim, cfg->dtype) && wide_rows(*out, cfg->head_dim, cfg->dtype) &&
             wide_rows(*k_cache, cfg->head_dim, cfg->dtype) && wide_rows(*v_cache, cfg->head_dim, cfg->dtype);
    const int dp = padded(cfg->head_dim), rows = rows_of_tile(cfg->head_dim, cfg->dtype);
    const Pieces p = pieces_for(*cfg, tokens, a.group, a.heads, pages->batch, static_cast<int64_t>(pages->columns) * k_cache->page, rows);
    a.splits = p.splits, a.least = p.least;
    a.part = static_cast<float *>(workspace);
    a.part_lse = a.part + static_cast<int64_t>(p.splits) * tokens * q->heads * dp;
    const hipError_t e = launch<true>(a, cfg->dtype, p.waves, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? SLOWMO_OK : fail_thread_hip(e, "slowmo_paged_attention");
  });
}

}  // extern "C"
