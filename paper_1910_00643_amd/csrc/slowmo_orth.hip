// Kernels of the orthogonalising call (include/slowmo_operators.h has the formulas).
//
// Matrix products bound it: 5 steps of X X^T (n n k, half of it by symmetry), A A (n n n, half) and
// P X (2 n n k).  They run on the matrix cores in halves with fp32 sums.  Of the two 16-bit types a
// half has 11 bits and bf16 has 8; X, A and P lie in a range known beforehand, so bf16's exponents buy
// nothing.  A step multiplies small singular values by a = 3.4, so a rounding of X early on comes out
// up to 3.4^5 times as large; X therefore keeps the next 11 bits too (x = hi + lo) until the last two steps,
// which enter where X enters linearly, in a X, while the products take hi alone.  Against 64 bits,
// matrices of 64 to 1024 a side with flat spectra, a few strong directions above noise, or decaying ones:
// 0.8e-3 to 1.5e-3, of deficient rank up to 2.9e-3 (hi alone up to 8.6e-3, products of bf16 up to 7e-2); of 33 to 63 rows
// up to 2.5e-3.  (X's lower bits in the last two steps too: 1.1 to 1.6 times as far off, since P has a on its diagonal
// there, which makes its elements smaller.)
// For fp32 results all factors are such pairs and a product is three: hi hi + hi lo + lo hi, 22 bits.
#include "slowmo_orth.h"

#include <type_traits>
#include <utility>

namespace slowmo {
namespace orth {
namespace {

typedef _Float16 half;
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32;

__device__ __forceinline__ float widen_bf16(uint16_t v) {
  return __builtin_bit_cast(float, static_cast<u32>(v) << 16);
}
__device__ __forceinline__ uint16_t narrow_bf16(float v) {
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
}

// hi + lo of a value already times its power of two.
__device__ __forceinline__ void split_half(float v, half &hi, half &lo) {
  hi = static_cast<half>(v);
  lo = static_cast<half>(v - static_cast<float>(hi));
}

__global__ __launch_bounds__(64) void k_addresses(Addresses *to, Few few, int32_t first, int32_t count) {
  const int i = threadIdx.x;
  if (i < count) to[first + i] = few.at[i];
}

// U at an element of the caller's matrix; with momentum from G and the updated M.
__device__ __forceinline__ float load_input(const Call &c, const Addresses &at, int64_t e) {
  return c.in_bf16 ? widen_bf16(static_cast<const uint16_t *>(at.in)[e])
                   : static_cast<const float *>(at.in)[e];
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ void load8(const float *p, float *v) {
  const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
}
__device__ __forceinline__ void load8(const uint16_t *p, float *v) {
  const u32x4 a = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __builtin_bit_cast(float, a[i] << 16);
    v[2 * i + 1] = __builtin_bit_cast(float, a[i] & 0xffff0000u);
  }
}

// Eight neighbours of a row of the caller's matrix, zeros past its end; `wide`: loads of 16 bytes.
template <typename T>
__device__ __forceinline__ void row8(const T *p, int left, bool wide, float *v) {
  if (wide && left >= 8) {
    load8(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = 0.f;
      if (i < left) {
        if constexpr (sizeof(T) == 2)
          v[i] = widen_bf16(p[i]);
        else
          v[i] = p[i];
      }
    }
  }
}

// Whether rows of a matrix at p, ld elements apart, all start at multiples of 16 bytes.
template <typename T>
__device__ __forceinline__ bool whole_rows(const T *p, int64_t ld) {
  return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(ld * sizeof(T))) & 15) == 0;
}

__device__ __forceinline__ double block_sum(double v, double *shared) {
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
  __syncthreads();
  return shared[0] + shared[1] + shared[2] + shared[3];
}

// A workgroup's share of the sum of squares of U, in 64 bits: squares of fp32 values neither overflow nor
// vanish there.  Updates the momentum on the way.  Memory bounds it: with momentum 5.3 TB/s (93 million fp32
// elements in 211 us), alone 3.9 TB/s (67 million in 68 us).  That U is read again by k_load is the price of not
// knowing its norm; by groups of matrices that the last-level cache would keep between the two, a call took
// 1.00 to 1.15 of the time, since every launch has its ends.
__global__ __launch_bounds__(256) void k_sums(Call c, const Item *items) {
  const Item it = items[blockIdx.x];
  const Matrix &m = c.matrices[it.matrix];
  const Addresses at = c.addresses[it.matrix];
  const u32 rows = m.tall ? m.k : m.n, cols = m.tall ? m.n : m.k, pieces = (cols + 7) / 8;
  const u32 all = rows * pieces, each = (all + it.j - 1) / it.j;  // at most 2^29
  const u32 last = min(all, (it.i + 1) * each);
  double sum = 0.;
  auto walk = [&](auto *in) {
    const bool wide = whole_rows(in, m.ld), wide_m = whole_rows(at.momentum, m.ld);
#pragma unroll 2
    for (u32 q = it.i * each + threadIdx.x; q < last; q += 256) {
      const u32 row = q / pieces, col = (q - row * pieces) * 8;
      const int64_t e = static_cast<int64_t>(row) * m.ld + col;
      const int left = static_cast<int>(cols - col);
      float u[8];
      row8(in + e, left, wide, u);
      if (c.momentum) {
        float h[8];
        row8(at.momentum + e, left, wide_m, h);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = fmaf(c.mu, h[i], u[i]);
        float *to = at.momentum + e;
        if (wide_m && left >= 8) {
          *reinterpret_cast<f32x4 *>(to) = f32x4{h[0], h[1], h[2], h[3]};
          *reinterpret_cast<f32x4 *>(to + 4) = f32x4{h[4], h[5], h[6], h[7]};
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (i < left) to[i] = h[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = c.nesterov ? fmaf(c.mu, h[i], u[i]) : h[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fma(static_cast<double>(u[i]), static_cast<double>(u[i]), sum);
    }
  };
  if (c.in_bf16)
    walk(static_cast<const uint16_t *>(at.in));
  else
    walk(static_cast<const float *>(at.in));
  __shared__ double shared[4];
  sum = block_sum(sum, shared);
  if (threadIdx.x == 0) c.sums[m.first_sum + it.i] = sum;
}

__device__ __forceinline__ double inverse_norm(double squares, float eps) {
  const double norm = sqrt(squares) + static_cast<double>(eps);
  // a matrix of zeros (and eps 0): zeros; an infinity or NaN anywhere: NaN everywhere
  return norm == 0. ? 0. : norm < 1.7e308 ? 1. / norm : __builtin_nan("");
}

// Where eps is large against |U|, X is small for the first steps: its elements times 2^kPowerX would lose their
// bits to a half's smallest numbers.  X is then held times one more power of two, which brings the bound on its norm to
// 0.5..1, where X_0's is with eps small.  The n x n matrices need none: beside a, which P is added to, their
// smallest numbers do not count.
__device__ __forceinline__ int lift(double bound) { return bound > 0. && bound < 0.5 ? -1 - ilogb(bound) : 0; }
// The bound after a step; infinity or NaN: no lift.
__device__ __forceinline__ double grown(double bound, const float *abc) {
  const double b2 = bound * bound;
  return bound * (fabs(static_cast<double>(abc[0])) +
                  b2 * (fabs(static_cast<double>(abc[1])) + b2 * fabs(static_cast<double>(abc[2]))));
}

typedef _Float16 half8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ void split8(const float *v, half8 &hi, half8 &lo) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    half h, l;
    split_half(v[e], h, l);
    hi[e] = h;
    lo[e] = l;
  }
}

// X_0 (n x k, turned if the caller's matrix is tall) as halves hi and lo, with zeros in the padding (which
// an earlier call's NaN may have reached).  Memory bounds it: 4.7 TB/s (93 million fp32 elements with momentum
// in 239 us).  A patch of 64 x 64 turns in shared memory; rows of 65 keep its columns on different banks.
__global__ __launch_bounds__(256) void k_load(Call c, const Item *items) {
  const Item it = items[blockIdx.x];
  const Matrix &m = c.matrices[it.matrix];
  const Addresses at = c.addresses[it.matrix];
  const int rows = m.tall ? m.k : m.n, cols = m.tall ? m.n : m.k, across = m.tall ? m.np : m.kp;
  const Places places(m.np, m.kp, c.buffers);
  half *x = c.arena + m.at, *x_lo = x + places.x_lo(0);
  __shared__ float turn[kPatch][kPatch + 1];
  __shared__ double shared[4];
  double squares = 0.;
  for (int i = threadIdx.x; i < m.sums; i += 256) squares += c.sums[m.first_sum + i];
  squares = block_sum(squares, shared);
  const double by = inverse_norm(squares, c.eps), size = sqrt(squares) * by;
  const int by_power = by > 0. ? ilogb(by) : 0;  // apart: of subnormal matrices the inverse is no fp32 number
  const float inverse = static_cast<float>(ldexp(by, -by_power));
  const int power = by_power + lift(size);
  if (it.i == 0 && it.j == 0 && threadIdx.x == 0) {
    float *gram = c.scales + static_cast<int64_t>(it.matrix) * kScales, *update = gram + kScales / 2;
    const bool pairs = c.buffers == kSquares;
    double bound = size;
    for (int t = 0; t < c.steps;) {
      const int here = lift(bound), first = t;
      bound = grown(bound, c.abc + 3 * t++);
      if (pairs && first == 0) bound = grown(bound, c.abc + 3 * t++);
      const float rest = c.exact && first == 0 ? inverse : 1.f;
      gram[first] = ldexpf(rest * rest, -2 * here);
      update[first] = ldexpf(rest, (t < c.steps ? lift(bound) : 0) - here);
    }
  }
  auto walk = [&](auto *in) {
    const bool wide = whole_rows(in, m.ld), wide_m = whole_rows(at.momentum, m.ld);
    for (int patch = it.j; patch < it.j + kPatches && patch * kPatch < across; ++patch) {
#pragma unroll
      for (int q = threadIdx.x; q < kPatch * kPatch / 8; q += 256) {
        const int r = q >> 3, c8 = (q & 7) * 8, row = it.i * kPatch + r, col = patch * kPatch + c8;
        float u[8] = {};
        if (row < rows && col < cols) {
          const int64_t e = row * m.ld + col;
          row8(in + e, cols - col, wide, u);
          if (c.momentum) {
            float h[8];
            row8(at.momentum + e, cols - col, wide_m, h);
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = c.nesterov ? fmaf(c.mu, h[i], u[i]) : h[i];
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = ldexpf(u[i], power + kPowerX) * (c.exact ? 1.f : inverse);
        if (m.tall) {
#pragma unroll
          for (int i = 0; i < 8; ++i) turn[r][c8 + i] = row < rows && col + i < cols ? u[i] : 0.f;
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) u[i] = row < rows && col + i < cols ? u[i] : 0.f;
          half8 hi, lo;
          split8(u, hi, lo);
          const int64_t to = (static_cast<int64_t>(col >> 5) * m.np + row) * kDeep + (col & 31);
          *reinterpret_cast<half8 *>(x + to) = hi;
          if (!c.exact) *reinterpret_cast<half8 *>(x_lo + to) = lo;
        }
      }
      if (!m.tall) continue;
      __syncthreads();
#pragma unroll
      for (int q = threadIdx.x; q < kPatch * kPatch / 8; q += 256) {
        const int r = q >> 3, c8 = (q & 7) * 8;
        float u[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = turn[c8 + i][r];
        half8 hi, lo;
        split8(u, hi, lo);
        const int n = patch * kPatch + r, k = it.i * kPatch + c8;
        const int64_t to = (static_cast<int64_t>(k >> 5) * m.np + n) * kDeep + (k & 31);
        *reinterpret_cast<half8 *>(x + to) = hi;
        if (!c.exact) *reinterpret_cast<half8 *>(x_lo + to) = lo;
      }
      __syncthreads();
    }
  };
  if (c.in_bf16)
    walk(static_cast<const uint16_t *>(at.in));
  else
    walk(static_cast<const float *>(at.in));
}

// 8 neighbouring results of one row of the caller's matrix (rows x cols, ld apart).
__device__ __forceinline__ void write_out(const Call &c, const Addresses &at, int64_t ld, int row, int rows,
                                          int col, int cols, const float *v, float scale) {
  if (row >= rows || col >= cols) return;
  const int64_t to = row * ld + col;
  if (c.out_bf16) {
    uint16_t *o = static_cast<uint16_t *>(at.out) + to;
    if (col + 8 <= cols && reinterpret_cast<uintptr_t>(o) % 16 == 0) {
      typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
      bf16x8 w;
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = static_cast<__bf16>(v[e] * scale);
      *reinterpret_cast<bf16x8 *>(o) = w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (col + e < cols) o[e] = narrow_bf16(v[e] * scale);
    }
  } else {
    float *o = static_cast<float *>(at.out) + to;
    if (col + 8 <= cols && reinterpret_cast<uintptr_t>(o) % 16 == 0) {
      *reinterpret_cast<f32x4 *>(o) = f32x4{v[0] * scale, v[1] * scale, v[2] * scale, v[3] * scale};
      *reinterpret_cast<f32x4 *>(o + 4) = f32x4{v[4] * scale, v[5] * scale, v[6] * scale, v[7] * scale};
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (col + e < cols) o[e] = v[e] * scale;
    }
  }
}

// ---- products -----------------------------------------------------------------
//
// Tiles of B x A by 4 waves of B/2 x A/2, where A runs along the result's rows.  Steps of 32 of the summed side
// go from memory straight to a ring of STAGES stages in shared memory (16 bytes a lane), STAGES - 1 steps ahead
// of their use.  A wave reads the next step's factors into registers between the products of this one, so that
// the matrix cores go on with one wave per SIMD too (B = 256: 256 accumulators a lane).
//
// What bounds them: 8192 x 8192 (256 x 256) the matrix cores at the clock that their power leaves, 1.09e15
// flop/s over the whole call, where a library's product of that size reaches 1.11e15.  (All 512 registers of a lane
// are taken; 4 to 52 more, 20 to 212 bytes, go to scratch memory in front of the loops and behind them.)  The smaller tiles are
// bound by the way from L2 to shared memory, 12.7 TB/s for 16 KB a step of 128 x 128 (0.33 us with every CU at
// work, 0.13 us of it products): 0.75e15 in lists of many matrices; and a launch of one round by its ends, 8 us
// of 16 (1024 x 1024 x 1024, 216 tiles).
//
// X and the n x n matrices lie in panels of 32 columns, [column / 32][row][column mod 32]: a step's share of a
// factor is one piece of memory (P X's X: one per panel) and every cache line of it is used whole.  (Rows
// after rows, a step's 64 bytes of each cost as many requests to L2 as 128, and L2 is what bounds the smaller
// tiles.)  In shared memory a row's 64 bytes are four pieces; where a factor is read along its rows,
// piece p of row r lies at p xor (r / 4 mod 4), so that 16 lanes that read the same piece of neighbouring
// rows meet all 64 banks once.  X of P X has the summed side down its columns: it is read turned, 4 rows x
// 16 columns per 16 lanes, which meets all banks as it lies.
// Everything is padded to whole tiles; nothing is checked in the loop.
//
// Pairs of halves: a panel's hi lo, lo hi and hi hi are two stages and three products, the third of what the
// other two left in registers; loads and reads per product are 2/3 of three passes' over the summed side, and
// what a pass would fetch again is at hand (a list of ResNet-18's matrices for 8 workers, X in 370 MB: its
// X X^T 242 -> 156 us, with P X 2.97 -> 2.45 ms a call; errors as before within 1.1).
// A tile of the diagonal of a matrix times itself needs one side's rows alone: 32 x 768 x 2560, 1.13 ->
// 1.10 ms a call.

// m0 is written and read within the block, with the one wait between that the two need; no vector register
// is written.  `base` comes from scalar instructions.
__device__ __forceinline__ void to_shared(u32 shared, u32 offset, const half *base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(shared), "v"(offset), "s"(base)
               : "memory");
}
// All but the N newest loads of this wave have arrived, its reads of shared memory are done, and so it is
// for every wave of the workgroup.
template <int N>
__device__ __forceinline__ void arrive() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <int... N, typename F>
__device__ __forceinline__ void each(std::integer_sequence<int, N...>, F &&f) {
  (f(std::integral_constant<int, N>{}), ...);
}

typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));

// UPDATE: P X by Update, else a symmetric product by Symmetric.
template <int A, int B, int STAGES, bool UPDATE, bool SPLIT>
__global__ __launch_bounds__(256, B == 256 ? 1 : A == 256 ? 2 : 3) void k_products(
    Call c, std::conditional_t<UPDATE, Update, Symmetric> st, const Tile *tiles) {
  extern __shared__ half ring[];
  constexpr int kBlocksA = A / 64, kBlocksB = B / 64;  // blocks of 32 x 32 along the sides of a wave's share
  constexpr int kShareA = A * kDeep, kStage = (A + B) * kDeep;  // halves of a stage
  constexpr int kLoadsA = A / 64, kLoadsB = B / 64;    // loads of a wave per stage
  constexpr int kWideA = A / 2, kWideB = B / 2;        // sides of a wave's share
  const Tile it = tiles[blockIdx.x];
  const Places places(it.np, it.kp, c.buffers);
  half *const arena = c.arena + it.at;
  // asked for ahead of the products
  const float held = st.scale >= 0 ? c.scales[static_cast<int64_t>(it.matrix) * kScales + st.scale] : 1.f;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wa = wave & 1, wb = wave >> 1;
  const int low = lane & 31, high = lane >> 5;

  // factor a: columns of the tile (j), factor b: rows (i).  The accumulators' four neighbours run along a.
  int64_t a_hi, a_lo, b_hi, b_lo;
  if constexpr (UPDATE) {
    a_hi = places.x(st.from);
    a_lo = places.x_lo(st.from);
    b_hi = places.buffer(st.by);
    b_lo = places.buffer_lo(st.by);
  } else if (st.left < 0) {
    a_hi = b_hi = places.x(st.from);
    a_lo = b_lo = places.x_lo(st.from);
  } else {
    a_hi = places.buffer(st.right);
    a_lo = places.buffer_lo(st.right);
    b_hi = places.buffer(st.left);
    b_lo = places.buffer_lo(st.left);
  }
  const int64_t panel = static_cast<int64_t>(it.np) * kDeep;
  const int64_t a_at = UPDATE ? static_cast<int64_t>(it.j) * (A / kDeep) * panel : static_cast<int64_t>(it.j) * A * kDeep;
  const int64_t a_step = UPDATE ? kDeep * kDeep : panel;
  const int64_t b_at = static_cast<int64_t>(it.i) * B * kDeep;

  // bytes of a lane's piece within a load's 1024: 16 rows of 4 pieces
  const u32 b_off = ((lane & ~3) | ((lane & 3) ^ ((lane >> 4) & 3))) * 16, a_off = UPDATE ? lane * 16 : b_off;
  const u32 shared0 = static_cast<u32>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) half *)ring));

  // A tile of the diagonal of a matrix times itself, of single halves: both factors are the same rows, so that
  // a stage holds two neighbouring panels of them and serves two steps.  The diagonal's list counts two as one.
  const bool twice = !UPDATE && !SPLIT && it.i == it.j;
  bool own = false;
  if constexpr (!UPDATE) own = twice && st.left == st.right;
  const int total = (SPLIT || (twice && !own)) ? 2 * it.count : it.count;  // stages
  const int first = twice && !own ? 2 * it.first : it.first;

  // The next stage to fetch.  Of pairs of halves a panel is two stages, a's hi with b's lo, then a's lo with
  // b's hi.
  const int64_t a_stride = own ? 2 * panel : a_step, b_stride = own ? 2 * panel : panel;
  const half *a_next = arena + a_hi + a_at + wave * kLoadsA * (UPDATE ? panel / 2 : 512) + first * a_stride;
  const half *b_next = arena + b_hi + b_at + wave * kLoadsB * 512 + first * b_stride + (own ? panel : 0);
  const int64_t a_other = a_lo - a_hi, b_other = b_lo - b_hi;
  constexpr int kStep = kLoadsA + kLoadsB;  // loads of a wave in a stage
  auto fetch_one = [&](int slot, int second, int q) {
    const u32 to = shared0 + slot * (kStage * 2);
    const half *a = a_next, *b = b_next;
    if (SPLIT && second) a += a_other;
    if (SPLIT && !second) b += b_other;
    if (q < kLoadsA)  // of X for P X, two loads to a panel's 32 rows
      to_shared(to + (wave * kLoadsA + q) * 1024, a_off, a + (UPDATE ? (q >> 1) * panel + (q & 1) * 512 : q * 512));
    else
      to_shared(to + kShareA * 2 + (wave * kLoadsB + q - kLoadsA) * 1024, b_off, b + (q - kLoadsA) * 512);
  };
  auto fetched = [&](int second) {
    if (SPLIT && !second) return;
    a_next += a_stride;
    b_next += b_stride;
  };

  half8 fa[2][2][kBlocksA], fb[2][2][kBlocksB];  // of this step and of the next, 16 deep each
  constexpr int kReads = 2 * (kBlocksA + kBlocksB);
  auto read_b = [&](const half *sb, int which, int kk, int y) {
    const int rb = wb * kWideB + y * 32 + low;
    fb[which][kk][y] = *reinterpret_cast<const half8 *>(sb + rb * kDeep + (((kk * 2 + high) ^ ((rb >> 2) & 3)) * 8));
  };
  auto read_a = [&](const half *sa, int which, int kk, int x) {
    if constexpr (UPDATE) {
      const int r = kk * 16 + high * 8 + ((lane >> 2) & 3), col = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
      const half *from = sa + ((wa * kWideA / 32 + x) * kDeep + r) * kDeep + col;
      typedef __attribute__((address_space(3))) short4v *shared4;
      const short4v lo4 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared4)(from));
      const short4v hi4 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared4)(from + 4 * kDeep));
      fa[which][kk][x] = __builtin_bit_cast(half8, __builtin_shufflevector(lo4, hi4, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      const int ra = wa * kWideA + x * 32 + low;
      fa[which][kk][x] = *reinterpret_cast<const half8 *>(sa + ra * kDeep + (((kk * 2 + high) ^ ((ra >> 2) & 3)) * 8));
    }
  };
  // read q of a stage's kReads, of a to registers to_a, of b to to_b
  auto read_one = [&](const half *sa, const half *sb, int to_a, int to_b, int q) {
    const int kk = q / (kBlocksA + kBlocksB), f = q % (kBlocksA + kBlocksB);
    if (f < kBlocksB)
      read_b(sb, to_b, kk, f);
    else
      read_a(sa, to_a, kk, f - kBlocksB);
  };

  f32x16 acc[kBlocksA][kBlocksB];
#pragma unroll
  for (int x = 0; x < kBlocksA; ++x)
#pragma unroll
    for (int y = 0; y < kBlocksB; ++y)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[x][y][r] = 0.f;
  constexpr int kProducts = 2 * kBlocksA * kBlocksB;
  auto multiply_one = [&](int of_a, int of_b, int q) {
    const int kk = q / (kBlocksA * kBlocksB), x = q / kBlocksB % kBlocksA, y = q % kBlocksB;
    acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[of_a][kk][x], fb[of_b][kk][y], acc[x][y], 0, 0, 0);
  };

  for (int s = 0; s < STAGES && s < total; ++s) {
#pragma unroll
    for (int q = 0; q < kStep; ++q) fetch_one(s, s & 1, q);
    fetched(s & 1);
  }
  if (total >= STAGES)
    arrive<kStep * (STAGES - 1)>();
  else
    arrive<0>();
  int left_steps = total, slot = 0;
  std::integral_constant<int, 0> even;
  std::integral_constant<int, 1> odd;
  std::integral_constant<int, kStep * (STAGES - 2)> full;
  // One step: the next one's factors go to registers while this one's are multiplied.  `pending` loads may
  // still be on their way when the next step's have arrived.  Reads and loads are issued one by one between
  // products: a wave issues in order, and in a row they hold it up for as long as the products take.
  auto step = [&](auto odd, auto pending, auto more) {
    constexpr int kThis = decltype(odd)::value;
    const int here = slot;
    slot = slot + 1 == STAGES ? 0 : slot + 1;
    __builtin_amdgcn_sched_barrier(0);  // the products before run on while this wave waits
    arrive<decltype(pending)::value>();
    each(std::make_integer_sequence<int, kProducts>{}, [&](auto i) {
      constexpr int I = decltype(i)::value;
#pragma unroll
      for (int q = I * kReads / kProducts; q < (I + 1) * kReads / kProducts; ++q)
        read_one(ring + slot * kStage, ring + slot * kStage + kShareA, 1 - kThis, 1 - kThis, q);
      if constexpr (decltype(more)::value) {  // to where this step was: everybody has read it
#pragma unroll
        for (int q = I * kStep / kProducts; q < (I + 1) * kStep / kProducts; ++q) fetch_one(here, 0, q);
      }
      multiply_one(kThis, kThis, I);
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (decltype(more)::value) fetched(0);
    --left_steps;
  };
  if (!SPLIT && (UPDATE || !own)) {
    // the factors of a step with r left are in registers r mod 2
#pragma unroll
    for (int q = 0; q < kReads; ++q) {
      if (total & 1)
        read_one(ring, ring + kShareA, 1, 1, q);
      else
        read_one(ring, ring + kShareA, 0, 0, q);
    }
    if (left_steps > STAGES && (left_steps & 1)) step(odd, full, std::true_type{});
    while (left_steps - 1 > STAGES) {
      step(even, full, std::true_type{});
      step(odd, full, std::true_type{});
    }
    if (left_steps > STAGES) step(even, full, std::true_type{});
    // nothing is left to fetch; what is on its way arrives one step after the other
    each(std::make_integer_sequence<int, STAGES - 1>{}, [&](auto n) {
      constexpr int kLeft = STAGES - decltype(n)::value;
      if (left_steps == kLeft)
        step(std::integral_constant<int, (kLeft & 1)>{}, std::integral_constant<int, kStep * (kLeft - 2)>{}, std::false_type{});
    });
  }
  if constexpr (!UPDATE && !SPLIT) {
    // The same with two steps to a stage: a stage's first is in registers 0, its second in registers 1.
    auto first_half = [&] {  // the second one's factors go to registers
      each(std::make_integer_sequence<int, kProducts>{}, [&](auto i) {
        constexpr int I = decltype(i)::value;
#pragma unroll
        for (int q = I * kReads / kProducts; q < (I + 1) * kReads / kProducts; ++q)
          read_one(ring + slot * kStage + kShareA, ring + slot * kStage + kShareA, 1, 1, q);
        multiply_one(0, 0, I);
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    auto stage = [&](auto pending, auto more) {
      __builtin_amdgcn_sched_barrier(0);
      first_half();
      const int here = slot;
      slot = slot + 1 == STAGES ? 0 : slot + 1;
      arrive<decltype(pending)::value>();
      each(std::make_integer_sequence<int, kProducts>{}, [&](auto i) {
        constexpr int I = decltype(i)::value;
#pragma unroll
        for (int q = I * kReads / kProducts; q < (I + 1) * kReads / kProducts; ++q)
          read_one(ring + slot * kStage, ring + slot * kStage, 0, 0, q);
        if constexpr (decltype(more)::value) {
#pragma unroll
          for (int q = I * kStep / kProducts; q < (I + 1) * kStep / kProducts; ++q) fetch_one(here, 0, q);
        }
        multiply_one(1, 1, I);
        __builtin_amdgcn_sched_barrier(0);
      });
      if constexpr (decltype(more)::value) fetched(0);
      --left_steps;
    };
    if (own) {
#pragma unroll
      for (int q = 0; q < kReads; ++q) read_one(ring, ring, 0, 0, q);
      while (left_steps > STAGES) stage(full, std::true_type{});
      each(std::make_integer_sequence<int, STAGES - 1>{}, [&](auto n) {
        constexpr int kLeft = STAGES - decltype(n)::value;
        if (left_steps == kLeft) stage(std::integral_constant<int, kStep * (kLeft - 2)>{}, std::false_type{});
      });
      first_half();
    }
  }
  if constexpr (SPLIT) {
    // A panel: hi lo, lo hi, and, of what both left in registers, hi hi: three products for two stages' loads and
    // reads.  The first product's factors are fa[type] and fb[0], the second's fa[1 - type] and fb[1], so that
    // the third's are fa[type] and fb[1] and the next panel, of the other type, has the rest.  `left`: stages
    // left, this panel's included, or more than STAGES + 1.
    auto panel_of = [&](auto type_, auto left_) {
      constexpr int T = decltype(type_)::value, L = decltype(left_)::value;
      constexpr bool kMore0 = L > STAGES, kMore1 = L > STAGES + 1, kLast = L == 2;
      int here = slot;
      slot = slot + 1 == STAGES ? 0 : slot + 1;
      __builtin_amdgcn_sched_barrier(0);
      arrive<kStep * ((kMore0 ? STAGES : L) - 2)>();
      each(std::make_integer_sequence<int, kProducts>{}, [&](auto i) {
        constexpr int I = decltype(i)::value;
#pragma unroll
        for (int q = I * kReads / kProducts; q < (I + 1) * kReads / kProducts; ++q)
          read_one(ring + slot * kStage, ring + slot * kStage + kShareA, 1 - T, 1, q);
        if constexpr (kMore0) {
#pragma unroll
          for (int q = I * kStep / kProducts; q < (I + 1) * kStep / kProducts; ++q) fetch_one(here, STAGES & 1, q);
        }
        multiply_one(T, 0, I);
        __builtin_amdgcn_sched_barrier(0);
      });
      if constexpr (kMore0) fetched(STAGES & 1);
      here = slot;
      if constexpr (!kLast) {
        slot = slot + 1 == STAGES ? 0 : slot + 1;
        __builtin_amdgcn_sched_barrier(0);
        arrive<kStep * ((kMore1 ? STAGES : L - 1) - 2)>();
      }
      constexpr int kReadsA = 2 * kBlocksA, kReadsB = 2 * kBlocksB;
      each(std::make_integer_sequence<int, kProducts>{}, [&](auto i) {
        constexpr int I = decltype(i)::value;
        if constexpr (!kLast) {
#pragma unroll
          for (int q = I * kReadsB / kProducts; q < (I + 1) * kReadsB / kProducts; ++q)
            read_b(ring + slot * kStage + kShareA, 0, q / kBlocksB, q % kBlocksB);
        }
        if constexpr (kMore1) {
#pragma unroll
          for (int q = I * kStep / kProducts; q < (I + 1) * kStep / kProducts; ++q) fetch_one(here, 1 - (STAGES & 1), q);
        }
        multiply_one(1 - T, 1, I);
        __builtin_amdgcn_sched_barrier(0);
      });
      if constexpr (kMore1) fetched(1 - (STAGES & 1));
      each(std::make_integer_sequence<int, kProducts>{}, [&](auto i) {
        constexpr int I = decltype(i)::value;
        if constexpr (!kLast) {
#pragma unroll
          for (int q = I * kReadsA / kProducts; q < (I + 1) * kReadsA / kProducts; ++q)
            read_a(ring + slot * kStage, 1 - T, q / kBlocksA, q % kBlocksA);
        }
        multiply_one(T, 1, I);
        __builtin_amdgcn_sched_barrier(0);
      });
      left_steps -= 2;
    };
    std::integral_constant<int, 1 << 20> many;
    // a panel with r stages left is of type r / 2 mod 2
#pragma unroll
    for (int q = 0; q < kReads; ++q) {
      if (total & 2)
        read_one(ring, ring + kShareA, 1, 0, q);
      else
        read_one(ring, ring + kShareA, 0, 0, q);
    }
    if (left_steps > STAGES + 1 && (left_steps & 2)) panel_of(odd, many);
    while (left_steps - 2 > STAGES + 1) {
      panel_of(even, many);
      panel_of(odd, many);
    }
    if (left_steps > STAGES + 1) panel_of(even, many);
    each(std::make_integer_sequence<int, (STAGES + 1) / 2>{}, [&](auto n) {
      constexpr int kLeft = ((STAGES + 1) / 2 - decltype(n)::value) * 2;
      if (left_steps == kLeft) panel_of(std::integral_constant<int, (kLeft / 2) & 1>{}, std::integral_constant<int, kLeft>{});
    });
  } else {
    each(std::make_integer_sequence<int, kProducts>{}, [&](auto i) { multiply_one(1, 1, decltype(i)::value); });
  }

  // A tile in several shares: each leaves its sums in memory, and the one that comes last adds them all
  // up, in their order whichever it is.  The sums pass the dies' separate L2 caches by themselves (8 bytes
  // at a time, at the scope of the whole card); a fence would write all of L2 back, 120 us a launch.
  if (it.pieces > 1) {
    typedef unsigned long long two;
    constexpr int64_t kTileSums = static_cast<int64_t>(A) * B / 2;
    two *sums = reinterpret_cast<two *>(c.partial) + it.slot * kTileSums + threadIdx.x;
#pragma unroll
    for (int x = 0; x < kBlocksA; ++x)
#pragma unroll
      for (int y = 0; y < kBlocksB; ++y)
#pragma unroll
        for (int g = 0; g < 8; ++g)
          __hip_atomic_store(sums + it.piece * kTileSums + ((x * kBlocksB + y) * 8 + g) * 256,
                             __builtin_bit_cast(two, f32x2{acc[x][y][2 * g], acc[x][y][2 * g + 1]}),
                             __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // they have reached memory
    __syncthreads();
    u32 *flag = reinterpret_cast<u32 *>(ring);
    if (threadIdx.x == 0) {
      const u32 before = __hip_atomic_fetch_add(c.tickets + it.ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (before + 1 == static_cast<u32>(it.pieces))
        __hip_atomic_store(c.tickets + it.ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      flag[0] = before;
    }
    __syncthreads();
    if (flag[0] + 1 != static_cast<u32>(it.pieces)) return;
#pragma unroll
    for (int x = 0; x < kBlocksA; ++x)
#pragma unroll
      for (int y = 0; y < kBlocksB; ++y) {
        f32x16 v;
#pragma unroll
        for (int r = 0; r < 16; ++r) v[r] = 0.f;
        for (int p = 0; p < it.pieces; ++p)
#pragma unroll
          for (int g = 0; g < 8; ++g) {
            const f32x2 w = __builtin_bit_cast(
                f32x2, __hip_atomic_load(sums + p * kTileSums + ((x * kBlocksB + y) * 8 + g) * 256, __ATOMIC_RELAXED,
                                         __HIP_MEMORY_SCOPE_AGENT));
            v[2 * g] += w[0];
            v[2 * g + 1] += w[1];
          }
        acc[x][y] = v;
      }
  }
  __syncthreads();

  const bool bare = st.first_step && c.exact;  // X_0 without its factor and lower halves
  const int ai = it.j * A + wa * kWideA, bi = it.i * B + wb * kWideB;  // first place along each factor
  if constexpr (UPDATE) {
    if (st.last) {
      // The caller's rows: results pass through shared memory, 32 rows of a wave's share at a time.
      constexpr int kPitch = (kWideA > kWideB ? kWideA : kWideB) + 4;
      float *stage = reinterpret_cast<float *>(ring) + wave * 32 * kPitch;
      const Matrix &m = c.matrices[it.matrix];
      const Addresses at = c.addresses[it.matrix];
      // X's power of two by itself: together with the others it may be below fp32's numbers
      const bool lifted = held > 0.f && held < 1.f;
      const float lower = lifted ? held : 1.f, scale = m.scale * (st.alpha * (lifted ? 1.f : held)) * (1.f / kScaleX);
      auto leave = [&](auto wide, int row0, int rows, int col0, int cols) {
        constexpr int kLanes = decltype(wide)::value / 8, kRows = 64 / kLanes;
        const int sub = lane / kLanes, c8 = (lane % kLanes) * 8;
#pragma unroll 1  // code that runs once comes slowly: short is fast
        for (int r = 0; r < 32; r += kRows) {
          const f32x4 p = *reinterpret_cast<const f32x4 *>(stage + (r + sub) * kPitch + c8),
                      q = *reinterpret_cast<const f32x4 *>(stage + (r + sub) * kPitch + c8 + 4);
          const float v[8] = {p[0] * lower, p[1] * lower, p[2] * lower, p[3] * lower,
                              q[0] * lower, q[1] * lower, q[2] * lower, q[3] * lower};
          write_out(c, at, m.ld, row0 + r + sub, rows, col0 + c8, cols, v, scale);
        }
      };
      if (m.tall) {  // k x n: rows along factor a
#pragma unroll
        for (int x = 0; x < kBlocksA; ++x) {
#pragma unroll
          for (int y = 0; y < kBlocksB; ++y)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              stage[((r >> 2) * 8 + high * 4 + (r & 3)) * kPitch + y * 32 + low] = acc[x][y][r];
          leave(std::integral_constant<int, kWideB>{}, ai + x * 32, m.k, bi, m.n);
        }
      } else {
#pragma unroll
        for (int y = 0; y < kBlocksB; ++y) {
#pragma unroll
          for (int x = 0; x < kBlocksA; ++x)
#pragma unroll
            for (int g = 0; g < 4; ++g)
              *reinterpret_cast<f32x4 *>(stage + low * kPitch + x * 32 + g * 8 + high * 4) =
                  f32x4{acc[x][y][4 * g], acc[x][y][4 * g + 1], acc[x][y][4 * g + 2], acc[x][y][4 * g + 3]};
          leave(std::integral_constant<int, kWideA>{}, bi + y * 32, m.n, ai, m.k);
        }
      }
      return;
    }
  }

  const float alpha = st.alpha * held, beta = UPDATE ? st.beta * held : st.beta;
  // A block of 32 x 32 is 2 KB in one piece, row `low` of it 64 bytes of which a lane holds four times 8.
  // It passes through shared memory to leave in stores of 1 KB; read turned there, it is its
  // mirror image's block.  Pieces of 16 bytes are placed as the factors' are.
  half *block = ring + wave * 2048;  // hi, lo
  auto place = [&](int row, int col) { return row * kDeep + (((col >> 3) ^ ((row >> 2) & 3)) * 8) + (col & 7); };
  auto where = [&](int row, int col) { return static_cast<int64_t>(col >> 5) * panel + static_cast<int64_t>(row) * kDeep; };
  auto put = [&](int part, int g, const half4 &v) {
    *reinterpret_cast<half4 *>(block + part * 1024 + place(low, g * 8 + high * 4)) = v;
  };
  auto leave = [&](int part, half *to) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int row = q * 16 + (lane >> 2), col = (lane & 3) * 8;
      *reinterpret_cast<half8 *>(to + row * kDeep + col) =
          *reinterpret_cast<const half8 *>(block + part * 1024 + place(row, col));
    }
  };
  auto leave_turned = [&](int part, half *to) {
    typedef __attribute__((address_space(3))) short4v *shared4;
#pragma unroll
    for (int q = 0; q < 2; ++q) {  // column q * 16 + lane mod 16, rows (lane / 16) * 8 and on
      const int row = (lane >> 4) * 8 + ((lane >> 2) & 3), col = q * 16 + (lane & 3) * 4;
      const short4v v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared4)(block + part * 1024 + place(row, col)));
      const short4v v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared4)(block + part * 1024 + place(row + 4, col)));
      *reinterpret_cast<short8v *>(to + (q * 16 + (lane & 15)) * kDeep + (lane >> 4) * 8) =
          __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  };
  auto four = [&](const half *from, int g) { return *reinterpret_cast<const half4 *>(from + low * kDeep + g * 8 + high * 4); };
#pragma unroll
  for (int y = 0; y < kBlocksB; ++y) {
    // What is added to a row of blocks, all of it asked for before any of it is used.
    constexpr int kMore = UPDATE || !SPLIT ? 2 : 4;
    half4 more[kBlocksA][kMore][4];
    asm volatile("" ::: "memory");  // and no earlier: the registers would not hold it
#pragma unroll
    for (int x = 0; x < kBlocksA; ++x) {
      const int64_t pos = where(bi + y * 32, ai + x * 32);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        if constexpr (UPDATE) {
          if (st.carry) {
            more[x][0][g] = four(arena + places.x(st.from) + pos, g);
            if (!bare) more[x][1][g] = four(arena + places.x_lo(0) + pos, g);
          }
        } else {
          constexpr int kNext = SPLIT ? 2 : 1;
          if (st.first >= 0) {
            more[x][0][g] = four(arena + places.buffer(st.first) + pos, g);
            if (SPLIT) more[x][1][g] = four(arena + places.buffer_lo(st.first) + pos, g);
          }
          if (st.second >= 0) {
            more[x][kNext][g] = four(arena + places.buffer(st.second) + pos, g);
            if (SPLIT) more[x][kNext + 1][g] = four(arena + places.buffer_lo(st.second) + pos, g);
          }
        }
      }
    }
#pragma unroll
    for (int x = 0; x < kBlocksA; ++x) {
      const int row0 = bi + y * 32, col0 = ai + x * 32;
      const int64_t pos = where(row0, col0);
      half4 hi[4], lo[4];
#pragma unroll
      for (int g = 0; g < 4; ++g) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v = acc[x][y][4 * g + e] * alpha;
          if constexpr (UPDATE) {
            if (st.carry)
              v = fmaf(beta, static_cast<float>(more[x][0][g][e]) + (bare ? 0.f : static_cast<float>(more[x][1][g][e])), v);
          } else {
            auto value = [&](int which) {
              const float h = static_cast<float>(more[x][which][g][e]);
              return SPLIT ? h + static_cast<float>(more[x][which + 1][g][e]) : h;
            };
            if (st.first >= 0) v = fmaf(beta, value(0), v);
            if (st.second >= 0) v = fmaf(st.gamma, value(SPLIT ? 2 : 1), v);
            if (row0 + low == col0 + g * 8 + high * 4 + e) v += st.delta;
          }
          half h, l;
          split_half(v, h, l);
          hi[g][e] = h;
          lo[g][e] = l;
        }
      }
      const bool keep_lo = SPLIT || (UPDATE && [&] { if constexpr (UPDATE) return st.carry_next != 0; else return false; }());
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        put(0, g, hi[g]);
        if (keep_lo) put(1, g, lo[g]);
      }
      if constexpr (UPDATE) {
        leave(0, arena + places.x(1 - st.from) + pos);
        if (keep_lo) leave(1, arena + places.x_lo(SPLIT ? 1 - st.from : 0) + pos);
      } else {
        leave(0, arena + places.buffer(st.out) + pos);
        if (SPLIT) leave(1, arena + places.buffer_lo(st.out) + pos);
        if (it.i != it.j) {
          const int64_t mirror = where(col0, row0);
          leave_turned(0, arena + places.buffer(st.out) + mirror);
          if (SPLIT) leave_turned(1, arena + places.buffer_lo(st.out) + mirror);
        }
      }
    }
  }
}

// A matrix of few rows from its load to its store: one workgroup.  There is so little work that it is done in
// 64 bits: with few directions (a rank of one or two) the largest singular values of X_0 are near 1, the early
// steps' roundings enter in full, and fp32 sums alone would cost a fp32 result five of its bits.  In 64 bits
// A = U U^T has all that the steps need: with B_0 = I and A_0 = A / |U|^2 a step is
//   G = a I + b A + c A A;   B <- G B;   A <- G (G A)
// (polynomials of the same A, so that they commute), n^3 each, and the result is s B U / |U|.  U is read
// twice, in chunks that fit shared memory; the n x n products take blocks of 2 x 2 a thread, of which
// shared memory's reads are what bounds them.  32 x 128: 53 us (with the steps on X itself, n n k each, 293); 256
// of them 62 us; 4 x 4 12 us.
__global__ __launch_bounds__(kTinyThreads) void k_tiny(Call c, Steps steps, const int32_t *list) {
  constexpr int kPitch = kTinySide;
  __shared__ float x[kTinyElements + kTinySide];
  __shared__ __align__(16) double matrices[5][kTinySide * kPitch];
  double *const gram = matrices[0], *const g = matrices[1], *const turn = matrices[2];
  double *b = matrices[3], *b_next = matrices[4];
  const int at_matrix = list[blockIdx.x];
  const Matrix &m = c.matrices[at_matrix];
  const Addresses at = c.addresses[at_matrix];
  const int n = m.n, k = m.k, tid = threadIdx.x, lane = tid & 63;
  const int chunk = min(k, kTinyElements / n), pitch = chunk | 1;  // odd: a column's elements on different banks

  // U from column k0 on, in the caller's order of memory
  auto fill = [&](int k0, int width, bool once) {
    for (int e = tid; e < n * width; e += kTinyThreads) {
      const int i = m.tall ? e % n : e / width, q = m.tall ? e / n : e % width;
      const int64_t from = m.tall ? (k0 + q) * m.ld + i : i * m.ld + k0 + q;
      float u = load_input(c, at, from);
      if (c.momentum) {
        float h = at.momentum[from];
        if (once) {
          h = fmaf(c.mu, h, u);
          at.momentum[from] = h;
        }
        u = c.nesterov ? fmaf(c.mu, h, u) : h;
      }
      x[i * pitch + q] = u;
    }
  };
  for (int e = tid; e < n * kPitch; e += kTinyThreads) gram[e] = 0.;
  // a group of lanes per element of A: few elements have long rows, many have short ones
  const int log2 = n <= 4 ? 6 : n <= 12 ? 4 : 3, lanes = 1 << log2;
  for (int k0 = 0; k0 < k; k0 += chunk) {
    const int width = min(chunk, k - k0);
    fill(k0, width, true);
    __syncthreads();
    for (int e = tid >> log2; e < n * n; e += kTinyThreads >> log2) {
      const int i = e / n, j = e - i * n;
      if (j > i) continue;
      double dot = 0.;
      for (int q = lane & (lanes - 1); q < width; q += lanes)
        dot = fma(static_cast<double>(x[i * pitch + q]), static_cast<double>(x[j * pitch + q]), dot);
      for (int o = lanes >> 1; o; o >>= 1) dot += __shfl_xor(dot, o);
      if ((lane & (lanes - 1)) == 0) {
        dot += gram[i * kPitch + j];
        gram[i * kPitch + j] = dot;
        gram[j * kPitch + i] = dot;
      }
    }
    __syncthreads();
  }
  double squares = 0.;
  for (int i = 0; i < n; ++i) squares += gram[i * kPitch + i];
  const double inverse = inverse_norm(squares, c.eps);
  __syncthreads();
  for (int e = tid; e < n * kPitch; e += kTinyThreads) gram[e] *= inverse * inverse;
  __syncthreads();

  const int half_n = (n + 1) / 2;  // past n: the padding, which reaches nothing else
  auto product = [&](const double *left, const double *right, auto &&to) {
    for (int block = tid; block < half_n * half_n; block += kTinyThreads) {
      const int i = block / half_n * 2, j = (block - block / half_n * half_n) * 2;
      double v[2][2] = {};
#pragma unroll 4
      for (int q = 0; q < n; ++q) {
        const double r0 = right[q * kPitch + j], r1 = right[q * kPitch + j + 1];
        const double l0 = left[i * kPitch + q], l1 = left[(i + 1) * kPitch + q];
        v[0][0] = fma(l0, r0, v[0][0]);
        v[0][1] = fma(l0, r1, v[0][1]);
        v[1][0] = fma(l1, r0, v[1][0]);
        v[1][1] = fma(l1, r1, v[1][1]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) to(i + (e >> 1), j + (e & 1), v[e >> 1][e & 1]);
    }
  };
  for (int t = 0; t < steps.count; ++t) {
    const double a0 = steps.abc[t][0], b0 = steps.abc[t][1], c0 = steps.abc[t][2];
    product(gram, gram, [&](int i, int j, double v) {
      v = b0 * gram[i * kPitch + j] + c0 * v + (i == j ? a0 : 0.);
      g[i * kPitch + j] = v;
      if (t == 0) b[i * kPitch + j] = v;
    });
    __syncthreads();
    if (t > 0) product(g, b, [&](int i, int j, double v) { b_next[i * kPitch + j] = v; });
    if (t + 1 < steps.count) {
      product(g, gram, [&](int i, int j, double v) { turn[i * kPitch + j] = v; });
      __syncthreads();
      product(g, turn, [&](int i, int j, double v) { gram[i * kPitch + j] = v; });
    }
    if (t > 0) {
      double *const old = b;
      b = b_next;
      b_next = old;
    }
    __syncthreads();
  }

  const double factor = inverse * static_cast<double>(m.scale);
  constexpr int kRows = 8;  // of a column, a thread
  for (int k0 = 0; k0 < k; k0 += chunk) {
    const int width = min(chunk, k - k0);
    if (chunk < k) {
      __syncthreads();
      fill(k0, width, false);
      __syncthreads();
    }
    for (int e = tid; e < (n + kRows - 1) / kRows * width; e += kTinyThreads) {
      const int r0 = e / width * kRows, q = e - e / width * width;
      double v[kRows] = {};
      for (int j = 0; j < n; ++j) {
        const double u = x[j * pitch + q];
#pragma unroll
        for (int r = 0; r < kRows; ++r) v[r] = fma(b[(r0 + r) * kPitch + j], u, v[r]);
      }
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        if (r0 + r >= n) break;
        const float o = static_cast<float>(v[r] * factor);
        const int64_t to = m.tall ? (k0 + q) * m.ld + r0 + r : (r0 + r) * m.ld + k0 + q;
        if (c.out_bf16)
          static_cast<uint16_t *>(at.out)[to] = narrow_bf16(o);
        else
          static_cast<float *>(at.out)[to] = o;
      }
    }
  }
}

// A small matrix from its load to its store: one workgroup, all steps, X, A and P as halves in shared
// memory, in panels of 32 columns as the products' factors lie there.  A call is one launch instead of 17:
// launches, each with its way to memory and back, are all that such a call takes.  N: 128, or 64 for pairs of
// halves, and the side of the tiles of X that are replaced one after the other; 4 waves have a quarter of
// a tile each.  128 x 96: 42 us where the launches of the products take 98; 64 x 64: 14 us.  A step takes 5.6 us at
// 128, most of it the turns from accumulators to halves and back; the rest is the way of code that runs once.
template <int N, bool SPLIT>
__global__ __launch_bounds__(256, 1) void k_small(Call c, Steps steps, Few few, int32_t first) {
  extern __shared__ half memory[];
  constexpr int kBlocks = N / 64, kParts = SPLIT ? 2 : 1, kMostTiles = kSmallLength / N;
  constexpr int kXs = N * kSmallLength, kAs = N * N;
  half *const x[2] = {memory, memory + kXs};  // hi, lo (lo: only at both ends, unless SPLIT)
  half *const gram[2] = {memory + kParts * kXs, memory + kParts * kXs + kAs};
  half *const poly[2] = {gram[0] + kParts * kAs, gram[0] + kParts * kAs + kAs};
  __shared__ double shared[4];
  const Matrix &m = c.matrices[first + blockIdx.x];
  if (m.tiny) return;
  const Addresses at = few.at[blockIdx.x];
  const int n = m.n, k = m.k, tiles = (k + N - 1) / N, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wa = wave & 1, wb = wave >> 1;
  const int low = lane & 31, high = lane >> 5;
  // where column `col`, of a multiple of 4, of row `row` is
  auto place = [&](int row, int col) {
    return ((col >> 5) * N + row) * kDeep + ((((col >> 3) & 3) ^ ((row >> 2) & 3)) * 8) + (col & 7);
  };

  const int rows = m.tall ? k : n, cols = m.tall ? n : k;
  // Twice over U, 8 neighbours of a row at a time.  Code that runs once comes slowly from memory, so that
  // loops here are kept short rather than unrolled.
  const int pieces = (cols + 7) / 8, units = rows * pieces;
  double squares = 0.;
  float inverse = 0.f;  // times 2^power: of subnormal matrices it is no fp32 number
  int power = 0;
  double size = 0.;     // of X_0
  // some units at a time, so that their loads are on their way together
  auto look = [&](auto *in, auto whole, int pass) {
    constexpr int kSome = decltype(whole)::value ? 4 : 1;
    const bool wide = whole_rows(in, m.ld), wide_m = whole_rows(at.momentum, m.ld);
#pragma unroll 1
    for (int q0 = tid; q0 < units; q0 += 256 * kSome) {
      float u[kSome][8], h[kSome][8];
#pragma unroll
      for (int i = 0; i < kSome; ++i) {
        const int q = min(q0 + i * 256, units - 1), row = q / pieces, col = (q - row * pieces) * 8;
        const int64_t from = row * m.ld + col;
        if constexpr (decltype(whole)::value) {
          load8(in + from, u[i]);
          if (c.momentum) load8(static_cast<const float *>(at.momentum) + from, h[i]);
        } else {
          row8(in + from, cols - col, wide, u[i]);
          if (c.momentum) row8(static_cast<const float *>(at.momentum) + from, cols - col, wide_m, h[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < kSome; ++i) {
        const int q = q0 + i * 256, row = q / pieces, col = (q - row * pieces) * 8;
        if (q >= units) continue;
        if (c.momentum) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if (pass == 0) {
              h[i][e] = fmaf(c.mu, h[i][e], u[i][e]);
              if (decltype(whole)::value || col + e < cols) at.momentum[row * m.ld + col + e] = h[i][e];
            }
            u[i][e] = c.nesterov ? fmaf(c.mu, h[i][e], u[i][e]) : h[i][e];
          }
        }
        if (pass == 0) {
#pragma unroll
          for (int e = 0; e < 8; ++e) squares = fma(static_cast<double>(u[i][e]), static_cast<double>(u[i][e]), squares);
          continue;
        }
        half8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) u[i][e] = ldexpf(u[i][e], power) * inverse;
        split8(u[i], hi, lo);
        if (!m.tall) {  // past the row's end: zeros, into the padding
          *reinterpret_cast<half8 *>(x[0] + place(row, col)) = hi;
          *reinterpret_cast<half8 *>(x[1] + place(row, col)) = lo;
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int to = place(min(col + e, N - 1), row & ~3) + (row & 3);
            if (col + e < cols) x[0][to] = hi[e], x[1][to] = lo[e];
          }
        }
      }
    }
  };
  auto both = [&](auto *in, auto whole) {
    look(in, whole, 0);
    for (int q = tid; q < N * tiles * N / 8; q += 256) {  // zeros where the padding is
      const half8 none = {};
      *reinterpret_cast<half8 *>(x[0] + q * 8) = none;
      *reinterpret_cast<half8 *>(x[1] + q * 8) = none;
    }
    squares = block_sum(squares, shared);
    const double by = inverse_norm(squares, c.eps);
    size = sqrt(squares) * by;
    power = by > 0. ? ilogb(by) : 0;
    inverse = static_cast<float>(ldexp(by, -power));
    power += kPowerX + lift(size);
    look(in, whole, 1);
  };
  auto by_rows = [&](auto *in) {
    if (cols % 8 == 0 && whole_rows(in, m.ld) && (!c.momentum || whole_rows(at.momentum, m.ld)))
      both(in, std::true_type{});
    else
      both(in, std::false_type{});
  };
  if (c.in_bf16)
    by_rows(static_cast<const uint16_t *>(at.in));
  else
    by_rows(static_cast<const float *>(at.in));
  __syncthreads();

  // this wave's quarter of tile t: rows wb * N / 2 + y * 32 + low, columns t * N + wa * N / 2 + x * 32 + g * 8 + high * 4
  half4 lower[kMostTiles][kBlocks][kBlocks][4];
  auto mine = [&](int t, int xb, int yb, int g) {
    return place(wb * (N / 2) + yb * 32 + low, t * N + wa * (N / 2) + xb * 32 + g * 8 + high * 4);
  };
  if constexpr (!SPLIT) {
#pragma unroll
    for (int t = 0; t < kMostTiles; ++t)
#pragma unroll
      for (int q = 0; q < kBlocks * kBlocks * 4; ++q)
        if (t < tiles)
          lower[t][q / (4 * kBlocks)][q / 4 % kBlocks][q % 4] =
              *reinterpret_cast<const half4 *>(x[1] + mine(t, q / (4 * kBlocks), q / 4 % kBlocks, q % 4));
    __syncthreads();  // what lay there makes room for A and P
  }

  f32x16 acc[kBlocks][kBlocks];
  auto along = [&](const half *from, int row0, int panel, int kk) {
    const int r = row0 + low;
    return *reinterpret_cast<const half8 *>(from + (panel * N + r) * kDeep + (((kk * 2 + high) ^ ((r >> 2) & 3)) * 8));
  };
  auto down = [&](const half *from, int panel_row, int panel, int kk) {  // columns of `panel`, rows panel_row * 32 and on
    typedef __attribute__((address_space(3))) short4v *shared4;
    const int r = panel_row * 32 + kk * 16 + high * 8 + ((lane >> 2) & 3), col = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
    const short4v v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared4)(from + place(r, panel * 32 + col)));
    const short4v v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared4)(from + place(r + 4, panel * 32 + col)));
    return __builtin_bit_cast(half8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  // acc += a b over N of the summed side, of pairs the products of `pass`: hi lo, lo hi, hi hi
  auto clear = [&] {
#pragma unroll
    for (int xb = 0; xb < kBlocks; ++xb)
#pragma unroll
      for (int yb = 0; yb < kBlocks; ++yb)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[xb][yb][r] = 0.f;
  };
  auto product = [&](int pass, auto &&a, auto &&b) {
#pragma unroll
    for (int s = 0; s < N / kDeep; ++s)
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        half8 fa[kBlocks], fb[kBlocks];
#pragma unroll
        for (int q = 0; q < kBlocks; ++q) {
          fa[q] = a(pass == 1, q, s, kk);
          fb[q] = b(pass == 0, q, s, kk);
        }
#pragma unroll
        for (int xb = 0; xb < kBlocks; ++xb)
#pragma unroll
          for (int yb = 0; yb < kBlocks; ++yb)
            acc[xb][yb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[xb], fb[yb], acc[xb][yb], 0, 0, 0);
      }
  };
  constexpr int kFirstPass = SPLIT ? 0 : 2;
  auto each_four = [&](auto &&f) {
#pragma unroll
    for (int xb = 0; xb < kBlocks; ++xb)
#pragma unroll
      for (int yb = 0; yb < kBlocks; ++yb)
#pragma unroll
        for (int g = 0; g < 4; ++g) f(xb, yb, g);
  };
  auto keep = [&](half *const to[2], int pos, const float *v) {
    half4 hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      half h, l;
      split_half(v[e], h, l);
      hi[e] = h;
      lo[e] = l;
    }
    *reinterpret_cast<half4 *>(to[0] + pos) = hi;
    if (SPLIT) *reinterpret_cast<half4 *>(to[1] + pos) = lo;
    return lo;
  };

  for (int s = 0; s < steps.count; ++s) {
    const float sa = steps.a_power[s], sp = steps.p_power[s], a0 = steps.abc[s][0];
    // of pairs of halves always: with a on P's diagonal, results of matrices of deficient rank were 1.3 times as
    // far off (64 x 40, rank 5: 1.6e-5 to 2.1e-5)
    const bool carry = SPLIT || steps.carry[s];
    // for the powers of two that X is held times, here and after the step
    const double after = grown(size, steps.abc[s]);
    float lowered = 1.f, on = 1.f;
    if (size < 0.5 || after < 0.5) {  // passed over as a rule: 41.8 us for 42.2 (128 x 96)
      lowered = ldexpf(1.f, -2 * lift(size));
      on = ldexpf(1.f, lift(after) - lift(size));
    }
    size = after;
    clear();
#pragma unroll
    for (int pass = kFirstPass; pass < 3; ++pass)
      for (int t = 0; t < tiles; ++t)
        product(pass,
                [&](bool lo, int q, int d, int kk) { return along(x[lo], wa * (N / 2) + q * 32, t * (N / kDeep) + d, kk); },
                [&](bool lo, int q, int d, int kk) { return along(x[lo], wb * (N / 2) + q * 32, t * (N / kDeep) + d, kk); });
    each_four([&](int xb, int yb, int g) {
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = acc[xb][yb][4 * g + e] * (sa / (kScaleX * kScaleX) * lowered);
      keep(gram, mine(0, xb, yb, g), v);
    });
    __syncthreads();
    clear();
#pragma unroll
    for (int pass = kFirstPass; pass < 3; ++pass)
      product(pass, [&](bool lo, int q, int d, int kk) { return along(gram[lo], wa * (N / 2) + q * 32, d, kk); },
              [&](bool lo, int q, int d, int kk) { return along(gram[lo], wb * (N / 2) + q * 32, d, kk); });
    each_four([&](int xb, int yb, int g) {
      const int pos = mine(0, xb, yb, g);
      const half4 h = *reinterpret_cast<const half4 *>(gram[0] + pos);
      half4 l;
      if (SPLIT) l = *reinterpret_cast<const half4 *>(gram[1] + pos);
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float value = static_cast<float>(h[e]) + (SPLIT ? static_cast<float>(l[e]) : 0.f);
        v[e] = fmaf(steps.abc[s][1] * (sp / sa), value, acc[xb][yb][4 * g + e] * (steps.abc[s][2] * (sp / (sa * sa))));
      }
      if (!carry && wa == wb && xb == yb) {  // a block of the diagonal
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (low == g * 8 + high * 4 + e) v[e] += a0 * sp;
      }
      keep(poly, pos, v);
    });
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kMostTiles; ++t) {
      if (t >= tiles) break;
      clear();
#pragma unroll
      for (int pass = kFirstPass; pass < 3; ++pass)
        product(pass, [&](bool lo, int q, int d, int kk) { return down(x[lo], d, (t * N + wa * (N / 2)) / 32 + q, kk); },
                [&](bool lo, int q, int d, int kk) { return along(poly[lo], wb * (N / 2) + q * 32, d, kk); });
      __syncthreads();  // everybody has read this tile of X
      each_four([&](int xb, int yb, int g) {
        const int pos = mine(t, xb, yb, g);
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = acc[xb][yb][4 * g + e] * (on / sp);
        if (carry) {
          const half4 h = *reinterpret_cast<const half4 *>(x[0] + pos);
          const half4 l = SPLIT ? *reinterpret_cast<const half4 *>(x[1] + pos) : lower[t][xb][yb][g];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = fmaf(a0 * on, static_cast<float>(h[e]) + static_cast<float>(l[e]), v[e]);
        }
        lower[t][xb][yb][g] = keep(x, pos, v);
      });
    }
    __syncthreads();
  }
  // The result, hi + lo, in the caller's rows.
  float lower_all = 1.f;
  if (size < 0.5) lower_all = ldexpf(1.f, -lift(size));
  if constexpr (!SPLIT) {
#pragma unroll
    for (int t = 0; t < kMostTiles; ++t)
      if (t < tiles) each_four([&](int xb, int yb, int g) { *reinterpret_cast<half4 *>(x[1] + mine(t, xb, yb, g)) = lower[t][xb][yb][g]; });
    __syncthreads();
  }
#pragma unroll 1
  for (int q = tid; q < units; q += 256) {
    const int row = q / pieces, col = (q - row * pieces) * 8;
    float v[8];
    if (!m.tall) {
      const half8 hi = *reinterpret_cast<const half8 *>(x[0] + place(row, col)),
                  lo = *reinterpret_cast<const half8 *>(x[1] + place(row, col));
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(hi[e]) + static_cast<float>(lo[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int from = place(min(col + e, cols - 1), row & ~3) + (row & 3);
        v[e] = static_cast<float>(x[0][from]) + static_cast<float>(x[1][from]);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= lower_all;
    write_out(c, at, m.ld, row, rows, col, cols, v, m.scale * (1.f / kScaleX));
  }
}

template <int N, bool SPLIT>
constexpr size_t small_bytes() {  // at both ends X's lower halves lie where A and P do in between
  const size_t parts = SPLIT ? 2 : 1;
  return sizeof(half) * (parts * N * kSmallLength + (SPLIT || 2 * N > kSmallLength ? 2 * parts * N * N : N * kSmallLength));
}
static_assert(small_bytes<128, false>() <= 160 * 1024 - 64 && small_bytes<64, true>() <= 160 * 1024 - 64, "shared memory");
static_assert(2 * kSmallSide * kSmallSide >= kSmallSide * kSmallLength || small_bytes<64, false>() >= 4 * 64 * kSmallLength, "X's lower halves fit where A and P lie");

}  // namespace

hipError_t launch_tiny(const Call &c, const Steps &steps, const int32_t *list, int32_t count, hipStream_t s) {
  k_tiny<<<count, kTinyThreads, 0, s>>>(c, steps, list);
  return hipGetLastError();
}

hipError_t prepare_small() {
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_small<kSmallSide, false>),
                                     hipFuncAttributeMaxDynamicSharedMemorySize, small_bytes<kSmallSide, false>());
  if (e == hipSuccess)
    e = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_small<kSmallSideSplit, true>),
                            hipFuncAttributeMaxDynamicSharedMemorySize, small_bytes<kSmallSideSplit, true>());
  if (e == hipSuccess)
    e = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_small<kSmallSideSplit, false>),
                            hipFuncAttributeMaxDynamicSharedMemorySize, small_bytes<kSmallSideSplit, false>());
  return e;
}

hipError_t launch_small(const Call &c, const Steps &steps, const Few &few, int32_t first, int32_t count, int32_t side,
                        bool split, hipStream_t s) {
  if (split)
    k_small<kSmallSideSplit, true><<<count, 256, small_bytes<kSmallSideSplit, true>(), s>>>(c, steps, few, first);
  else if (side <= kSmallSideSplit)
    k_small<kSmallSideSplit, false><<<count, 256, small_bytes<kSmallSideSplit, false>(), s>>>(c, steps, few, first);
  else
    k_small<kSmallSide, false><<<count, 256, small_bytes<kSmallSide, false>(), s>>>(c, steps, few, first);
  return hipGetLastError();
}

hipError_t launch_addresses(const Call &c, const Few &few, int32_t first, int32_t count, hipStream_t s) {
  k_addresses<<<1, 64, 0, s>>>(c.addresses, few, first, count);
  return hipGetLastError();
}

hipError_t launch_sums(const Call &c, const Item *items, int32_t count, hipStream_t s) {
  k_sums<<<count, 256, 0, s>>>(c, items);
  return hipGetLastError();
}

hipError_t launch_load(const Call &c, const Item *items, int32_t count, hipStream_t s) {
  k_load<<<count, 256, 0, s>>>(c, items);
  return hipGetLastError();
}

namespace {

// The kernel for a kind of tiles: rings as deep as the workgroups that share a CU leave room for.  (Of small
// tiles in lists too short for that, rings of 9 stages took 1.01 to 1.06 of the time of 3: their longer code,
// which comes from memory once a launch, costs what they hide.)
template <bool UPDATE, typename F>
hipError_t with_products(int kind, bool split, F &&f) {
  auto sized = [&](auto a, auto b, auto stages) {
    constexpr int A = a(), B = b(), S = stages();
    constexpr size_t bytes = sizeof(half) * S * (A + B) * kDeep;
    return split ? f(k_products<A, B, S, UPDATE, true>, bytes) : f(k_products<A, B, S, UPDATE, false>, bytes);
  };
  std::integral_constant<int, 128> small;
  std::integral_constant<int, 256> large;
  std::integral_constant<int, 3> three;
  if (kind == kLarge) return sized(large, large, std::integral_constant<int, 4>{});
  if constexpr (UPDATE)
    if (kind == kWide) return sized(large, small, three);
  return sized(small, small, three);
}

}  // namespace

// More shared memory than a kernel may have unasked.
hipError_t prepare_products(bool split) {
  auto allow = [](auto *k, size_t bytes) {
    return hipFuncSetAttribute(reinterpret_cast<const void *>(k), hipFuncAttributeMaxDynamicSharedMemorySize,
                               static_cast<int>(bytes));
  };
  for (int kind : {kSmall, kLarge, kWide}) {
    hipError_t e = with_products<false>(kind, split, allow);
    if (e == hipSuccess) e = with_products<true>(kind, split, allow);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_symmetric(const Call &c, int kind, const Symmetric &p, const Tile *tiles, int32_t count,
                            bool split, hipStream_t s) {
  return with_products<false>(kind, split, [&](auto *k, size_t bytes) {
    k<<<count, 256, bytes, s>>>(c, p, tiles);
    return hipGetLastError();
  });
}

hipError_t launch_update(const Call &c, int kind, const Update &p, const Tile *tiles, int32_t count, bool split,
                         hipStream_t s) {
  return with_products<true>(kind, split, [&](auto *k, size_t bytes) {
    k<<<count, 256, bytes, s>>>(c, p, tiles);
    return hipGetLastError();
  });
}

}  // namespace orth
}  // namespace slowmo
