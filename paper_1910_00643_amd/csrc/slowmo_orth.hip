// Kernels of the orthogonalising call (include/slowmo_operators.h has the formulas).
//
// Matrix products bound it: 5 steps of X X^T (n n k, half of it by symmetry), A A (n n n, half) and
// P X (2 n n k).  They run on the matrix cores in halves with fp32 sums.  Of the two 16-bit types a
// half has 11 bits and bf16 has 8; X, A and P lie in a range known beforehand, so bf16's exponents buy
// nothing.  A step multiplies small singular values by a = 3.4, so a rounding of X early on comes out
// up to 3.4^5 times as large; X therefore keeps the next 11 bits too (x = hi + lo), which enter where X
// enters linearly, in a X, while the products take hi alone.  Against 64 bits, 512 x 2048 and 1024 x
// 1024 with flat, decaying and deficient spectra: 0.3e-3 to 1.7e-3 (hi alone 1.2e-3 to 8.6e-3, bf16
// 0.9e-2 to 7e-2).  For fp32 results all factors are such pairs and a product is three: hi hi + hi lo +
// lo hi, 22 bits.
#include "slowmo_orth.h"

#include <type_traits>

namespace slowmo {
namespace orth {
namespace {

typedef _Float16 half;
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
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

// The sum of squares of U over a patch, in 64 bits: squares of fp32 values neither overflow nor
// vanish there.  Updates the momentum on the way.
__global__ __launch_bounds__(256) void k_squares(Call c, const Item *items) {
  const Item it = items[blockIdx.x];
  const Matrix &m = c.matrices[it.matrix];
  const Addresses at = c.addresses[it.matrix];
  const int rows = m.tall ? m.k : m.n, cols = m.tall ? m.n : m.k;
  const int col = it.j * kPatch + (threadIdx.x & 63);
  double sum = 0.;
  for (int r = threadIdx.x >> 6; r < kPatch; r += 4) {
    const int row = it.i * kPatch + r;
    if (row >= rows || col >= cols) continue;
    const int64_t e = row * m.ld + col;
    float u = load_input(c, at, e);
    if (c.momentum) {
      const float h = fmaf(c.mu, at.momentum[e], u);
      at.momentum[e] = h;
      u = c.nesterov ? fmaf(c.mu, h, u) : h;
    }
    sum = fma(static_cast<double>(u), static_cast<double>(u), sum);
  }
  __shared__ double sums[4];
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) c.squares[blockIdx.x] = sums[0] + sums[1] + sums[2] + sums[3];
}

__global__ __launch_bounds__(256) void k_norms(Call c) {
  const Matrix &m = c.matrices[blockIdx.x];
  double sum = 0.;
  for (int i = threadIdx.x; i < m.patches; i += 256) sum += c.squares[m.first_patch + i];
  __shared__ double sums[4];
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x) return;
  const double norm = sqrt(sums[0] + sums[1] + sums[2] + sums[3]) + static_cast<double>(c.eps);
  // a matrix of zeros (and eps 0): zeros; an infinity or NaN anywhere: NaN everywhere
  c.inverse[blockIdx.x] = norm == 0. ? 0.f : norm < 1.7e308 ? static_cast<float>(1. / norm) : __builtin_nanf("");
}

// X_0 (n x k, turned if the caller's matrix is tall) as halves hi and lo, with zeros in the padding (which
// an earlier call's NaN may have reached).
__global__ __launch_bounds__(256) void k_load(Call c, const Item *items) {
  const Item it = items[blockIdx.x];
  const Matrix &m = c.matrices[it.matrix];
  const Addresses at = c.addresses[it.matrix];
  const int rows = m.tall ? m.k : m.n, cols = m.tall ? m.n : m.k;
  half *x = c.arena + m.x[0], *x_lo = c.arena + m.x_lo[0];
  const float inverse = c.inverse[it.matrix];
  __shared__ float turn[kPatch][kPatch + 1];
  const int lane = threadIdx.x & 63;
  for (int r = threadIdx.x >> 6; r < kPatch; r += 4) {
    const int row = it.i * kPatch + r, col = it.j * kPatch + lane;
    float u = 0.f;
    if (row < rows && col < cols) {
      const int64_t e = row * m.ld + col;
      if (c.momentum) {
        const float h = at.momentum[e];
        u = c.nesterov ? fmaf(c.mu, h, load_input(c, at, e)) : h;
      } else {
        u = load_input(c, at, e);
      }
      u = u * inverse * kScaleX;
    }
    if (m.tall) {
      turn[r][lane] = u;
    } else {
      const int64_t to = static_cast<int64_t>(row) * m.kp + col;
      split_half(u, x[to], x_lo[to]);
    }
  }
  if (!m.tall) return;
  __syncthreads();
  for (int r = threadIdx.x >> 6; r < kPatch; r += 4) {
    const int64_t to = static_cast<int64_t>(it.j * kPatch + r) * m.kp + it.i * kPatch + lane;
    split_half(turn[lane][r], x[to], x_lo[to]);
  }
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
// Tiles of T x T by 4 waves of T/2 x T/2.  Steps of 32 of the summed side go from memory straight to a
// ring of kRing stages in shared memory (16 bytes a lane), kRing - 1 steps ahead of their use: memory's
// latency is 0.7 us and a step's products take 0.25 us (T = 256).  A wave reads the next 16's factors into
// registers before it issues the products of this 16, across the barrier of a step too, so that with
// one wave per SIMD (T = 256: 256 accumulators a lane) the matrix cores go on.
//
// Rows of 32 halves (both factors contiguous along the summed side: X X^T, A A, and P of P X) are four
// pieces of 16 bytes; piece p of row r lies at p xor (r / 4 mod 4), so that 16 lanes that read the same
// piece of neighbouring rows meet all 64 banks once.  X of P X lies with the summed side across: its
// rows are read turned (4 rows x 16 columns per 16 lanes), with piece p of row r at p xor 4 (r mod 4).
// Everything is padded to whole tiles; nothing is checked in the loop.

constexpr int kDeep = 32, kRing = 4;

__device__ __forceinline__ void to_shared(u32 shared, u32 offset, const half *base) {
  // m0 is written and read within this block; the wait covers its hazard and that of a base that a
  // vector instruction has just brought to scalar registers.  No vector register is written.
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(shared), "v"(offset),
               "s"(base)
               : "memory");
}
// All but the N newest loads of this wave have arrived, its reads of shared memory are done, and so it is
// for every wave of the workgroup.
template <int N>
__device__ __forceinline__ void arrive() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));

template <int T, int PHASE, bool SPLIT>
__global__ __launch_bounds__(256, T == 256 ? 1 : 2) void k_products(Call c, Step st, const Item *items) {
  extern __shared__ half ring[];
  constexpr int kBlocks = T / 64;            // blocks of 32 x 32 along a side of a wave's share
  constexpr int kShare = T * kDeep;          // halves of one factor in a stage
  constexpr int kLoads = kShare * 2 / 1024 / 4;  // loads of a wave per factor and stage
  constexpr int kWide = T / 2;               // side of a wave's share
  const Item it = items[blockIdx.x];
  const Matrix &m = c.matrices[it.matrix];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wa = wave & 1, wb = wave >> 1;
  const int low = lane & 31, high = lane >> 5;

  // factor a: columns of the tile (j), factor b: rows (i).  The accumulators' four neighbours run along a.
  const int depth = PHASE == kGram ? m.kp : m.np, steps = depth / kDeep;
  const int64_t a_hi = PHASE == kPolynomial ? m.a : m.x[st.from];
  const int64_t a_lo = PHASE == kPolynomial ? m.a_lo : m.x_lo[st.from];
  const int64_t b_hi = PHASE == kUpdate ? m.p : a_hi, b_lo = PHASE == kUpdate ? m.p_lo : a_lo;
  const int64_t a_at = PHASE == kUpdate ? static_cast<int64_t>(it.j) * T : static_cast<int64_t>(it.j) * T * depth;
  const int64_t b_at = static_cast<int64_t>(it.i) * T * depth;
  const int64_t a_step = PHASE == kUpdate ? static_cast<int64_t>(kDeep) * m.kp : kDeep;
  const int total = SPLIT ? 3 * steps : steps;

  u32 a_off[kLoads], b_off[kLoads];          // bytes
#pragma unroll
  for (int q = 0; q < kLoads; ++q) {
    const int load = wave * kLoads + q;
    const int row = load * 16 + (lane >> 2), piece = (lane & 3) ^ ((row >> 2) & 3);
    b_off[q] = (row * depth + piece * 8) * 2;
    if constexpr (PHASE == kUpdate) {
      constexpr int kAcross = T / 8;         // pieces of a row
      const int r = load * (64 / kAcross) + lane / kAcross, p = (lane % kAcross) ^ (4 * (r & 3));
      a_off[q] = (r * m.kp + p * 8) * 2;
    } else {
      a_off[q] = b_off[q];
    }
  }
  const u32 shared0 = static_cast<u32>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) half *)ring));

  auto fetch = [&](int t) {
    // split: the small products first (hi lo, lo hi), while their sums are small, then hi hi
    const int seg = SPLIT ? (t >= 2 * steps ? 2 : t >= steps ? 1 : 0) : 2;
    const int at = SPLIT ? t - seg * steps : t;
    const half *a = c.arena + (seg == 1 ? a_lo : a_hi) + a_at + at * a_step;
    const half *b = c.arena + (seg == 0 ? b_lo : b_hi) + b_at + static_cast<int64_t>(at) * kDeep;
    const u32 slot = shared0 + (t % kRing) * (2 * kShare * 2) + wave * kLoads * 1024;
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      to_shared(slot + q * 1024, a_off[q], a);
      to_shared(slot + kShare * 2 + q * 1024, b_off[q], b);
    }
  };

  half8 fa[2][kBlocks], fb[2][kBlocks];
  auto read = [&](int t, int kk, half8 *a, half8 *b) {
    const half *sa = ring + (t % kRing) * 2 * kShare, *sb = sa + kShare;
#pragma unroll
    for (int x = 0; x < kBlocks; ++x) {
      const int rb = wb * kWide + x * 32 + low;
      b[x] = *reinterpret_cast<const half8 *>(sb + rb * kDeep + (((kk * 2 + high) ^ ((rb >> 2) & 3)) * 8));
      if constexpr (PHASE == kUpdate) {
        const int r = kk * 16 + high * 8 + ((lane >> 2) & 3);
        const int col = wa * kWide + x * 32 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
        const int piece = (col >> 3) ^ (4 * (r & 3));
        const half *from = sa + r * T + piece * 8 + (col & 7);
        typedef __attribute__((address_space(3))) short4v *shared4;
        const short4v lo4 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared4)(from));
        const short4v hi4 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared4)(from + 4 * T));
        a[x] = __builtin_bit_cast(half8, __builtin_shufflevector(lo4, hi4, 0, 1, 2, 3, 4, 5, 6, 7));
      } else {
        const int ra = wa * kWide + x * 32 + low;
        a[x] = *reinterpret_cast<const half8 *>(sa + ra * kDeep + (((kk * 2 + high) ^ ((ra >> 2) & 3)) * 8));
      }
    }
  };

  f32x16 acc[kBlocks][kBlocks];
#pragma unroll
  for (int x = 0; x < kBlocks; ++x)
#pragma unroll
    for (int y = 0; y < kBlocks; ++y)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[x][y][r] = 0.f;
  auto multiply = [&](const half8 *a, const half8 *b) {
#pragma unroll
    for (int x = 0; x < kBlocks; ++x)
#pragma unroll
      for (int y = 0; y < kBlocks; ++y)
        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[x], b[y], acc[x][y], 0, 0, 0);
  };

  constexpr int kPending = 2 * kLoads * (kRing - 2);
  for (int t = 0; t < kRing && t < total; ++t) fetch(t);
  if (total >= kRing)
    arrive<kPending + 2 * kLoads>();
  else
    arrive<0>();
  read(0, 0, fa[0], fb[0]);
  for (int t = 0; t < total; ++t) {
    read(t, 1, fa[1], fb[1]);
    multiply(fa[0], fb[0]);
    if (t + 1 < total) {
      if (t + kRing <= total)
        arrive<kPending>();
      else
        arrive<0>();
      if (t + kRing < total) fetch(t + kRing);  // where step t was: everybody has read it
      read(t + 1, 0, fa[0], fb[0]);
    }
    multiply(fa[1], fb[1]);
  }
  __syncthreads();

  // The results pass through shared memory, 32 rows of a wave's share at a time, to leave in whole rows.
  constexpr int kPitch = kWide + 4, kLanes = kWide / 8, kRows = 64 / kLanes;
  float *stage = reinterpret_cast<float *>(ring) + wave * 32 * kPitch;
  const int sub = lane / kLanes, c8 = (lane % kLanes) * 8;
  // rows y of factor b, along a
  auto direct = [&](int y) {
#pragma unroll
    for (int x = 0; x < kBlocks; ++x)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4 *>(stage + low * kPitch + x * 32 + g * 8 + high * 4) =
            f32x4{acc[x][y][4 * g], acc[x][y][4 * g + 1], acc[x][y][4 * g + 2], acc[x][y][4 * g + 3]};
  };
  // rows x of factor a, along b
  auto turned = [&](int x) {
#pragma unroll
    for (int y = 0; y < kBlocks; ++y)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        stage[((r >> 2) * 8 + high * 4 + (r & 3)) * kPitch + y * 32 + low] = acc[x][y][r];
  };
  auto take = [&](int r, float *v) {
    const f32x4 p = *reinterpret_cast<const f32x4 *>(stage + r * kPitch + c8),
                q = *reinterpret_cast<const f32x4 *>(stage + r * kPitch + c8 + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = p[e], v[4 + e] = q[e];
  };
  const int ai = it.j * T + wa * kWide, bi = it.i * T + wb * kWide;  // first place along each factor

  if constexpr (PHASE == kUpdate) {
    const Addresses at = c.addresses[it.matrix];
    if (st.last && m.tall) {  // the caller's matrix is k x n: rows of factor a
      const float scale = m.scale / (kScaleX * kScaleP);
#pragma unroll
      for (int x = 0; x < kBlocks; ++x) {
        turned(x);
#pragma unroll
        for (int r = 0; r < 32; r += kRows) {
          float v[8];
          take(r + sub, v);
          write_out(c, at, m.ld, ai + x * 32 + r + sub, m.k, bi + c8, m.n, v, scale);
        }
      }
      return;
    }
#pragma unroll
    for (int y = 0; y < kBlocks; ++y) {
      direct(y);
#pragma unroll
      for (int r = 0; r < 32; r += kRows) {
        const int row = bi + y * 32 + r + sub;
        float v[8];
        take(r + sub, v);
        if (st.last) {
          write_out(c, at, m.ld, row, m.n, ai + c8, m.k, v, m.scale / (kScaleX * kScaleP));
          continue;
        }
        const int64_t pos = static_cast<int64_t>(row) * m.kp + ai + c8;
        half8 nh, nl;
        if (st.carry) {
          const half8 h = *reinterpret_cast<const half8 *>(c.arena + m.x[st.from] + pos);
          const half8 l = *reinterpret_cast<const half8 *>(c.arena + m.x_lo[0] + pos);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            v[e] = fmaf(st.a, static_cast<float>(h[e]) + static_cast<float>(l[e]), v[e] * (1.f / kScaleP));
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] *= 1.f / kScaleP;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          half h, l;
          split_half(v[e], h, l);
          nh[e] = h;
          nl[e] = l;
        }
        *reinterpret_cast<half8 *>(c.arena + m.x[1 - st.from] + pos) = nh;
        if (SPLIT)
          *reinterpret_cast<half8 *>(c.arena + m.x_lo[1 - st.from] + pos) = nl;
        else if (st.carry_next)
          *reinterpret_cast<half8 *>(c.arena + m.x_lo[0] + pos) = nl;
      }
    }
  } else {
    half *to_hi = c.arena + (PHASE == kGram ? m.a : m.p), *to_lo = c.arena + (PHASE == kGram ? m.a_lo : m.p_lo);
    auto rows = [&](int row0, int col0) {  // 32 staged rows of the symmetric result
#pragma unroll
      for (int r = 0; r < 32; r += kRows) {
        const int row = row0 + r + sub, col = col0 + c8;
        const int64_t pos = static_cast<int64_t>(row) * m.np + col;
        float v[8];
        take(r + sub, v);
        if constexpr (PHASE == kGram) {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] *= kScaleA / (kScaleX * kScaleX);
        } else {
          const half8 h = *reinterpret_cast<const half8 *>(c.arena + m.a + pos);
          half8 l;
          if (SPLIT) l = *reinterpret_cast<const half8 *>(c.arena + m.a_lo + pos);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float x = static_cast<float>(h[e]) + (SPLIT ? static_cast<float>(l[e]) : 0.f);
            v[e] = fmaf(st.b * (kScaleP / kScaleA), x, st.c * (kScaleP / (kScaleA * kScaleA)) * v[e]);
            if (!st.carry && row == col + e) v[e] += st.a * kScaleP;
          }
        }
        half8 nh, nl;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          half h, l;
          split_half(v[e], h, l);
          nh[e] = h;
          nl[e] = l;
        }
        *reinterpret_cast<half8 *>(to_hi + pos) = nh;
        if (SPLIT) *reinterpret_cast<half8 *>(to_lo + pos) = nl;
      }
    };
#pragma unroll
    for (int y = 0; y < kBlocks; ++y) {
      direct(y);
      rows(bi + y * 32, ai);
    }
    if (it.i != it.j) {
#pragma unroll
      for (int x = 0; x < kBlocks; ++x) {
        turned(x);
        rows(ai + x * 32, bi);
      }
    }
  }
}

// A tiny matrix from its load to its store: one workgroup, all steps, X, A and P in shared memory.
// There is so little work that it is done in 64 bits: with few directions (a rank of one or two) the
// largest singular values of X_0 are near 1, the early steps' roundings enter in full, and fp32 sums
// alone would cost a fp32 result five of its bits.
__global__ __launch_bounds__(kTinyThreads) void k_tiny(Call c, Steps steps, const int32_t *list) {
  __shared__ double x[kTinyElements], gram[kTinySide * kTinySide], poly[kTinySide * kTinySide];
  __shared__ double sums[kTinyThreads / 64];
  const int32_t at_matrix = list[blockIdx.x];
  const Matrix &m = c.matrices[at_matrix];
  const Addresses at = c.addresses[at_matrix];
  const int n = m.n, k = m.k, count = n * k, tid = threadIdx.x, lane = tid & 63;
  double sum = 0.;
  for (int e = tid; e < count; e += kTinyThreads) {  // in the caller's order; x is n x k
    const int cols = m.tall ? n : k, row = e / cols, col = e - row * cols;
    const int64_t from = row * m.ld + col;
    float u = load_input(c, at, from);
    if (c.momentum) {
      const float h = fmaf(c.mu, at.momentum[from], u);
      at.momentum[from] = h;
      u = c.nesterov ? fmaf(c.mu, h, u) : h;
    }
    const double v = u;
    x[m.tall ? col * k + row : e] = v;
    sum = fma(v, v, sum);
  }
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) sums[tid >> 6] = sum;
  __syncthreads();
  sum = 0.;
  for (int w = 0; w < kTinyThreads / 64; ++w) sum += sums[w];
  const double norm = sqrt(sum) + static_cast<double>(c.eps);
  const double inverse = norm == 0. ? 0. : norm < 1.7e308 ? 1. / norm : __builtin_nan("");
  for (int e = tid; e < count; e += kTinyThreads) x[e] *= inverse;
  __syncthreads();
  // a group of lanes per element of A: few elements have long rows, many have short ones
  const int log2 = n <= 4 ? 6 : n <= 12 ? 4 : 3, lanes = 1 << log2;
  for (int t = 0; t < steps.count; ++t) {
    for (int e0 = (tid >> log2); e0 < n * n; e0 += kTinyThreads >> log2) {
      const int i = e0 / n, j = e0 - i * n;
      double dot = 0.;
      for (int q = lane & (lanes - 1); q < k; q += lanes) dot = fma(x[i * k + q], x[j * k + q], dot);
      for (int o = lanes >> 1; o; o >>= 1) dot += __shfl_xor(dot, o);
      if ((lane & (lanes - 1)) == 0) gram[e0] = dot;
    }
    __syncthreads();
    const float *abc = steps.abc[t];
    for (int e = tid; e < n * n; e += kTinyThreads) {
      const int i = e / n, j = e - i * n;
      double dot = 0.;
      for (int q = 0; q < n; ++q) dot = fma(gram[i * n + q], gram[q * n + j], dot);
      poly[e] = abc[1] * gram[e] + abc[2] * dot + (i == j ? static_cast<double>(abc[0]) : 0.);
    }
    __syncthreads();
    for (int col = tid; col < k; col += kTinyThreads) {
      double v[kTinySide];
#pragma unroll
      for (int q = 0; q < kTinySide; ++q) v[q] = q < n ? x[q * k + col] : 0.;
      for (int i = 0; i < n; ++i) {
        double dot = 0.;
#pragma unroll
        for (int q = 0; q < kTinySide; ++q)
          if (q < n) dot = fma(poly[i * n + q], v[q], dot);
        x[i * k + col] = dot;
      }
    }
    __syncthreads();
  }
  for (int e = tid; e < count; e += kTinyThreads) {
    const int cols = m.tall ? n : k, row = e / cols, col = e - row * cols;
    const float o = static_cast<float>(x[m.tall ? col * k + row : e] * static_cast<double>(m.scale));
    const int64_t to = row * m.ld + col;
    if (c.out_bf16)
      static_cast<uint16_t *>(at.out)[to] = narrow_bf16(o);
    else
      static_cast<float *>(at.out)[to] = o;
  }
}

}  // namespace

hipError_t launch_tiny(const Call &c, const Steps &steps, const int32_t *list, int32_t count, hipStream_t s) {
  k_tiny<<<count, kTinyThreads, 0, s>>>(c, steps, list);
  return hipGetLastError();
}

hipError_t launch_addresses(const Call &c, const Few &few, int32_t first, int32_t count, hipStream_t s) {
  k_addresses<<<1, 64, 0, s>>>(c.addresses, few, first, count);
  return hipGetLastError();
}

hipError_t launch_squares(const Call &c, const Item *items, int32_t count, hipStream_t s) {
  k_squares<<<count, 256, 0, s>>>(c, items);
  return hipGetLastError();
}

hipError_t launch_norms(const Call &c, int32_t matrices, hipStream_t s) {
  k_norms<<<matrices, 256, 0, s>>>(c);
  return hipGetLastError();
}

hipError_t launch_load(const Call &c, const Item *items, int32_t count, hipStream_t s) {
  k_load<<<count, 256, 0, s>>>(c, items);
  return hipGetLastError();
}

namespace {
template <int T>
constexpr size_t shared_bytes() {
  return sizeof(half) * kRing * 2 * T * kDeep;
}

template <typename F>
hipError_t with_products(int tile, Phase phase, bool split, F &&f) {
  auto sized = [&](auto t) {
    constexpr int T = t();
    if (phase == kGram)
      return split ? f(k_products<T, kGram, true>, shared_bytes<T>()) : f(k_products<T, kGram, false>, shared_bytes<T>());
    if (phase == kPolynomial)
      return split ? f(k_products<T, kPolynomial, true>, shared_bytes<T>())
                   : f(k_products<T, kPolynomial, false>, shared_bytes<T>());
    return split ? f(k_products<T, kUpdate, true>, shared_bytes<T>())
                 : f(k_products<T, kUpdate, false>, shared_bytes<T>());
  };
  return tile == 256 ? sized(std::integral_constant<int, 256>{}) : sized(std::integral_constant<int, 128>{});
}
}  // namespace

// More shared memory than a kernel may have unasked.
hipError_t prepare_products(int tile, bool split) {
  for (Phase p : {kGram, kPolynomial, kUpdate}) {
    hipError_t e = with_products(tile, p, split, [](auto *k, size_t bytes) {
      return hipFuncSetAttribute(reinterpret_cast<const void *>(k), hipFuncAttributeMaxDynamicSharedMemorySize,
                                 static_cast<int>(bytes));
    });
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_products(const Call &c, int tile, Phase phase, const Step &st, const Item *items, int32_t count,
                           bool split, hipStream_t s) {
  return with_products(tile, phase, split, [&](auto *k, size_t bytes) {
    k<<<count, 256, bytes, s>>>(c, st, items);
    return hipGetLastError();
  });
}

}  // namespace orth
}  // namespace slowmo
