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

namespace slowmo {
namespace orth {
namespace {

typedef _Float16 half;
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
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

// X_0 and its transpose as halves, with zeros in the padding (which an earlier call's NaN may have
// reached).
template <bool SPLIT>
__global__ __launch_bounds__(256) void k_load(Call c, const Item *items) {
  const Item it = items[blockIdx.x];
  const Matrix &m = c.matrices[it.matrix];
  const Addresses at = c.addresses[it.matrix];
  const int rows = m.tall ? m.k : m.n, cols = m.tall ? m.n : m.k;
  const int prows = m.tall ? m.kp : m.np, pcols = m.tall ? m.np : m.kp;
  half *natural = c.arena + (m.tall ? m.xt[0] : m.x), *turned = c.arena + (m.tall ? m.x : m.xt[0]);
  // lo parts: of XT always, of X where products are split
  half *natural_lo = m.tall ? c.arena + m.xt_lo[0] : SPLIT ? c.arena + m.x_lo : nullptr;
  half *turned_lo = m.tall ? (SPLIT ? c.arena + m.x_lo : nullptr) : c.arena + m.xt_lo[0];
  const float inverse = c.inverse[it.matrix];
  __shared__ half hi[kPatch][kPatch + 2], lo[kPatch][kPatch + 2];
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
    split_half(u, hi[r][lane], lo[r][lane]);
    const int64_t to = static_cast<int64_t>(row) * pcols + col;
    natural[to] = hi[r][lane];
    if (natural_lo) natural_lo[to] = lo[r][lane];
  }
  __syncthreads();
  for (int r = threadIdx.x >> 6; r < kPatch; r += 4) {
    const int64_t to = static_cast<int64_t>(it.j * kPatch + r) * prows + it.i * kPatch + lane;
    turned[to] = hi[lane][r];
    if (turned_lo) turned_lo[to] = lo[lane][r];
  }
}

// C = A B^T over tiles of 128 x 128, 4 waves of 64 x 64.  Both factors lie with the summed side
// contiguous and padded, so nothing is checked in the loop.  A step of 64 goes from memory straight to
// shared memory, 16 bytes a lane; there the 16-byte pieces of a row of 128 bytes are placed at
// (piece xor row mod 8), so that lanes that read the same piece of neighbouring rows meet different banks.
template <int PHASE, bool SPLIT>
__global__ __launch_bounds__(256) void k_products(Call c, Step st, const Item *items) {
  __shared__ half tiles[2][2][kTile * kDepth];
  const Item it = items[blockIdx.x];
  const Matrix &m = c.matrices[it.matrix];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int depth = PHASE == kGram ? m.kp : m.np;
  const int64_t rows_hi = PHASE == kGram ? m.x : PHASE == kPolynomial ? m.a : m.xt[st.from];
  const int64_t rows_lo = PHASE == kGram ? m.x_lo : PHASE == kPolynomial ? m.a_lo : m.xt_lo[st.from];
  const int64_t cols_hi = PHASE == kUpdate ? m.p : rows_hi;
  const int64_t cols_lo = PHASE == kUpdate ? m.p_lo : rows_lo;
  const int steps = depth / kDepth, total = SPLIT ? 3 * steps : steps;

  auto fetch = [&](int t) {
    // split: the small products first (hi lo, lo hi), while their sums are small, then hi hi
    const int seg = SPLIT ? t / steps : 2;
    const int64_t at = static_cast<int64_t>(SPLIT ? t - seg * steps : t) * kDepth;
    const half *a = c.arena + (seg == 1 ? rows_lo : rows_hi) + static_cast<int64_t>(it.i) * kTile * depth + at;
    const half *b = c.arena + (seg == 0 ? cols_lo : cols_hi) + static_cast<int64_t>(it.j) * kTile * depth + at;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int row = (wave * 4 + q) * 8 + (lane >> 3);
      const int piece = (lane & 7) ^ (lane >> 3);
      const int64_t off = static_cast<int64_t>(row) * depth + piece * 8;
      half *la = &tiles[t & 1][0][(wave * 4 + q) * 8 * kDepth], *lb = &tiles[t & 1][1][(wave * 4 + q) * 8 * kDepth];
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(a + off),
                                       (__attribute__((address_space(3))) void *)la, 16, 0, 0);
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(b + off),
                                       (__attribute__((address_space(3))) void *)lb, 16, 0, 0);
    }
  };

  f32x16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  fetch(0);
  for (int t = 0; t < total; ++t) {
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();  // this step's tiles are there, and nobody reads the other pair any more
    half8 fa[4][2], fb[4][2];
    const half *ta = tiles[t & 1][0], *tb = tiles[t & 1][1];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int ra = wm * 64 + i * 32 + (lane & 31), rb = wn * 64 + i * 32 + (lane & 31);
        const int piece = kk * 2 + (lane >> 5);
        fa[kk][i] = *reinterpret_cast<const half8 *>(ta + ra * kDepth + ((piece ^ (ra & 7)) * 8));
        fb[kk][i] = *reinterpret_cast<const half8 *>(tb + rb * kDepth + ((piece ^ (rb & 7)) * 8));
      }
    }
    if (t + 1 < total) fetch(t + 1);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fb[kk][j], fa[kk][i], acc[i][j], 0, 0, 0);
  }

  // A lane holds, of a block of 32 x 32, row (lane & 31) and four times four neighbouring columns.
  const Addresses at = c.addresses[it.matrix];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int row = it.i * kTile + wm * 64 + i * 32 + (lane & 31);
        const int col = it.j * kTile + wn * 64 + j * 32 + g * 8 + (lane >> 5) * 4;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = acc[i][j][g * 4 + e];
        const int64_t pos = static_cast<int64_t>(row) * m.np + col;
        if constexpr (PHASE == kUpdate) {
          const half4 hi = *reinterpret_cast<const half4 *>(c.arena + m.xt[st.from] + pos);
          const half4 lo = *reinterpret_cast<const half4 *>(c.arena + m.xt_lo[SPLIT ? st.from : 0] + pos);
          half4 nh, nl;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = static_cast<float>(hi[e]) + static_cast<float>(lo[e]);
            v[e] = fmaf(st.a, x, v[e] * (1.f / kScaleP));
            half h, l;
            split_half(v[e], h, l);
            nh[e] = h;
            nl[e] = l;
          }
          if (!st.last) {
            *reinterpret_cast<half4 *>(c.arena + m.xt[1 - st.from] + pos) = nh;
            *reinterpret_cast<half4 *>(c.arena + m.xt_lo[SPLIT ? 1 - st.from : 0] + pos) = nl;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int64_t to = static_cast<int64_t>(col + e) * m.kp + row;
              c.arena[m.x + to] = nh[e];
              if (SPLIT) c.arena[m.x_lo + to] = nl[e];
            }
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if (row >= m.k || col + e >= m.n) continue;
              const int64_t to = m.tall ? row * m.ld + col + e : (col + e) * m.ld + row;
              const float o = v[e] * (m.scale / kScaleX);
              if (c.out_bf16)
                static_cast<uint16_t *>(at.out)[to] = narrow_bf16(o);
              else
                static_cast<float *>(at.out)[to] = o;
            }
          }
        } else {
          half4 nh, nl, ah, al;
          if constexpr (PHASE == kPolynomial) {
            ah = *reinterpret_cast<const half4 *>(c.arena + m.a + pos);
            if (SPLIT) al = *reinterpret_cast<const half4 *>(c.arena + m.a_lo + pos);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if constexpr (PHASE == kGram) {
              v[e] *= kScaleA / (kScaleX * kScaleX);
            } else {
              const float x = static_cast<float>(ah[e]) + (SPLIT ? static_cast<float>(al[e]) : 0.f);
              v[e] = fmaf(st.b * (kScaleP / kScaleA), x, st.c * (kScaleP / (kScaleA * kScaleA)) * v[e]);
            }
            half h, l;
            split_half(v[e], h, l);
            nh[e] = h;
            nl[e] = l;
          }
          half *to_hi = c.arena + (PHASE == kGram ? m.a : m.p), *to_lo = c.arena + (PHASE == kGram ? m.a_lo : m.p_lo);
          *reinterpret_cast<half4 *>(to_hi + pos) = nh;
          if (SPLIT) *reinterpret_cast<half4 *>(to_lo + pos) = nl;
          if (it.i != it.j) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int64_t to = static_cast<int64_t>(col + e) * m.np + row;
              to_hi[to] = nh[e];
              if (SPLIT) to_lo[to] = nl[e];
            }
          }
        }
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

hipError_t launch_load(const Call &c, const Item *items, int32_t count, bool split, hipStream_t s) {
  if (split)
    k_load<true><<<count, 256, 0, s>>>(c, items);
  else
    k_load<false><<<count, 256, 0, s>>>(c, items);
  return hipGetLastError();
}

hipError_t launch_products(const Call &c, Phase phase, const Step &st, const Item *items, int32_t count,
                           bool split, hipStream_t s) {
  if (phase == kGram)
    split ? k_products<kGram, true><<<count, 256, 0, s>>>(c, st, items)
          : k_products<kGram, false><<<count, 256, 0, s>>>(c, st, items);
  else if (phase == kPolynomial)
    split ? k_products<kPolynomial, true><<<count, 256, 0, s>>>(c, st, items)
          : k_products<kPolynomial, false><<<count, 256, 0, s>>>(c, st, items);
  else
    split ? k_products<kUpdate, true><<<count, 256, 0, s>>>(c, st, items)
          : k_products<kUpdate, false><<<count, 256, 0, s>>>(c, st, items);
  return hipGetLastError();
}

}  // namespace orth
}  // namespace slowmo
