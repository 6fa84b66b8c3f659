// What the attention kernels share: tiles of rows in shared memory, their way into the matrix cores, the
// mask, and the place of a workgroup in a batch of packed sequences.
//
// Products are 32 x 32 x 16.  A lane of a wave is (low, high) = (lane % 32, lane / 32); it holds row (or
// column) `low` of a factor, elements 8 high .. 8 high + 7 of 16, and of a product the column `low`, rows
// 8 (i / 4) + 4 high + i % 4, i = 0..15.  The 16 summed elements may come in any order that both factors
// share, and that is what saves the exchange between two products in a row: the first is computed transposed
// (scores of 32 keys by 32 queries), so that a lane's 8 results of 16 keys, rows {4 high .. + 3, 8 + 4 high .. + 3},
// are its column of the second one's right factor as they stand, and the left factor's rows are read in that order.
// With it a query's statistics lie in two lanes alone.
//
// fp32 goes by eight products of depth 2 on the same fragments: element i of both halves of the wave is one of them.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <utility>

#include "../../include/slowmo_attention.h"
#include "slowmo_status.h"

namespace slowmo {
namespace attention {

using u32 = uint32_t;
#define SLOWMO_INLINE __attribute__((always_inline))  // of lambdas: what they refer to would go through memory otherwise
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef u32 u32x2 __attribute__((ext_vector_type(2)));
typedef u32 u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2E = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kLongest = 1 << 30;  // positions of a sequence: sums of two fit 32 bits

template <typename T>
struct Kind;
template <>
struct Kind<__bf16> {
  using frag = bf16x8;
};
template <>
struct Kind<float> {
  using frag = f32x8;
};

// A tile of rows in shared memory, 16-byte chunks, a power of two of them to a row.  Chunk c of a row lies at
// c ^ turn(row): 16 lanes that read one chunk of 16 rows, and 32 lanes that read 4 rows of 4 chunks, meet in no bank.
template <typename T, int DP>
struct Tile {
  static constexpr int E = 16 / sizeof(T);              // elements of a chunk
  static constexpr int used = DP / E;
  static constexpr int C = used <= 4 ? 4 : used <= 8 ? 8 : used <= 16 ? 16 : used <= 32 ? 32 : 64;
  static constexpr int row_bytes = C * 16;
  // of a tile: at most 32 KB, of fp32 16, so that two workgroups of up to 128 elements share a compute unit
  static constexpr int rows = row_bytes <= (sizeof(T) == 2 ? 512 : 256) ? 64 : 32;
  static constexpr int bytes = rows * row_bytes;
  static __device__ __forceinline__ int turn(int row) {
    if constexpr (C >= 16) return ((row & 3) << 2) | ((row >> 2) & 3);
    else if constexpr (C == 8) return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
    else return (row >> 2) & 3;
  }
};

__device__ __forceinline__ f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(f32x8 a, f32x8 b, f32x16 c) {
#pragma unroll
  for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
  return c;
}

// m0 is written and read within the block, with the one wait between that the two need; no vector register
// is written.  The compiler keeps m0 to itself (named as clobbered it warns of it) and has no other use for it in these kernels.
__device__ __forceinline__ void to_shared(u32 shared, u32 offset, const void *base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(shared), "v"(offset), "s"(base)
               : "memory");
}
__device__ __forceinline__ void to_shared(u32 shared, const void *from) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(shared), "v"(from) : "memory");
}
// This wave's loads have arrived and its reads of shared memory are done, and so it is for every wave.
__device__ __forceinline__ void arrive() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

template <typename P>
__device__ __forceinline__ P uniform(P v) {
  if constexpr (sizeof(P) == 8) {
    u32x2 w = __builtin_bit_cast(u32x2, v);
    w[0] = __builtin_amdgcn_readfirstlane(w[0]);
    w[1] = __builtin_amdgcn_readfirstlane(w[1]);
    return __builtin_bit_cast(P, w);
  } else {
    return __builtin_bit_cast(P, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(u32, v)));
  }
}

using lds = __attribute__((address_space(3))) char;
__device__ __forceinline__ u32 offset_of(const void *p) {
  return static_cast<u32>(reinterpret_cast<uintptr_t>((const lds *)p));
}

// Shared memory by its offset.  A tile begins at a multiple of its rows' length, a power of two, so that a chunk's place
// in a row is an exclusive or: one instruction from a lane's address to any chunk of its row.
template <typename V>
__device__ __forceinline__ V shared_at(u32 offset) {
  return *reinterpret_cast<const __attribute__((address_space(3))) V *>(offset);
}

// The rows of a product's left factor: row `row` of the tile, elements 16 step + 8 high .. + 7.
template <typename T, int DP>
__device__ __forceinline__ typename Kind<T>::frag row_frag(const char *tile, int row, int step, int high) {
  using L = Tile<T, DP>;
  const u32 at = offset_of(tile) + row * L::row_bytes;
  if constexpr (sizeof(T) == 2) {
    return shared_at<bf16x8>((at + ((high ^ L::turn(row)) << 4)) ^ (step << 5));
  } else {
    const u32 first = (at + ((2 * high ^ L::turn(row)) << 4)) ^ (step << 6);
    const f32x4 a = shared_at<f32x4>(first), b = shared_at<f32x4>(first ^ 16);
    return f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  }
}

// The same for the tile transposed: element 32 block + low of the rows 16 step + {4 high .. + 3, 8 + 4 high .. + 3}.
// bf16: a transposing read hands 16 lanes a column each of 4 rows of 16.  Rows 8 further on have their chunks turned by 2 more.
template <typename T, int DP>
__device__ __forceinline__ typename Kind<T>::frag column_frag(const char *tile, int block, int step, int lane) {
  using L = Tile<T, DP>;
  const int high = lane >> 5;
  if constexpr (sizeof(T) == 2) {
    const int in = lane & 15, chunk = ((lane >> 4) & 1) * 2 + ((in & 3) >> 1), row = 4 * high + (in >> 2);
    const u32 at = offset_of(tile) + row * L::row_bytes + ((chunk ^ L::turn(row)) << 4) + (in & 1) * 8;
    s16x4 got[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const u32 from = (at ^ (block << 6) ^ (s << 5)) + (16 * step + 8 * s) * L::row_bytes;
      got[s] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) s16x4 *>(from));
    }
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(bf16x8, s16x8{got[0][0], got[0][1], got[0][2], got[0][3], got[1][0], got[1][1], got[1][2],
                                            got[1][3]});
  } else {
    const int low = lane & 31, chunk = 8 * block + (low >> 2);
    f32x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int row = 16 * step + 8 * (i >> 2) + 4 * high + (i & 3);
      v[i] = *reinterpret_cast<const float *>(tile + row * L::row_bytes + ((chunk ^ L::turn(row)) << 4) + (low & 3) * 4);
    }
    return v;
  }
}

// Rows to a tile: row r comes from base + row_at(r) elements (base and row_at of rows past the end: some row that
// may be read).  wide: 16 bytes a lane straight to shared memory, 32-bit offsets; else element by element.
template <typename T, int DP, typename F>
__device__ __forceinline__ void bring_rows(char *tile, int rows, const T *base, int dim, bool wide, F &&row_at) {
  using L = Tile<T, DP>;
  if (wide) {
    const int lane = threadIdx.x & 63, wave = uniform(static_cast<int>(threadIdx.x >> 6)), waves = blockDim.x >> 6;
    const u32 shared = uniform(offset_of(tile));
    const T *from = uniform(base);
    for (int n = wave; n < rows * L::row_bytes / 1024; n += waves) {
      const int at = n * 64 + lane, row = at / L::C, c = (at & (L::C - 1)) ^ L::turn(row);
      const u32 offset = (static_cast<u32>(row_at(row)) + c * L::E) * sizeof(T);
      if (c * L::E < dim) to_shared(uniform(shared + n * 1024), offset, from);
    }
  } else {
    for (int i = threadIdx.x; i < rows * L::used; i += blockDim.x) {
      const int row = i / L::used, c = i % L::used;
      const T *x = base + row_at(row);
      T *to = reinterpret_cast<T *>(tile + row * L::row_bytes + ((c ^ L::turn(row)) << 4));
#pragma unroll
      for (int e = 0; e < L::E; ++e) to[e] = c * L::E + e < dim ? x[c * L::E + e] : static_cast<T>(0.f);
    }
  }
}

// Eight results of a product as the right factor of the next one.
template <typename T>
__device__ __forceinline__ typename Kind<T>::frag as_frag(const f32x16 &p, int half) {
  if constexpr (sizeof(T) == 2) {
    bf16x8 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bf16x2 two = __builtin_convertvector(f32x2{p[8 * half + 2 * i], p[8 * half + 2 * i + 1]}, bf16x2);
      f[2 * i] = two[0];
      f[2 * i + 1] = two[1];
    }
    return f;
  } else {
    return f32x8{p[8 * half], p[8 * half + 1], p[8 * half + 2], p[8 * half + 3], p[8 * half + 4], p[8 * half + 5],
                 p[8 * half + 6], p[8 * half + 7]};
  }
}

// Eight elements of a row in memory from element d on, zeros past the head's end.
template <typename T>
__device__ __forceinline__ typename Kind<T>::frag load_frag(const T *row, int d, int dim, bool wide) {
  typename Kind<T>::frag f;
  if (wide) {  // 16-byte pieces, whole inside the head or outside it
    if constexpr (sizeof(T) == 2) {
      f = __builtin_bit_cast(bf16x8, d < dim ? *reinterpret_cast<const u32x4 *>(row + d) : u32x4{0, 0, 0, 0});
    } else {
      const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
      const f32x4 a = d < dim ? *reinterpret_cast<const f32x4 *>(row + d) : zero;
      const f32x4 b = d + 4 < dim ? *reinterpret_cast<const f32x4 *>(row + d + 4) : zero;
      f = f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = d + i < dim ? row[d + i] : static_cast<T>(0.f);
  }
  return f;
}

// The value is waited for here: its first use inside a loop would wait in every turn, and with it for the loads to
// shared memory that are under way (a tile 18 instead of 3 us).
template <typename V>
__device__ __forceinline__ void settle(V &v) {
  asm volatile("" : "+v"(v));
}

// Keeps what follows a uniform condition behind it: the mask's comparisons, which few tiles need, would otherwise be
// made for every one.
__device__ __forceinline__ void branch() { asm volatile(""); }

// The order of a stretch of N steps of PRODUCTS products that take READS reads of shared memory: AHEAD steps' reads first, then
// a step's products and the reads of the one AHEAD of it in turn.  Left to itself the compiler reads for one product at a
// time and waits for it.
template <int PRODUCTS, int READS, int AHEAD, int... I>
__device__ __forceinline__ void read_ahead(std::integer_sequence<int, I...>) {
  __builtin_amdgcn_sched_group_barrier(0x100, AHEAD * READS, 0);
  ((__builtin_amdgcn_sched_group_barrier(0x8, PRODUCTS, 0), __builtin_amdgcn_sched_group_barrier(0x100, READS, 0), (void)I), ...);
  __builtin_amdgcn_sched_group_barrier(0x8, AHEAD * PRODUCTS, 0);
}
template <typename T, int N, int PRODUCTS, int READS, int AHEAD>
__device__ __forceinline__ void read_ahead() {
  if constexpr (sizeof(T) == 2 && N > AHEAD) read_ahead<PRODUCTS, READS, AHEAD>(std::make_integer_sequence<int, N - AHEAD>{});
  __builtin_amdgcn_sched_barrier(0);
}

// The two halves of the wave exchanged: x's upper with y's lower.
__device__ __forceinline__ void swap_halves(u32 &x, u32 &y) {
  const auto r = __builtin_amdgcn_permlane32_swap(x, y, false, false);
  x = r[0];
  y = r[1];
}
__device__ __forceinline__ float both_max(float v) {
  u32 a = __builtin_bit_cast(u32, v), b = a;
  swap_halves(a, b);
  return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
__device__ __forceinline__ float both_sum(float v) {
  u32 a = __builtin_bit_cast(u32, v), b = a;
  swap_halves(a, b);
  return __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
}

// A lane's column of a transposed result, elements 8 (i / 4) + 4 high + i % 4 of 32 a block, times `by`, to a row.
template <typename T, int NB>
__device__ __forceinline__ void store_columns(T *row, const f32x16 (&acc)[NB], float by, int dim, int high, bool wide,
                                              bool write) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        u32 w[2][2];
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
          for (int i = 0; i < 2; ++i)
            w[q][i] = __builtin_bit_cast(
                u32, __builtin_convertvector(f32x2{acc[b][8 * a + 4 * q + 2 * i] * by, acc[b][8 * a + 4 * q + 2 * i + 1] * by},
                                             bf16x2));
        swap_halves(w[0][0], w[1][0]);
        swap_halves(w[0][1], w[1][1]);
        // now lane (low, high) has elements 32 b + 16 a + 8 high .. + 7
        const int d = 32 * b + 16 * a + 8 * high;
        const u32x4 all = {w[0][0], w[0][1], w[1][0], w[1][1]};
        if (!write || d >= dim) continue;
        if (wide) {
          *reinterpret_cast<u32x4 *>(row + d) = all;
        } else {
          const bf16x8 v = __builtin_bit_cast(bf16x8, all);
          for (int i = 0; i < 8 && d + i < dim; ++i) row[d + i] = v[i];
        }
      }
  } else {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int d = 32 * b + 8 * q + 4 * high;
        if (!write || d >= dim) continue;
        const f32x4 v = {acc[b][4 * q] * by, acc[b][4 * q + 1] * by, acc[b][4 * q + 2] * by, acc[b][4 * q + 3] * by};
        if (wide) {
          *reinterpret_cast<f32x4 *>(row + d) = v;
        } else {
          for (int i = 0; i < 4 && d + i < dim; ++i) row[d + i] = v[i];
        }
      }
  }
}

// A [tokens][heads][D] array as the kernels have it; strides in elements.
struct Rows {
  void *data;
  int64_t token, head;
};

// Where a workgroup is: tile `tile` of `height` rows of sequence `b`, whose rows lie at begin .. begin + n - 1.
// Sequence b's workgroups start at floor(begin rows / height) + b, which leaves room for all its tiles before the
// next one's: no prefix sum and no longest length is needed.  b = batch: the rows behind the last sequence.
struct Place {
  int b, n, tile;
  int64_t begin;
};
__device__ __forceinline__ int64_t clamped(int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; }
__device__ __forceinline__ int64_t lane_of(int64_t v, int lane) {
  const u32x2 w = __builtin_bit_cast(u32x2, v);
  return __builtin_bit_cast(int64_t, u32x2{static_cast<u32>(__builtin_amdgcn_readlane(w[0], lane)),
                                           static_cast<u32>(__builtin_amdgcn_readlane(w[1], lane))});
}
// The first entry of a stretch of at most 256 that holds the last one that `before` is true of (it is true up to some
// entry and false from there on): halved down to that from 1024 sequences on, for 1024 to 8192 of them 3 to 6 single entries in
// place of 4 to 32 stretches, for 2^20, the most, 13 in place of 4096.  One token of each of 1024 and 8192 sequences over a cache of 50 each, 8 heads of 64: 29.8 -> 26.3 us and
// 464 -> 167 us.
template <typename F>
__device__ __forceinline__ int stretch_of(int batch, F &&before) {
  int lo = 0, hi = batch + 1;
  if (batch >= 1024)
    while (hi - lo > 256) {
      const int mid = lo + (hi - lo) / 2;
      if (before(mid)) lo = mid;
      else hi = mid;
    }
  return lo;
}
// Four lanes' worth of entries are asked for at once: one trip to memory for up to 255 sequences.
__device__ __forceinline__ Place place_of(const int64_t *offsets, int batch, int64_t tokens, int group, int height,
                                          int64_t slot) {
  const int lane = threadIdx.x & 63, shift = __builtin_ctz(height);
  Place p{-1, 0, 0, 0};
  int64_t end = tokens;
  const int start = stretch_of(batch, [&](int b) { return (clamped(uniform(offsets[b]), 0, tokens) * group >> shift) + b <= slot; });
  for (int first = start; first <= batch; first += 256) {
    int64_t v[4];
#pragma unroll
    for (int c = 0; c < 4; ++c)
      v[c] = first + 64 * c <= batch ? clamped(offsets[min(first + 64 * c + lane, batch)], 0, tokens) : 0;
    int got = 64;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int b = first + 64 * c + lane;
      if (got < 64 || first + 64 * c > batch) continue;
      got = __popcll(__ballot(b <= batch && (v[c] * group >> shift) + b <= slot));
      if (got) p.b = first + 64 * c + got - 1, p.begin = lane_of(v[c], got - 1);
      if (got < 64 && p.b < batch) end = lane_of(v[c], got);
    }
    if (got < 64) break;
  }
  if (p.b < 0) return p;
  end = p.b < batch ? max(end, p.begin) : tokens;
  p.n = static_cast<int>(end - p.begin);
  p.tile = static_cast<int>(slot - p.b - (p.begin * group >> shift));
  return p;
}

// Rows, token by token and head by head within, from row0 on as tokens and heads: by one division for a workgroup.
struct Split {
  int t0, o0, group;
  u32 by_group;  // 2^32 / group, rounded up: exact for what is asked here, o0 and some hundred rows
  __device__ __forceinline__ Split(int64_t row0, int group, u32 by_group) : group(group), by_group(by_group) {
    if (group == 1) t0 = static_cast<int>(row0), o0 = 0;
    else if (row0 >> 32) t0 = static_cast<int>(row0 / group), o0 = static_cast<int>(row0 - static_cast<int64_t>(t0) * group);
    else t0 = static_cast<int>(static_cast<u32>(row0) / static_cast<u32>(group)), o0 = static_cast<int>(row0) - t0 * group;
  }
  __device__ __forceinline__ int token(int r) const { return t0 + (group > 1 ? __umulhi(o0 + r, by_group) : r); }
  __device__ __forceinline__ int head(int r, int token) const { return o0 + r - (token - t0) * group; }
};
inline u32 by_group(int group) { return static_cast<u32>(((uint64_t(1) << 32) + group - 1) / group); }

inline int64_t slots_of(int64_t tokens, int64_t group, int64_t height, int64_t batch) {
  return tokens * group / height + batch + 1;
}

// Workgroup -> (head, slot).  Workgroup b runs on XCD b mod 8: the tiles of one key head share an XCD's
// L2 as far as the number of heads lets them.
__device__ __forceinline__ bool head_slot(int64_t item, int heads, int64_t slots, int &head, int64_t &slot) {
  if (heads % 8 == 0) {
    const int per = heads / 8;
    const int64_t y = item / 8;
    head = static_cast<int>(item % 8) * per + static_cast<int>(y % per);
    slot = y / per;
  } else if (8 % heads == 0) {
    const int x = static_cast<int>(item % 8);
    head = x % heads;
    slot = item / 8 * (8 / heads) + x / heads;
  } else {
    head = static_cast<int>(item % heads);
    slot = item / heads;
  }
  return slot < slots;
}
inline int64_t items_of(int64_t heads, int64_t slots) {
  return heads % 8 != 0 && 8 % heads == 0 ? (slots + 8 / heads - 1) / (8 / heads) * 8 : heads * slots;
}

// The mask from a query's side: it sees the keys lo..hi and those below `sinks`.
struct Mask {
  int causal, window, sinks;  // window 0: none
};
struct Sight {
  int lo, hi, sinks;
};
__device__ __forceinline__ Sight sight_of(const Mask &m, int p, int keys) {
  Sight s;
  const int last = m.causal ? min(p, keys - 1) : keys - 1;
  s.lo = 0, s.hi = last, s.sinks = 0;
  if (m.window) {
    s.lo = max(0, p - m.window + 1);
    s.hi = min(last, p + m.window - 1);
    s.sinks = min(m.sinks, last + 1);
  }
  return s;
}
__device__ __forceinline__ bool sees(const Sight &s, int j) { return (j >= s.lo && j <= s.hi) || j < s.sinks; }

// Whether a value is an infinity or no number.
__device__ __forceinline__ bool wild(float v) { return (__builtin_bit_cast(u32, v) & 0x7f800000u) == 0x7f800000u; }

// The element d of row `row` of a tile.
template <typename T, int DP>
__device__ __forceinline__ T *element(char *tile, int row, int d) {
  using L = Tile<T, DP>;
  return reinterpret_cast<T *>(tile + row * L::row_bytes + (((d / L::E) ^ L::turn(row)) << 4)) + d % L::E;
}

// Where a row of a tile is seen by some columns of a product only, what is wild in it must not meet the
// others' zeros (0 times infinity).  Only a pass whose result came out wild is done again, tile by tile, with what is wild
// taken out of the tiles (tame, or, where the tile is a factor of something else as well, a copy without it) and added to
// the columns that see it (add_wild).  All waves of the workgroup come to these.
template <typename T, int DP, int ROWS>
__device__ __forceinline__ bool any_wild(char *tile) {
  int any = 0;
  for (int i = threadIdx.x; i < ROWS * DP; i += blockDim.x)
    any |= wild(static_cast<float>(*element<T, DP>(tile, i / DP, i % DP)));
  return __syncthreads_or(any);
}
// `seen(row)`: whether the lane's column sees the tile's row.  `times` what is wild: 0 makes NaN of it.
template <typename T, int DP, int ROWS, int NB, typename F>
__device__ __forceinline__ void add_wild(char *tile, f32x16 (&acc)[NB], float times, F &&seen) {
  const int high = (threadIdx.x & 63) >> 5;
  for (int row = 0; row < ROWS; ++row) {
    const bool mine = seen(row);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float v = static_cast<float>(*element<T, DP>(tile, row, 32 * b + 8 * (i / 4) + 4 * high + i % 4));
        if (mine && wild(v)) acc[b][i] += v * times;
      }
  }
}
template <typename T, int DP, int ROWS>
__device__ __forceinline__ void tame(char *to, char *tile) {
  for (int i = threadIdx.x; i < ROWS * DP; i += blockDim.x) {
    const T e = *element<T, DP>(tile, i / DP, i % DP);
    *element<T, DP>(to, i / DP, i % DP) = wild(static_cast<float>(e)) ? static_cast<T>(0.f) : e;
  }
  __syncthreads();
}

// The tiles of keys that some row of a workgroup sees: `head` tiles from the sinks, then those from `first` on.
struct Walk {
  int head, first, count;
  __device__ __forceinline__ int at(int u) const { return u < head ? u : first + (u - head); }
};
// Positions from `held` on have no page: of them the walk takes in what makes each row that sees one see one of its tiles,
// and no more, however far a sequence's length says that it reaches.
__device__ __forceinline__ Walk walk_of(const Mask &m, int p_lo, int p_hi, int keys, int tile, int held = kLongest) {
  const Sight a = sight_of(m, p_lo, keys), b = sight_of(m, p_hi, keys);
  int lo = a.lo, hi = b.hi;
  const int sinks = min(b.sinks, held + 1), end = max(held, b.lo);
  Walk w{0, 0, 0};
  if (sinks > lo) hi = max(hi, sinks - 1), lo = 0;
  else if (hi < lo && sinks > 0) lo = 0, hi = sinks - 1;
  hi = min(hi, end);
  if (hi < lo) return w;
  w.first = lo / tile;
  w.head = sinks > 0 ? min((sinks + tile - 1) / tile, w.first) : 0;
  w.count = w.head + hi / tile - w.first + 1;
  return w;
}
// A walk over `count` tiles in pieces of `per`: at least `least` tiles each, at most `splits` pieces.
__device__ __forceinline__ int pieces_of(int count, int splits, int least, int &per) {
  per = max(least, (count + splits - 1) / splits);
  return count ? (count + per - 1) / per : 1;
}

// ---- the C entries ----

template <int DP, typename F>
void with_kind(int32_t dtype, F &&f) {
  if (dtype == SLOWMO_BF16) f(__bf16{}, std::integral_constant<int, DP>{});
  else f(float{}, std::integral_constant<int, DP>{});
}
template <typename F>
void dispatch(int32_t dtype, int dim, F &&f) {
  if (dim <= 32) with_kind<32>(dtype, f);
  else if (dim <= 64) with_kind<64>(dtype, f);
  else if (dim <= 96) with_kind<96>(dtype, f);
  else if (dim <= 128) with_kind<128>(dtype, f);
  else if (dim <= 192) with_kind<192>(dtype, f);
  else with_kind<256>(dtype, f);
}
inline int padded(int dim) { return dim <= 32 ? 32 : dim <= 64 ? 64 : dim <= 96 ? 96 : dim <= 128 ? 128 : dim <= 192 ? 192 : 256; }

inline int rows_of_tile(int dim, int32_t dtype) {
  int rows = 0;
  dispatch(dtype, dim, [&](auto kind, auto dp) { rows = Tile<decltype(kind), dp()>::rows; });
  return rows;
}

// Waves of a workgroup: as many as a sequence's rows fill on the average.
inline int waves_of(int64_t tokens, int64_t group, int64_t batch, int most) {
  const int64_t rows = tokens * group / std::max<int64_t>(batch, 1);
  int waves = 1;
  while (waves < most && waves * 32 < rows) waves *= 2;
  return waves;
}

inline bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
inline size_t size_of(int32_t dtype) { return dtype == SLOWMO_BF16 ? 2 : 4; }
inline Rows rows_of(const slowmo_heads &h) { return {h.data, h.token_stride, h.head_stride}; }

const char *check_config(const slowmo_attention_config *c);
constexpr int kMostShared = 1 << 12;  // query heads of a key head
slowmo_status check_call(const slowmo_attention_config *cfg, int32_t batch, const int64_t *q_offsets, const int64_t *k_offsets,
                         int64_t tokens, int64_t keys);
slowmo_status check_group(int64_t tokens, int32_t q_heads, int32_t k_heads);
Mask mask_of(const slowmo_attention_config &c);
// `written`: its rows may not fall on one another.
slowmo_status check_rows(const slowmo_heads *h, int64_t rows, int32_t dim, int32_t dtype, bool written);
slowmo_status check_cache(const slowmo_cache *c, int32_t dim, int32_t dtype, bool written);
slowmo_status check_pages(const slowmo_pages *p, int64_t tokens);

// An array's stretch in memory, and what it covers of every `period` bytes, for two such periods.
struct Extent {
  uintptr_t lo = 0, hi = 0;
  int64_t period[2] = {0, 0}, width[2] = {0, 0};
};
Extent extent(const slowmo_heads &h, int64_t rows, int32_t dim, int32_t dtype);
Extent extent(const slowmo_cache &c, int32_t dim, int32_t dtype);
Extent extent(const void *p, size_t bytes);
bool overlap(const Extent &x, const Extent &y);

// Whether rows can go to shared memory 16 bytes at a time, with 32-bit offsets inside a tile.
bool wide_rows(const slowmo_heads &h, int32_t dim, int32_t dtype);
bool wide_rows(const slowmo_cache &c, int32_t dim, int32_t dtype);

constexpr int64_t kMostBlocks = 1 << 22;  // workgroups of a launch: a grid has less than 2^32 threads

}  // namespace attention
}  // namespace slowmo
