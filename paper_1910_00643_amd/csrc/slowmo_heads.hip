// Norm of queries and keys for each head with the position rotation in the same pass, and its
// gradient (include/slowmo_operators.h has the formulas).
//
// Memory bounds both: a pass reads and writes every element once (forward 2 accesses an element,
// backward 3).  A head's row lies in the registers of one group of lanes from its load to its
// store: every lane holds both elements of its pairs, so that the rotation needs no other lane and
// the mean of squares is the only exchange.  A wave has queries or keys only -- one weight and one
// sum for its gradient in registers -- and, where a token has enough heads, one token at a time, whose
// angles are fetched once.
// Measured: forward 4.2 TB/s (8192 tokens of 32 heads of 64, bf16, 67 MB in 16 us), 4.3 TB/s on two axes in
// fp32 (12 017 tokens of 32 heads of 72, 221 MB in 52 us), both within the last-level cache, as repeated calls on the
// same buffers are; backward 4.8 TB/s (32 768 tokens of 40 heads of 128,
// 1.0 GB in 213 us); a large copy reaches 4.8 TB/s.  48 single tokens: 4.6 us of a call's 10, the rest its
// launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "../../include/slowmo_operators.h"
#include "slowmo_status.h"

namespace slowmo {
namespace {

constexpr int kWaves = 4;                      // waves per workgroup
constexpr int kThreads = 64 * kWaves;
constexpr int kPairs = SLOWMO_MAX_HEAD_DIM / 2;
constexpr int kMostBlocks = 1 << 23;           // workgroups of a launch: a grid has less than 2^32 threads
constexpr int kFill = 8192;                    // waves that fill the card: 256 CUs, 8 waves per SIMD
constexpr int kWalks = 768;                    // workgroups of a backward pass: all run at once, 3 per CU

struct Rows {
  void *data;
  int64_t token, head;
};

// Queries or keys.  A turn of a wave takes `groups` rows: heads of one token, or, where it has fewer
// heads than there are groups, all heads of `together` tokens.
struct Side {
  Rows x, g, y;          // inputs; backward: gradients of the outputs; outputs
  const float *weight;
  int64_t units;         // blocks of `together` tokens times `parts`
  int32_t heads, together;
  int32_t parts;         // waves that share a token's heads
};

struct HeadArgs {
  int64_t tokens;
  int64_t first;         // forward: the unit that this launch begins with
  const float *table;
  const int64_t *positions;
  int64_t table_rows, position_stride;
  Side side[2];
  const int64_t *slots;
  int64_t slot_rows;
  float *partial;        // backward: [workgroups][2][D] sums for the weights' gradients
  int32_t dim, rot;
  int32_t chunks;        // pieces of 2V elements in a row
  int32_t lanes, groups; // lanes of a row, rows of a wave
  int32_t lanes_log2;    // with the norm: lanes is a power of two
  int32_t q_blocks;      // backward: workgroups of the queries, the keys' come after them
  int32_t axes;
  float eps;
  uint32_t pair_axis[kPairs / 16];  // 2 bits a pair
};

template <typename T>
__device__ __forceinline__ float widen(T v);
template <>
__device__ __forceinline__ float widen<float>(float v) { return v; }
template <>
__device__ __forceinline__ float widen<uint16_t>(uint16_t v) {
  return __builtin_bit_cast(float, static_cast<uint32_t>(v) << 16);
}

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Two fp32 values rounded to nearest even, the first in the low half.
__device__ __forceinline__ uint32_t narrow2(float a, float b) {
  f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// A vector's load and store; NT: past the caches, for rows that nobody reads again soon.
template <bool NT, typename V>
__device__ __forceinline__ V fetch(const void *p) {
  if constexpr (NT)
    return __builtin_nontemporal_load(static_cast<const V *>(p));
  else
    return *static_cast<const V *>(p);
}
template <bool NT, typename V>
__device__ __forceinline__ void leave(void *p, V v) {
  if constexpr (NT)
    __builtin_nontemporal_store(v, static_cast<V *>(p));
  else
    *static_cast<V *>(p) = v;
}

template <typename T, int V>
struct Piece;  // V neighbouring elements

template <>
struct Piece<float, 8> {
  template <bool NT = false>
  static __device__ __forceinline__ void load(const float *p, float *o) {
    const f32x4 a = fetch<NT, f32x4>(p), b = fetch<NT, f32x4>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = a[i], o[4 + i] = b[i];
  }
  template <bool NT = false>
  static __device__ __forceinline__ void store(float *p, const float *o) {
    leave<NT>(p, f32x4{o[0], o[1], o[2], o[3]});
    leave<NT>(p + 4, f32x4{o[4], o[5], o[6], o[7]});
  }
};
template <>
struct Piece<float, 4> {
  template <bool NT = false>
  static __device__ __forceinline__ void load(const float *p, float *o) {
    const f32x4 a = fetch<NT, f32x4>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = a[i];
  }
  template <bool NT = false>
  static __device__ __forceinline__ void store(float *p, const float *o) {
    leave<NT>(p, f32x4{o[0], o[1], o[2], o[3]});
  }
};
template <typename T>
struct Piece<T, 1> {
  template <bool NT = false>
  static __device__ __forceinline__ void load(const T *p, float *o) { o[0] = widen(*p); }
  template <bool NT = false>
  static __device__ __forceinline__ void store(T *p, const float *o) {
    if constexpr (sizeof(T) == 4)
      *p = o[0];
    else
      *p = static_cast<uint16_t>(narrow2(o[0], 0.f));
  }
};
template <>
struct Piece<uint16_t, 8> {
  template <bool NT = false>
  static __device__ __forceinline__ void load(const uint16_t *p, float *o) {
    const u32x4 a = fetch<NT, u32x4>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[2 * i] = __builtin_bit_cast(float, a[i] << 16);
      o[2 * i + 1] = __builtin_bit_cast(float, a[i] & 0xffff0000u);
    }
  }
  template <bool NT = false>
  static __device__ __forceinline__ void store(uint16_t *p, const float *o) {
    leave<NT>(p, u32x4{narrow2(o[0], o[1]), narrow2(o[2], o[3]), narrow2(o[4], o[5]), narrow2(o[6], o[7])});
  }
};
template <>
struct Piece<uint16_t, 4> {
  template <bool NT = false>
  static __device__ __forceinline__ void load(const uint16_t *p, float *o) {
    const u32x2 a = fetch<NT, u32x2>(p);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      o[2 * i] = __builtin_bit_cast(float, a[i] << 16);
      o[2 * i + 1] = __builtin_bit_cast(float, a[i] & 0xffff0000u);
    }
  }
  template <bool NT = false>
  static __device__ __forceinline__ void store(uint16_t *p, const float *o) {
    leave<NT>(p, u32x2{narrow2(o[0], o[1]), narrow2(o[2], o[3])});
  }
};

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(
      float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}

// The sum over aligned groups of 1 << log2 lanes, the same bits in every lane of a group.
__device__ __forceinline__ float group_sum(float v, int log2) {
  if (log2 > 0) v += dpp<0xB1>(v);   // quad_perm 1,0,3,2
  if (log2 > 1) v += dpp<0x4E>(v);   // quad_perm 2,3,0,1
  if (log2 > 2) v += dpp<0x141>(v);  // row_half_mirror
  if (log2 > 3) v += dpp<0x140>(v);  // row_mirror
  if (log2 > 4) v += __shfl_xor(v, 16);
  if (log2 > 5) v += __shfl_xor(v, 32);
  return v;
}

// Where a lane's share of a row lies: V elements at u and V at v (elements from the row's start),
// of which the i-th of each are a pair (PAIRS apart) or neighbours are (interleaved, and past the
// rotated part, where nothing is turned).
struct Place {
  int32_t u, v;
  bool here, both;  // the lane has a share; the second half of it exists (V == 1 in an odd row)
  bool turned;
  int32_t pair;     // first pair
};

template <int V, bool INTER>
__device__ __forceinline__ Place place(const HeadArgs &a, int chunk) {
  Place p;
  p.here = chunk < a.chunks;
  const int turning = a.rot / (2 * V);
  p.turned = chunk < turning;
  p.pair = chunk * V;
  if (!INTER && p.turned) {
    p.u = chunk * V;
    p.v = a.rot / 2 + chunk * V;
  } else {
    p.u = chunk * 2 * V;
    p.v = p.u + V;
  }
  p.both = V > 1 || p.v < a.dim;
  return p;
}

__device__ __forceinline__ int axis_of(const HeadArgs &a, int pair) {
  return (a.pair_axis[pair >> 4] >> (2 * (pair & 15))) & 3;
}

// cos and sin of a lane's pairs for token t.  `axis`: of the lane's pairs where they share one, else -1 less all
// of them, two bits each.
template <int V>
__device__ __forceinline__ void angles(const HeadArgs &a, const Place &p, int axis, int64_t t, float *c,
                                       float *s) {
#pragma unroll
  for (int i = 0; i < V; ++i) c[i] = 1.f, s[i] = 0.f;
  if (!p.here || !p.turned) return;
  const int half = a.rot / 2;
  if (axis >= 0) {
    const int64_t at = a.positions[axis * a.position_stride + t];
    if (at >= 0 && at < a.table_rows) {
      const float *row = a.table + at * a.rot + p.pair;
      Piece<float, V>::load(row, c);
      Piece<float, V>::load(row + half, s);
    } else if (at != -1) {
#pragma unroll
      for (int i = 0; i < V; ++i) c[i] = s[i] = __builtin_nanf("");
    }
    return;
  }
  // every axis' position, then every pair's angle, each all on their way together
  const uint32_t axes = -1 - axis;
  int64_t at[SLOWMO_MAX_AXES], of[V];
#pragma unroll
  for (int i = 0; i < SLOWMO_MAX_AXES; ++i) at[i] = a.positions[min(i, a.axes - 1) * a.position_stride + t];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t which = (axes >> (2 * i)) & 3;
    of[i] = which < 2 ? (which ? at[1] : at[0]) : which == 2 ? at[2] : at[3];
  }
  if (a.table_rows > 0) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float *row = a.table + (of[i] >= 0 && of[i] < a.table_rows ? of[i] : 0) * a.rot + p.pair + i;
      c[i] = row[0];
      s[i] = row[half];
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if (of[i] >= 0 && of[i] < a.table_rows) continue;
    c[i] = of[i] == -1 ? 1.f : __builtin_nanf("");
    s[i] = of[i] == -1 ? 0.f : __builtin_nanf("");
  }
}

template <int V>
__device__ __forceinline__ int shared_axis(const HeadArgs &a, const Place &p) {
  if (a.axes == 1 || !p.here || !p.turned) return 0;
  const int first = axis_of(a, p.pair);
  int all = first;
  bool one = true;
  for (int i = 1; i < V; ++i) {
    const int axis = axis_of(a, p.pair + i);
    one &= axis == first;
    all |= axis << (2 * i);
  }
  return one ? first : -1 - all;
}

// Turns a lane's pairs by the angle (DIR 1) or back (DIR -1).  Past the rotated part c = 1, s = 0,
// whichever two elements are taken as a pair.
template <int V, bool INTER, int DIR>
__device__ __forceinline__ void turn_pairs(float *u, float *v, const float *c, const float *s) {
  if constexpr (INTER && V > 1) {
#pragma unroll
    for (int i = 0; i < V; ++i) {  // pair i: elements 2i, 2i + 1 of u followed by v
      float *x = i < V / 2 ? u + 2 * i : v + (2 * i - V);
      const float sn = DIR > 0 ? s[i] : -s[i], p = x[0], q = x[1];
      x[0] = p * c[i] - q * sn;
      x[1] = p * sn + q * c[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float sn = DIR > 0 ? s[i] : -s[i], p = u[i], q = v[i];
      u[i] = p * c[i] - q * sn;
      v[i] = p * sn + q * c[i];
    }
  }
}

template <typename T, int V, bool NT>
__device__ __forceinline__ void load_row(const Rows &r, int64_t t, int64_t h, const Place &p, float *u,
                                         float *v) {
  const T *x = static_cast<const T *>(r.data) + t * r.token + h * r.head;
  Piece<T, V>::template load<NT>(x + p.u, u);
  if (p.both)
    Piece<T, V>::template load<NT>(x + p.v, v);
  else
    v[0] = 0.f;
}
template <typename T, int V, bool NT>
__device__ __forceinline__ void store_row(const Rows &r, int64_t t, int64_t h, const Place &p,
                                          const float *u, const float *v) {
  T *x = static_cast<T *>(r.data) + t * r.token + h * r.head;
  Piece<T, V>::template store<NT>(x + p.u, u);
  if (p.both) Piece<T, V>::template store<NT>(x + p.v, v);
}

template <int V>
__device__ __forceinline__ void load_weight(const float *w, const Place &p, float *u, float *v) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    u[i] = w && p.here ? w[p.u + i] : 1.f;
    v[i] = w && p.here && p.both ? w[p.v + i] : 1.f;
  }
}

// A row of a turn: which token and head lane group g has.
struct Row {
  int64_t t;
  int32_t h;
  bool live;
};
__device__ __forceinline__ Row row_of(const HeadArgs &a, const Side &s, int64_t block, int turn, int g) {
  Row r;
  if (s.together > 1) {
    const int ahead = g / s.heads;
    r.t = block * s.together + ahead;
    r.h = g - ahead * s.heads;
    r.live = ahead < s.together && r.t < a.tokens;
  } else {
    r.t = block;
    r.h = turn * a.groups + g;
    r.live = g < a.groups && r.h < s.heads;
  }
  if (!r.live) r.t = min(r.t, a.tokens - 1);  // read for its angles all the same
  return r;
}

// One turn of a wave or a few; where tokens are few, a turn each, so that the card is full.
// NCH: pieces of a row per lane (more than one only in the element-by-element variant).
template <typename T, int V, int NCH, bool INTER, bool NORM, bool NT>
__global__ __launch_bounds__(kThreads) void k_head_forward(HeadArgs a) {
  const int lane = threadIdx.x & 63;
  int64_t unit = a.first + static_cast<int64_t>(blockIdx.x) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool key = unit >= a.side[0].units;
  const Side &s = a.side[key];
  if (key) unit -= a.side[0].units;
  if (unit >= s.units) return;
  const int64_t block = unit / s.parts;
  const int part = static_cast<int>(unit - block * s.parts);
  const int g = lane / a.lanes, l = lane - g * a.lanes;

  Row row = row_of(a, s, block, part, g);
  Place p[NCH];
  float c[NCH][V], sn[NCH][V], w[NCH][2 * V];
#pragma unroll
  for (int j = 0; j < NCH; ++j) {
    p[j] = place<V, INTER>(a, l + a.lanes * j);
    angles<V>(a, p[j], shared_axis<V>(a, p[j]), row.t, c[j], sn[j]);
    if constexpr (NORM) load_weight<V>(s.weight, p[j], w[j], w[j] + V);
  }
  const float inv_dim = 1.f / static_cast<float>(a.dim);
  for (int turn = part; turn * a.groups < s.heads; turn += s.parts) {
    row = row_of(a, s, block, turn, g);
    float u[NCH][V], v[NCH][V], sq = 0.f;
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
#pragma unroll
      for (int i = 0; i < V; ++i) u[j][i] = v[j][i] = 0.f;
      if (row.live && p[j].here) load_row<T, V, NT>(s.x, row.t, row.h, p[j], u[j], v[j]);
      if constexpr (NORM) {
#pragma unroll
        for (int i = 0; i < V; ++i) sq = fmaf(u[j][i], u[j][i], fmaf(v[j][i], v[j][i], sq));
      }
    }
    if constexpr (NORM) {
      const float r = rsqrtf(group_sum(sq, a.lanes_log2) * inv_dim + a.eps);
#pragma unroll
      for (int j = 0; j < NCH; ++j) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          u[j][i] *= r * w[j][i];
          v[j][i] *= r * w[j][V + i];
        }
      }
    }
    int64_t to = row.t;
    bool store = row.live;
    if (key && a.slots && store) {
      to = a.slots[row.t];
      store = to >= 0 && to < a.slot_rows;
    }
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      turn_pairs<V, INTER, 1>(u[j], v[j], c[j], sn[j]);
      if (store && p[j].here) store_row<T, V, NT>(s.y, to, row.h, p[j], u[j], v[j]);
    }
  }
}

// The gradient.  Waves walk over their side's units; the sums for the weight's gradient stay in registers
// over the whole walk and are joined over the wave's groups, then over the workgroup, and written once:
// k_head_weights adds them up in a fixed order.
template <typename T, int V, int NCH, bool INTER, bool NORM, bool NT>
__global__ __launch_bounds__(kThreads) void k_head_backward(HeadArgs a) {
  extern __shared__ float joined[];  // [kWaves][dim]
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool key = static_cast<int>(blockIdx.x) >= a.q_blocks;
  const Side &s = a.side[key];
  const int64_t first = (static_cast<int64_t>(blockIdx.x) - (key ? a.q_blocks : 0)) * kWaves + wave;
  const int64_t step = static_cast<int64_t>(key ? gridDim.x - a.q_blocks : a.q_blocks) * kWaves;
  const int g = lane / a.lanes, l = lane - g * a.lanes;

  Place p[NCH];
  int axis[NCH];
  float w[NCH][2 * V], dw[NCH][2 * V];
#pragma unroll
  for (int j = 0; j < NCH; ++j) {
    p[j] = place<V, INTER>(a, l + a.lanes * j);
    axis[j] = shared_axis<V>(a, p[j]);
    if constexpr (NORM) {
      load_weight<V>(s.weight, p[j], w[j], w[j] + V);
#pragma unroll
      for (int i = 0; i < 2 * V; ++i) dw[j][i] = 0.f;
    }
  }
  const float inv_dim = 1.f / static_cast<float>(a.dim);
  for (int64_t unit = first; unit < s.units; unit += step) {
    const int64_t block = unit / s.parts;
    const int part = static_cast<int>(unit - block * s.parts);
    Row row = row_of(a, s, block, part, g);
    float c[NCH][V], sn[NCH][V];
#pragma unroll
    for (int j = 0; j < NCH; ++j) angles<V>(a, p[j], axis[j], row.t, c[j], sn[j]);
    for (int turn = part; turn * a.groups < s.heads; turn += s.parts) {
      row = row_of(a, s, block, turn, g);
      float u[NCH][V], v[NCH][V], xu[NCH][V], xv[NCH][V], sq = 0.f;
#pragma unroll
      for (int j = 0; j < NCH; ++j) {
#pragma unroll
        for (int i = 0; i < V; ++i) u[j][i] = v[j][i] = xu[j][i] = xv[j][i] = 0.f;
        if (row.live && p[j].here) {
          load_row<T, V, NT>(s.g, row.t, row.h, p[j], u[j], v[j]);
          if constexpr (NORM) load_row<T, V, NT>(s.x, row.t, row.h, p[j], xu[j], xv[j]);
        }
        turn_pairs<V, INTER, -1>(u[j], v[j], c[j], sn[j]);
        if constexpr (NORM) {
#pragma unroll
          for (int i = 0; i < V; ++i) sq = fmaf(xu[j][i], xu[j][i], fmaf(xv[j][i], xv[j][i], sq));
        }
      }
      if constexpr (NORM) {
        const float r = rsqrtf(group_sum(sq, a.lanes_log2) * inv_dim + a.eps);
        float dot = 0.f;
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
#pragma unroll
          for (int i = 0; i < V; ++i) {
            xu[j][i] *= r;
            xv[j][i] *= r;
            const float pu = u[j][i] * xu[j][i], pv = v[j][i] * xv[j][i];
            // a row that is not there has x = 0 and, where its angles are none, NaN for g: not 0 of it
            dw[j][i] += row.live ? pu : 0.f;
            dw[j][V + i] += row.live ? pv : 0.f;
            u[j][i] *= w[j][i];
            v[j][i] *= w[j][V + i];
            dot = fmaf(u[j][i], xu[j][i], fmaf(v[j][i], xv[j][i], dot));
          }
        }
        dot = group_sum(dot, a.lanes_log2) * inv_dim;
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
#pragma unroll
          for (int i = 0; i < V; ++i) {
            u[j][i] = r * fmaf(-xu[j][i], dot, u[j][i]);
            v[j][i] = r * fmaf(-xv[j][i], dot, v[j][i]);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < NCH; ++j)
        if (row.live && p[j].here) store_row<T, V, NT>(s.y, row.t, row.h, p[j], u[j], v[j]);
    }
  }
  if constexpr (NORM) {
    if (!a.partial) return;
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
#pragma unroll
      for (int i = 0; i < 2 * V; ++i) {
        for (int o = a.lanes; o < 64; o <<= 1) dw[j][i] += __shfl_xor(dw[j][i], o);
        const int e = i < V ? p[j].u + i : p[j].v + i - V;
        if (g == 0 && p[j].here && (i < V || p[j].both)) joined[wave * a.dim + e] = dw[j][i];
      }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.dim; e += kThreads) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) sum += joined[i * a.dim + e];
      a.partial[static_cast<int64_t>(blockIdx.x) * a.dim + e] = sum;
    }
  }
}

// Adds the workgroups' sums: 16 columns of the queries' or the keys' a workgroup, 64 lanes down each: 768
// sums in 12 dependent loads, 4.8 us.
__global__ __launch_bounds__(1024) void k_head_weights(const float *partial, int32_t q_blocks, int32_t blocks,
                                                       int32_t dim, float *dq, float *dk) {
  __shared__ float sums[64][17];
  const int col = threadIdx.x & 15, row = threadIdx.x >> 4;
  const int e = blockIdx.x * 16 + col;
  const bool key = blockIdx.y != 0;
  float sum = 0.f;
  if (e < dim) {
#pragma unroll 4
    for (int b = (key ? q_blocks : 0) + row; b < (key ? blocks : q_blocks); b += 64)
      sum += partial[static_cast<int64_t>(b) * dim + e];
  }
  sums[row][col] = sum;
  __syncthreads();
  float *to = key ? dk : dq;
  if (row != 0 || e >= dim || !to) return;
  float all = 0.f;
#pragma unroll 8
  for (int r = 0; r < 64; ++r) all += sums[r][col];
  to[e] = all;
}

// ---- host -------------------------------------------------------------------

struct Shape {
  int v, nch, lanes, lanes_log2, chunks;
};

bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// The widest piece (elements of a pair's side per lane) that every row allows: 8 or 4 where the
// head, its turned part and every pointer and stride divide by it, element by element otherwise.
Shape shape_of(const slowmo_head_config &c, const slowmo_heads *const *every, int n) {
  const size_t size = c.dtype == SLOWMO_BF16 ? 2 : 4;
  auto fits = [&](int v) {
    if (c.head_dim % (2 * v) || c.rotary_dim % (2 * v)) return false;
    if (c.rotary_dim && !aligned(c.table, 16)) return false;
    const size_t to = std::min<size_t>(16, v * size);
    for (int i = 0; i < n; ++i) {
      if (!every[i]->heads) continue;
      if (!aligned(every[i]->data, to) || every[i]->token_stride * size % to ||
          every[i]->head_stride * size % to)
        return false;
    }
    return true;
  };
  // Whether a lane of v pairs would have several axes: its angles are then fetched pair by pair, so that lanes of 4
  // pairs, of which fewer do, are taken (8 / 4, three axes: 30 000 tokens of 24 heads of 64, forward, 83 / 64 us;
  // 43 869 of 16 of 80, backward, 158 / 159, without the norm 130 / 108).
  auto mixes = [&](int v) {
    if (!c.pair_axis || c.n_axes < 2) return false;
    for (int i = 0; i < c.rotary_dim / 2; ++i)
      if (c.pair_axis[i] != c.pair_axis[i / v * v]) return true;
    return false;
  };
  Shape s{};
  s.v = fits(8) && !mixes(8) ? 8 : fits(4) ? 4 : 1;
  s.chunks = s.v > 1 ? c.head_dim / (2 * s.v) : (c.head_dim + 1) / 2;
  s.nch = s.v > 1 ? 1 : 4;
  while ((s.nch << s.lanes_log2) < s.chunks) ++s.lanes_log2;
  // the mean is exchanged among a power of two; without it lanes need not be left over
  s.lanes = c.norm ? 1 << s.lanes_log2 : (s.chunks + s.nch - 1) / s.nch;
  return s;
}

const char *check(const slowmo_head_config *c, int64_t tokens) {
  if (!c) return "cfg is NULL";
  if (c->dtype != SLOWMO_F32 && c->dtype != SLOWMO_BF16) return "unknown dtype";
  if (c->head_dim < 1 || c->head_dim > SLOWMO_MAX_HEAD_DIM)
    return "head_dim must be in 1..SLOWMO_MAX_HEAD_DIM";
  if (c->rotary_dim < 0 || c->rotary_dim > c->head_dim || c->rotary_dim % 2)
    return "rotary_dim must be even and in 0..head_dim";
  if (c->interleaved != 0 && c->interleaved != 1) return "interleaved must be 0 or 1";
  if (c->norm != 0 && c->norm != 1) return "norm must be 0 or 1";
  if (!c->norm && (c->q_weight || c->k_weight)) return "without the norm there are no weights";
  if (!(std::isfinite(c->eps) && c->eps >= 0.f)) return "eps must be finite and >= 0";
  if (c->n_axes < 1 || c->n_axes > SLOWMO_MAX_AXES) return "n_axes must be in 1..SLOWMO_MAX_AXES";
  if (tokens < 0 || tokens > (int64_t(1) << 31)) return "tokens must be in 0..2^31";
  if (c->rotary_dim) {
    if (c->pair_axis)
      for (int i = 0; i < c->rotary_dim / 2; ++i)
        if (c->pair_axis[i] >= c->n_axes) return "a pair_axis entry is not an axis";
    if (c->table_rows < 0 || c->table_rows > (int64_t(1) << 40)) return "table_rows must be in 0..2^40";
    if (tokens && c->table_rows && !c->table) return "table is NULL";
    if (tokens && !c->positions) return "positions is NULL";
    if (c->position_stride < 0 || c->position_stride > (int64_t(1) << 40) ||
        (c->n_axes > 1 && c->position_stride && c->position_stride < tokens))
      return "position_stride must be 0 or in tokens..2^40";
  }
  return nullptr;
}

const char *check_heads(const slowmo_heads *h, int64_t tokens) {
  if (!h) return "a slowmo_heads is NULL";
  if (h->heads < 0 || h->heads > (1 << 20)) return "heads must be in 0..2^20";
  if (h->token_stride < 0 || h->head_stride < 0 || h->token_stride > (int64_t(1) << 40) ||
      h->head_stride > (int64_t(1) << 40))
    return "strides must be in 0..2^40";
  // so that no offset or extent passes 64 bits
  if (static_cast<double>(h->token_stride) * static_cast<double>(std::max<int64_t>(tokens - 1, 0)) +
          static_cast<double>(h->head_stride) * std::max(h->heads - 1, 0) > std::exp2(50.))
    return "an array reaches past 2^50 elements";
  if (h->heads && tokens && !h->data) return "data is NULL";
  return nullptr;
}

// Whether rows or heads of an array that is written fall on one another.
bool folds(const slowmo_heads &h, int64_t tokens, int64_t dim) {
  if (!h.heads || tokens == 0) return false;
  const int64_t across = h.head_stride * (h.heads - 1) + dim, down = h.token_stride * (tokens - 1) + dim;
  const bool heads_fold = h.heads > 1 && h.head_stride < dim;
  const bool tokens_fold = tokens > 1 && h.token_stride < dim;
  if (heads_fold || tokens_fold) return true;
  // rows apart from one another either way round: [token][head] or [head][token]
  return tokens > 1 && h.heads > 1 && h.token_stride < across && h.head_stride < down;
}

struct Extent {
  uintptr_t lo, hi;
};
Extent extent(const slowmo_heads &h, int64_t tokens, const slowmo_head_config &c) {
  const uintptr_t lo = reinterpret_cast<uintptr_t>(h.data), size = c.dtype == SLOWMO_BF16 ? 2 : 4;
  if (!h.heads || !tokens) return {lo, lo};
  return {lo, lo + size * static_cast<uintptr_t>(h.token_stride * (tokens - 1) +
                                                 h.head_stride * (h.heads - 1) + c.head_dim)};
}

bool same_rows(const slowmo_heads &a, const slowmo_heads &b) {
  return a.data == b.data && a.token_stride == b.token_stride && a.head_stride == b.head_stride;
}

// Whether two arrays share an element: interleaved ones (queries beside keys) do not, if they
// have the same strides and the distance between them keeps their heads apart.
bool overlap(const slowmo_heads &a, int64_t ta, const slowmo_heads &b, int64_t tb,
             const slowmo_head_config &c) {
  const Extent x = extent(a, ta, c), y = extent(b, tb, c);
  if (x.lo == x.hi || y.lo == y.hi || x.hi <= y.lo || y.hi <= x.lo) return false;
  if (a.token_stride == b.token_stride && a.token_stride > 0) {
    const int64_t size = c.dtype == SLOWMO_BF16 ? 2 : 4;
    const int64_t wa = a.head_stride * (a.heads - 1) + c.head_dim,
                  wb = b.head_stride * (b.heads - 1) + c.head_dim;
    int64_t d = (static_cast<int64_t>(y.lo) - static_cast<int64_t>(x.lo)) / size % a.token_stride;
    if (d < 0) d += a.token_stride;
    // within one token's stretch a lies at 0..wa, b at d..d + wb
    if (wa <= a.token_stride && wa <= d && d + wb <= a.token_stride) return false;
  }
  return true;
}

Rows rows_of(const slowmo_heads &h) { return {h.data, h.token_stride, h.head_stride}; }

void fill(HeadArgs &a, const slowmo_head_config &c, int64_t tokens, const slowmo_heads &q,
          const slowmo_heads &k, const Shape &s) {
  a.tokens = tokens;
  a.table = c.table;
  a.positions = c.positions;
  a.table_rows = c.rotary_dim ? c.table_rows : 0;
  a.position_stride = c.position_stride;
  a.dim = c.head_dim;
  a.rot = c.rotary_dim;
  a.chunks = s.chunks;
  a.lanes = s.lanes;
  a.lanes_log2 = s.lanes_log2;
  a.groups = 64 / s.lanes;
  a.axes = c.n_axes;
  a.eps = c.eps;
  if (c.pair_axis)
    for (int i = 0; i < c.rotary_dim / 2; ++i)
      a.pair_axis[i >> 4] |= static_cast<uint32_t>(c.pair_axis[i]) << (2 * (i & 15));
  for (int key = 0; key < 2; ++key) {
    Side &d = a.side[key];
    const slowmo_heads &h = key ? k : q;
    d.x = rows_of(h);
    d.weight = key ? c.k_weight : c.q_weight;
    d.heads = h.heads;
    d.together = std::max(1, h.heads ? a.groups / h.heads : 1);
    // few tokens: their heads go to several waves, down to one turn each
    const int64_t blocks = (tokens + d.together - 1) / d.together, turns = (h.heads + a.groups - 1) / a.groups;
    d.parts = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(turns, kFill / std::max<int64_t>(blocks, 1))));
    d.units = h.heads ? blocks * d.parts : 0;
  }
}

// Workgroups of a side of the backward kernel: enough to fill the card, no more than there is work.
int32_t backward_blocks(int64_t units, double share) {
  return static_cast<int32_t>(std::min<int64_t>((units + kWaves - 1) / kWaves,
                                                std::max<int64_t>(1, static_cast<int64_t>(kWalks * share))));
}

template <typename F>
void by_bool(bool b, F &&f) {
  if (b)
    f(std::true_type{});
  else
    f(std::false_type{});
}

// Whether rows are loaded and stored past the caches: where a pass moves several times what they hold.
// Time past them over time through them: 70 MB 1.43, 220 MB 1.01, 500 MB 1.08, 1 GB 0.92.
bool streams(const HeadArgs &a, const slowmo_head_config &c, int passes) {
  const int64_t bytes = a.tokens * (a.side[0].heads + a.side[1].heads) * a.dim * (c.dtype == SLOWMO_BF16 ? 2 : 4);
  return passes * bytes >= (int64_t(768) << 20);
}

template <typename F>
void dispatch(const slowmo_head_config &c, const Shape &s, bool streaming, F &&f) {
  by_bool(c.interleaved, [&](auto inter) {
    by_bool(c.norm, [&](auto norm) {
      auto typed = [&](auto zero) {
        using T = decltype(zero);
        std::integral_constant<int, 1> one;
        if (s.v == 8)
          by_bool(streaming, [&](auto nt) { f(zero, std::integral_constant<int, 8>{}, one, inter, norm, nt); });
        else if (s.v == 4)
          by_bool(streaming, [&](auto nt) { f(zero, std::integral_constant<int, 4>{}, one, inter, norm, nt); });
        else
          f(T{}, one, std::integral_constant<int, 4>{}, inter, norm, std::false_type{});
      };
      if (c.dtype == SLOWMO_BF16)
        typed(uint16_t{});
      else
        typed(float{});
    });
  });
}

}  // namespace
}  // namespace slowmo

using namespace slowmo;

extern "C" {

slowmo_status slowmo_head_norm_rotary(const slowmo_head_config *cfg, int64_t tokens,
                                      const slowmo_heads *q, const slowmo_heads *k,
                                      const slowmo_heads *q_out, const slowmo_heads *k_out,
                                      const int64_t *k_slots, int64_t k_rows, void *stream) {
  return walled([&]() -> slowmo_status {
    if (const char *bad = check(cfg, tokens)) return fail_thread(SLOWMO_ERR_ARG, bad);
    const slowmo_heads *every[] = {q, k, q_out, k_out};
    const size_t size = cfg->dtype == SLOWMO_BF16 ? 2 : 4;
    if (k_slots && (k_rows < 0 || k_rows > (int64_t(1) << 40)))
      return fail_thread(SLOWMO_ERR_ARG, "k_rows must be in 0..2^40");
    const int64_t out_rows = k_slots ? k_rows : tokens;
    for (int i = 0; i < 4; ++i) {
      if (const char *bad = check_heads(every[i], i == 3 ? out_rows : tokens))
        return fail_thread(SLOWMO_ERR_ARG, bad);
      if (!aligned(every[i]->data, size))
        return fail_thread(SLOWMO_ERR_ALIGN, "data is not aligned to its element size");
    }
    if (q->heads != q_out->heads || k->heads != k_out->heads)
      return fail_thread(SLOWMO_ERR_ARG, "an output has another number of heads than its input");
    for (const float *w : {cfg->q_weight, cfg->k_weight, cfg->table})
      if (!aligned(w, 4)) return fail_thread(SLOWMO_ERR_ALIGN, "a weight or the table is not 4-byte aligned");
    if (!aligned(cfg->positions, 8) || !aligned(k_slots, 8))
      return fail_thread(SLOWMO_ERR_ALIGN, "positions and k_slots must be 8-byte aligned");
    if (folds(*q_out, tokens, cfg->head_dim) || folds(*k_out, out_rows, cfg->head_dim))
      return fail_thread(SLOWMO_ERR_ARG, "rows of an output overlap each other");
    if (overlap(*q_out, tokens, *k_out, out_rows, *cfg) || overlap(*q_out, tokens, *k, tokens, *cfg) ||
        overlap(*k_out, out_rows, *q, tokens, *cfg) ||
        (overlap(*q_out, tokens, *q, tokens, *cfg) && !same_rows(*q_out, *q)) ||
        (overlap(*k_out, out_rows, *k, tokens, *cfg) && (k_slots || !same_rows(*k_out, *k))))
      return fail_thread(SLOWMO_ERR_ARG, "an output overlaps an input or the other output");
    if (!tokens || !(q->heads + k->heads)) return SLOWMO_OK;
    const Shape s = shape_of(*cfg, every, 4);
    HeadArgs a{};
    fill(a, *cfg, tokens, *q, *k, s);
    a.side[0].y = rows_of(*q_out);
    a.side[1].y = rows_of(*k_out);
    a.slots = k_slots;
    a.slot_rows = k_rows;
    const int64_t units = a.side[0].units + a.side[1].units;
    hipError_t e = hipSuccess;
    dispatch(*cfg, s, streams(a, *cfg, 2), [&](auto zero, auto v, auto nch, auto inter, auto norm, auto nt) {
      for (; a.first < units && e == hipSuccess; a.first += static_cast<int64_t>(kMostBlocks) * kWaves) {
        const int64_t blocks = std::min<int64_t>(kMostBlocks, (units - a.first + kWaves - 1) / kWaves);
        k_head_forward<decltype(zero), v(), nch(), inter(), norm(), nt()>
            <<<static_cast<uint32_t>(blocks), kThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
        e = hipGetLastError();
      }
    });
    return e == hipSuccess ? SLOWMO_OK : fail_thread_hip(e, "slowmo_head_norm_rotary");
  });
}

size_t slowmo_head_backward_bytes(const slowmo_head_config *cfg, int64_t tokens, int32_t q_heads,
                                  int32_t k_heads) {
  if (!cfg || !cfg->norm || cfg->head_dim < 1 || cfg->head_dim > SLOWMO_MAX_HEAD_DIM || tokens <= 0 ||
      q_heads < 0 || k_heads < 0 || q_heads > (1 << 20) || k_heads > (1 << 20))
    return 0;
  // the number of workgroups depends on the pieces, so on alignment: the most there can be
  return static_cast<size_t>(std::min<int64_t>(kWalks + 2, tokens * (static_cast<int64_t>(q_heads) + k_heads) + 2)) *
         cfg->head_dim * sizeof(float);
}

slowmo_status slowmo_head_norm_rotary_backward(const slowmo_head_config *cfg, int64_t tokens,
                                               const slowmo_heads *gq, const slowmo_heads *gk,
                                               const slowmo_heads *q, const slowmo_heads *k,
                                               const slowmo_heads *dq, const slowmo_heads *dk,
                                               float *dq_weight, float *dk_weight, void *workspace,
                                               size_t workspace_bytes, void *stream) {
  return walled([&]() -> slowmo_status {
    if (const char *bad = check(cfg, tokens)) return fail_thread(SLOWMO_ERR_ARG, bad);
    const slowmo_heads *every[] = {gq, gk, dq, dk, q, k};
    const size_t size = cfg->dtype == SLOWMO_BF16 ? 2 : 4;
    const int used = cfg->norm ? 6 : 4;  // without the norm the inputs are not read
    for (int i = 0; i < 6; ++i) {
      if (const char *bad = check_heads(every[i], i < used ? tokens : 0))
        return fail_thread(SLOWMO_ERR_ARG, bad);
      if (!aligned(every[i]->data, size))
        return fail_thread(SLOWMO_ERR_ALIGN, "data is not aligned to its element size");
    }
    if (gq->heads != q->heads || dq->heads != q->heads || gk->heads != k->heads || dk->heads != k->heads)
      return fail_thread(SLOWMO_ERR_ARG, "a gradient has another number of heads than its input");
    for (const float *w : {cfg->q_weight, cfg->k_weight, cfg->table,
                           static_cast<const float *>(dq_weight), static_cast<const float *>(dk_weight)})
      if (!aligned(w, 4)) return fail_thread(SLOWMO_ERR_ALIGN, "a weight or the table is not 4-byte aligned");
    if (!aligned(cfg->positions, 8))
      return fail_thread(SLOWMO_ERR_ALIGN, "positions must be 8-byte aligned");
    if (!cfg->norm && (dq_weight || dk_weight))
      return fail_thread(SLOWMO_ERR_ARG, "without the norm there is no weight gradient");
    if (folds(*dq, tokens, cfg->head_dim) || folds(*dk, tokens, cfg->head_dim))
      return fail_thread(SLOWMO_ERR_ARG, "rows of an output overlap each other");
    const slowmo_heads *outs[] = {dq, dk};
    for (int o = 0; o < 2; ++o) {
      if (overlap(*outs[o], tokens, *outs[1 - o], tokens, *cfg))
        return fail_thread(SLOWMO_ERR_ARG, "the outputs overlap");
      for (int i = 0; i < used; ++i) {
        if (i == 2 || i == 3) continue;
        const bool own_gradient = i == o && same_rows(*outs[o], *every[i]);
        if (!own_gradient && overlap(*outs[o], tokens, *every[i], tokens, *cfg))
          return fail_thread(SLOWMO_ERR_ARG, "an output overlaps an input");
      }
    }
    const Shape s = shape_of(*cfg, every, used);
    HeadArgs a{};
    fill(a, *cfg, tokens, *q, *k, s);
    a.side[0].g = rows_of(*gq);
    a.side[1].g = rows_of(*gk);
    a.side[0].y = rows_of(*dq);
    a.side[1].y = rows_of(*dk);
    const bool weights = dq_weight || dk_weight;
    const double heads = std::max(1, q->heads + k->heads);
    a.q_blocks = backward_blocks(a.side[0].units, q->heads / heads);
    const int32_t blocks = a.q_blocks + backward_blocks(a.side[1].units, k->heads / heads);
    if (weights && blocks) {
      if (!workspace) return fail_thread(SLOWMO_ERR_ARG, "workspace is NULL");
      if (!aligned(workspace, 16)) return fail_thread(SLOWMO_ERR_ALIGN, "workspace must be 16-byte aligned");
      if (workspace_bytes < static_cast<size_t>(blocks) * a.dim * sizeof(float))
        return fail_thread(SLOWMO_ERR_NOMEM, "workspace is smaller than slowmo_head_backward_bytes()");
      a.partial = static_cast<float *>(workspace);
    }
    hipError_t e = hipSuccess;
    if (blocks) {
      dispatch(*cfg, s, streams(a, *cfg, cfg->norm ? 3 : 2), [&](auto zero, auto v, auto nch, auto inter, auto norm, auto nt) {
        const uint32_t lds = norm() ? kWaves * a.dim * sizeof(float) : 0;
        k_head_backward<decltype(zero), v(), nch(), inter(), norm(), nt()>
            <<<blocks, kThreads, lds, static_cast<hipStream_t>(stream)>>>(a);
        e = hipGetLastError();
      });
      if (e != hipSuccess) return fail_thread_hip(e, "slowmo_head_norm_rotary_backward");
    }
    if (weights) {
      k_head_weights<<<dim3((a.dim + 15) / 16, 2), 1024, 0, static_cast<hipStream_t>(stream)>>>(
          a.partial, a.q_blocks, blocks, a.dim, dq_weight, dk_weight);
      e = hipGetLastError();
      if (e != hipSuccess)
        return fail_thread_hip(e, "slowmo_head_norm_rotary_backward (gradients of q and k are written, "
                                  "those of the weights are not)");
    }
    return SLOWMO_OK;
  });
}

}  // extern "C"
