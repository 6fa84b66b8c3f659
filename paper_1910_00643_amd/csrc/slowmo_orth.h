// Tables and launches that the orthogonalising call's host side (slowmo_orth.cpp) and kernels
// (slowmo_orth.hip) share.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace slowmo {
namespace orth {

// Halves are stored times a power of two that keeps them away from the subnormal range: X and A are
// below 8 in size (their spectral norms are near 1), b A + c A A below 32.
constexpr float kScaleX = 8192.f, kScaleA = 8192.f, kScaleP = 2048.f;

constexpr int kPatch = 64;       // side of an elementwise kernel's patch
constexpr int kInline = 64;      // matrices whose addresses travel with one launch

// Matrices that one workgroup takes from load to store.
constexpr int kTinySide = 32, kTinyElements = 4096, kTinyThreads = 512;

// One matrix.  n <= k; X is n x k; np, kp: sides padded to whole tiles.  Offsets count halves from
// the start of the arena; lo: the values' next 11 bits.
struct Matrix {
  int64_t x[2], a, p;
  int64_t x_lo[2], a_lo, p_lo;  // x_lo[1], a_lo, p_lo only where products are split
  int64_t ld;
  int32_t n, k, np, kp;
  int32_t tall;                        // the caller's matrix is k x n
  float scale;
  int32_t first_patch, patches;        // its patches in the list of them
};

// One workgroup's share of a phase.
struct Item {
  int32_t matrix, i, j, pad;
};

struct Addresses {
  const void *in;
  float *momentum;
  void *out;
};

// The addresses of up to kInline matrices, as a kernel's argument.
struct Few {
  Addresses at[kInline];
};

struct Call {
  const Matrix *matrices;
  Addresses *addresses;
  double *squares;     // one sum per patch
  float *inverse;      // 1 / (|U|_F + eps) per matrix, NaN where the norm is not finite
  _Float16 *arena;
  float eps, mu;
  int32_t in_bf16, out_bf16, momentum, nesterov;
};

enum Phase { kGram = 0, kPolynomial = 1, kUpdate = 2 };

struct Step {
  float a, b, c;
  int32_t from;        // which of x[2] is read
  int32_t last;
  int32_t carry;       // a X enters from hi + lo, and P is b A + c A A alone; else P has a on its diagonal
  int32_t carry_next;  // the next step needs lo
};

struct Steps {
  float abc[16][3];
  int32_t count;
};

hipError_t launch_tiny(const Call &c, const Steps &steps, const int32_t *list, int32_t count, hipStream_t s);
hipError_t launch_addresses(const Call &c, const Few &few, int32_t first, int32_t count, hipStream_t s);
hipError_t launch_squares(const Call &c, const Item *items, int32_t count, hipStream_t s);
hipError_t launch_norms(const Call &c, int32_t matrices, hipStream_t s);
hipError_t launch_load(const Call &c, const Item *items, int32_t count, hipStream_t s);
hipError_t prepare_products(int tile, bool split);
hipError_t launch_products(const Call &c, int tile, Phase phase, const Step &step, const Item *items,
                           int32_t count, bool split, hipStream_t s);

}  // namespace orth
}  // namespace slowmo
