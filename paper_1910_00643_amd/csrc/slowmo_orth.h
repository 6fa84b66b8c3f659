// Tables and launches that the orthogonalising call's host side (slowmo_orth.cpp) and kernels
// (slowmo_orth.hip) share.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace slowmo {
namespace orth {

constexpr int kDeep = 32;        // elements of the summed side in a step of a product
constexpr int kPatch = 64;       // side of an elementwise kernel's patch; kPatches of them in a row per workgroup
constexpr int kPatches = 4;
constexpr int kInline = 64;      // matrices whose addresses travel with one launch
constexpr int kMostSums = 1024;  // workgroups that share a matrix's sum of squares
constexpr int kSquares = 4;      // n x n buffers of a matrix: A, P, W, Q (A, P where steps go one by one)

// Kinds of tiles: 128 x 128, 256 x 256, and, for P X, 128 rows of 256.
enum Kind { kSmall = 0, kLarge = 1, kWide = 2, kKinds = 3 };
constexpr int32_t kRowsOf[kKinds] = {128, 256, 128}, kColsOf[kKinds] = {128, 256, 256};
constexpr int32_t kSlotsOf[kKinds] = {768, 256, 512};  // workgroups that run at a time

// Matrices that one workgroup takes from load to store.
constexpr int kTinySide = 32, kTinyElements = 4096, kTinyThreads = 512;
constexpr int64_t kTinyWork = int64_t(1) << 18;  // most of n n k, where the matrix is longer than kTinyElements

// X is held as halves times this power of two: its elements are below 8 in size (checked on the
// coefficients), and what of them is subnormal as a half is below 2^-27.
constexpr int kPowerX = 13;
constexpr float kScaleX = 1 << kPowerX;

// A list of small matrices alone goes by one workgroup each too: n up to 128 and k up to 256 for products
// of halves, n up to 64 for those of pairs of halves (X, A and P fill shared memory).
constexpr int kSmallSide = 128, kSmallSideSplit = 64, kSmallLength = 256;

// One matrix.  n <= k; X is n x k; np, kp: sides padded to whole tiles.  X and the n x n buffers lie in
// panels of kDeep columns, [column / kDeep][row][column mod kDeep].  From `at` on (halves from the start
// of the arena): X, the X it is replaced by, X's lower halves (the values' next 11 bits), the n x n buffers;
// where products are split, the other X's and the n x n buffers' lower halves after that.
struct Matrix {
  int64_t at, ld;
  int32_t n, k, np, kp;
  int32_t tall, tiny;                    // the caller's matrix is k x n; it is k_tiny's
  float scale;
  int32_t first_sum, sums;               // its partial sums of squares
};

struct Places {
  int64_t wide, square, squares;
  __host__ __device__ Places(int64_t np, int64_t kp, int64_t buffers)
      : wide(np * kp), square(np * np), squares(buffers) {}
  __host__ __device__ int64_t x(int which) const { return which ? wide : 0; }
  __host__ __device__ int64_t x_lo(int which) const { return which ? 3 * wide + squares * square : 2 * wide; }
  __host__ __device__ int64_t buffer(int which) const { return 3 * wide + which * square; }
  __host__ __device__ int64_t buffer_lo(int which) const { return 4 * wide + (squares + which) * square; }
  __host__ __device__ int64_t total(bool split) const { return split ? buffer_lo(static_cast<int>(squares)) : buffer(static_cast<int>(squares)); }
};

// A workgroup's share of an elementwise phase: of a sum of squares (i of `j`), or the patches from
// (i, j) on.
struct Item {
  int32_t matrix, i, j, pad;
};

// A workgroup's share of a product: steps first..first + count - 1 of tile (i, j) (of a symmetric product's
// diagonal, i = j: in twos); where a tile is in
// `pieces` > 1 shares, `slot` counts the places of their partial sums and `ticket` its counter.  What it
// needs of the matrix comes along: one load in front of the first of its data.
struct Tile {
  int64_t at;                            // the matrix's first half in the arena
  int32_t np, kp;
  int32_t i, j, first, count;
  int32_t piece, pieces, slot, ticket;
  int32_t matrix, pad[3];
};
static_assert(sizeof(Tile) == 64, "one cache line's half");

struct Addresses {
  const void *in;
  float *momentum;
  void *out;
};

// The addresses of up to kInline matrices, as a kernel's argument.
struct Few {
  Addresses at[kInline];
};

// Floats of a matrix in Call::scales: one for X X^T of each step, one for each update of X.
constexpr int kScales = 2 * 16;

struct Call {
  const Matrix *matrices;
  Addresses *addresses;
  double *sums;
  _Float16 *arena;
  float *partial;        // partial sums of tiles
  uint32_t *tickets;     // zero between calls
  float eps, mu;
  float *scales;         // [matrix][kScales]: what a product of X is times for the powers of two that X is held
                         // times while it is small and, where `exact`, for the rest of 1 / (|U| + eps) at the first step
  const float *abc;      // the steps' coefficients
  int32_t steps;
  int32_t in_bf16, out_bf16, momentum, nesterov;
  int32_t exact;         // X_0 is held as U times a power of two: 8 bits of bf16 fit a half whole, and no lower
                         // halves are needed
  int32_t buffers;       // n x n buffers of a matrix
};

// (`first_step`: of X_0, which Call::exact may have held without its factor; `scale`: the place in Call::scales,
// -1: none.)
// out = alpha * left * right (+ beta * first) (+ gamma * second) (+ delta on the diagonal), symmetric;
// buffers are numbered, left = -1: X X^T.  The factors hold the buffers' powers of two.
struct Symmetric {
  int32_t from, left, right, first, second, out;  // first, second: -1: none
  float alpha, beta, gamma, delta;
  int32_t first_step, scale;
};

// x[1 - from] = alpha * buffer[by] x[from] (+ beta * (hi + lo of x[from])); or the caller's result.
struct Update {
  int32_t from, by, carry, carry_next, last;
  float alpha, beta;
  int32_t first_step, scale;
};

struct Steps {
  float abc[16][3];
  float a_power[16], p_power[16];  // the powers of two that A and P are held times in step by step products
  int32_t carry[16];
  int32_t count;
};

hipError_t launch_tiny(const Call &c, const Steps &steps, const int32_t *list, int32_t count, hipStream_t s);
// Matrices first..first + count - 1, all of them small or tiny (which are left out).
// side: the longest of their shorter sides.
hipError_t launch_small(const Call &c, const Steps &steps, const Few &few, int32_t first, int32_t count, int32_t side,
                        bool split, hipStream_t s);
hipError_t prepare_small();
hipError_t launch_addresses(const Call &c, const Few &few, int32_t first, int32_t count, hipStream_t s);
hipError_t launch_sums(const Call &c, const Item *items, int32_t count, hipStream_t s);
hipError_t launch_load(const Call &c, const Item *items, int32_t count, hipStream_t s);
hipError_t prepare_products(bool split);
hipError_t launch_symmetric(const Call &c, int kind, const Symmetric &p, const Tile *tiles, int32_t count,
                            bool split, hipStream_t s);
hipError_t launch_update(const Call &c, int kind, const Update &p, const Tile *tiles, int32_t count, bool split,
                         hipStream_t s);

}  // namespace orth
}  // namespace slowmo
