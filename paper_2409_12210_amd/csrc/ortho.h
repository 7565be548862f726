// What the orthogonalised update's entry point and its kernels share.
#pragma once
#include <math.h>

#include "common.h"

namespace modse_ortho {

constexpr int MAX_STEPS = 32, MAX_MATS = 4096;
constexpr int PAD = 128;  // rows and columns of what is stored are padded to this with zeros: no kernel has edges to look at

// the largest |a + b s^2 + c s^4| for 0 <= s <= top
inline double ratio_bound(double a, double b, double c, double top) {
  auto at = [=](double u) { return fabs(a + (b + c * u) * u); };
  double most = at(0) > at(top * top) ? at(0) : at(top * top);
  const double u = c != 0 ? -b / (2 * c) : 0;
  if (u > 0 && u < top * top && at(u) > most) most = at(u);
  return most;
}

// Square matrices of a matrix's workspace: A and the next A of a group of steps, R = b A + c A A likewise, Q the product of the
// steps' polynomials so far (twice), S = a A + R A on the way to the next A.
enum Slot { SLOT_A, SLOT_R, SLOT_A2, SLOT_R2, SLOT_Q, SLOT_S, N_SLOTS };

// the largest |a s + b s^3 + c s^5| for 0 <= s <= top
__host__ __device__ inline double quintic_bound(double a, double b, double c, double top) {
  auto at = [=](double u) { return fabs((a + (b + c * u) * u) * sqrt(u)); };
  double most = at(top * top);
  auto candidate = [&](double u) {
    if (u > 0 && u < top * top && at(u) > most) most = at(u);
  };
  // zeros of the derivative: a + 3 b u + 5 c u^2 = 0, u = s^2
  if (c != 0) {
    const double disc = 9 * b * b - 20 * a * c;
    if (disc >= 0) {
      candidate((-3 * b + sqrt(disc)) / (10 * c));
      candidate((-3 * b - sqrt(disc)) / (10 * c));
    }
  } else if (b != 0) {
    candidate(-a / (3 * b));
  }
  return most;
}

// One matrix of the set, in device memory.  Tile lists hold copies, so that a workgroup knows all it needs after one load.
struct alignas(128) Mat {
  int32_t which;  // its place in the set
  int32_t mt, nt; // in a tile list: the tile's row and column
  const float* G;
  void* U;
  char* X[2];     // [mp, np] stored pairs
  char* slot;     // matrices [mp, mp] of them
  int32_t rows, cols;
  int32_t m, n;   // the shorter and the longer side: a tall matrix is stored transposed
  int32_t mp, np;
  int32_t square_tile, update_tile;  // its first tiles in the launches' lists
  int32_t part, parts;               // its partial sums of squares
};
// of a product, and of the matrices that are added to it
struct Factors {
  float product, first, second;
};

}  // namespace modse_ortho

struct OrthoLayout {
  size_t mats, bounds, factors, squares, sums, square_list, update_list, data, total;
  int32_t square_tiles, update_tiles, parts;
  int32_t tile;
  int32_t slots;  // squares of a matrix, from SLOT_A on
  int32_t group[modse_ortho::MAX_STEPS];  // steps of every group of them
  int32_t n_groups;
  double most[modse_ortho::MAX_STEPS + 1];  // what the first steps make of singular values up to 1, at most
};
// coeffs == null: a layout that serves any steps
modse_status ortho_layout(const modse_matrix_set* set, const float* coeffs, int steps, OrthoLayout& w);
hipError_t launch_orthogonalize(const modse_matrix_set* set, const OrthoLayout& w, const float* coeffs, float eps, char* ws, hipStream_t s);
