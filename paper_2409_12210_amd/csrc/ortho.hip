// The orthogonalised update: X = G / (|G| + eps), then X <- a X + (b A + c A^2) X with A = X X^T, for every matrix of a set.
//
// All of it is matrix products: for an m x n matrix (m the shorter side; a tall one is stored transposed) X X^T, A A and R X.
// The iteration enlarges small singular values by up to a per step, and with them the rounding errors of the large ones, so the
// products need float32 precision.  They get it from the 16-bit matrix instructions, whose rate is sixteen times that of the
// float32 ones: a value is stored as hi + lo, two float16 numbers with 11 bits each, times a power of two that keeps the
// largest value that the matrix can have (a bound on its singular values) below 2^15, and a product is hi hi + hi lo + lo hi,
// summed in float32.  What is left out, lo lo, is 2^-24 of the product in the mean, as a float32 rounding is: errors against float64
// as those of float32 products (1.0e-6 both after five single steps of 512 x 1024).
//
// Storage: rows of blocks of 32 values, 64 bytes of hi and then 64 of lo, so that a cache line feeds one step of a product.
//
// Squares are symmetric: only tiles on and below the diagonal are computed.  With tiles of 128 they alone are stored, and a panel that
// reaches beyond the diagonal is read as columns there; small tiles are written twice.
//
// Groups of steps.  p(A) X for several steps in a row needs X only at its ends: with R_i = b A_i + c A_i^2 and P_i = a_i I + R_i,
// A_(i+1) = P_i A_i P_i and X_g = P_(g-1) ... P_0 X, all of whose factors are m x m, symmetric and commute.  In units of m^3
// (n = r m, squares at half price) a group of g steps costs 3 r + 4 g - 3 where single steps cost g (3 r + 1).  What a rounding
// puts into A grows by up to a^2 in every A_(i+1), so groups are short: F32_ROUNDINGS.
#include <algorithm>

#include "gemm_bf16_util.h"
#include "ops.h"
#include "ortho.h"

namespace {
using namespace modse_ortho;
using modse_gemm::dma_b128_s;
using modse_gemm::lds_address;
using modse_gemm::uniform_int;
using modse_gemm::uniform_ptr;

typedef _Float16 half_t;
typedef half_t half4 __attribute__((ext_vector_type(4)));
typedef half_t half8 __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------- table, norms, factors
struct MatArg {
  const float* G;
  void* U;
  int64_t data;  // offset of its buffers
  int32_t rows, cols, square_tile, update_tile, part, parts;
};
constexpr int MATS_PER_LAUNCH = 64;
struct MatArgs {
  MatArg mat[MATS_PER_LAUNCH];
  Mat* table;
  char* data;
  int32_t first, count;
};
__host__ __device__ inline int padded(int v) { return (v + PAD - 1) / PAD * PAD; }

constexpr int PART = 1 << 13;  // elements of a partial sum of squares
// The table, and sums of squares in float64 (no overflow, and the order of the additions is of no account).  blockIdx.y: matrix.
// Bound by memory: a full layer's 277 M values, 1.1 GB, take 188 us, 5.9 TB/s.
__global__ __launch_bounds__(256) void ortho_squares_kernel(MatArgs a, double* __restrict__ sums) {
  __shared__ double s[4];
  const MatArg& t = a.mat[blockIdx.y];
  const int parts = t.parts, part0 = t.part;
  const int64_t n = (int64_t)t.rows * t.cols;
  const float* const G = t.G;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    Mat m;
    m.which = a.first + blockIdx.y;
    m.mt = m.nt = 0;
    m.G = t.G;
    m.U = t.U;
    m.rows = t.rows;
    m.cols = t.cols;
    m.m = min(t.rows, t.cols);
    m.n = max(t.rows, t.cols);
    m.mp = padded(m.m);
    m.np = padded(m.n);
    const size_t x = (size_t)m.mp * m.np * 4;
    m.X[0] = a.data + t.data;
    m.X[1] = m.X[0] + x;
    m.slot = m.X[1] + x;
    m.square_tile = t.square_tile;
    m.update_tile = t.update_tile;
    m.part = t.part;
    m.parts = t.parts;
    a.table[m.which] = m;
  }
  for (int part = blockIdx.x; part < parts; part += gridDim.x) {
    const int64_t end = min(n, ((int64_t)part + 1) * PART);
    double v = 0;
    const int64_t first = (int64_t)part * PART + threadIdx.x * 4;
    Vec<float> g[PART / 1024];
#pragma unroll
    for (int i = 0; i < PART / 1024; ++i) g[i].load(G + first + i * 1024, (int)(end - first - i * 1024), 0.f);
#pragma unroll
    for (int i = 0; i < PART / 1024; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) v += (double)g[i][j] * g[i][j];
    for (int b = 32; b; b >>= 1) v += __shfl_xor(v, b, 64);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0) sums[part0 + part] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
  }
}

// the power of two that takes what is at most `bound` to at most 2^15 (twice that in error)
__device__ inline double store_scale(double bound) {
  int e = 0;
  if (bound > 0 && bound < 1e300) frexp(bound, &e);
  return ldexp(1.0, 15 - e);
}

// What is known of a matrix on its way through the steps: bounds of singular values, and the powers of two that go with what is stored.
struct Bound {
  double x, q;                    // of the present X (in a group: of what X would be), of Q
  double in_x, in_a, in_r, in_q;  // X, A, R, Q as stored
  float out;                      // 1 / in_x, of the result
  float pad;
};

// Behind every A: the largest singular value of X is at most the root of A's Frobenius norm, which is what the factors of the step's
// other products and of the next A go by.  (Bounds that come from the polynomials alone lag behind values that shrink, and what is
// stored loses bits.)  It is also at most what the polynomials so far make of singular values up to 1, with 1 % for rounding, once: a
// polynomial that is steep beyond the last one's range would make much of the 1 % of every step, and of a Frobenius norm, which is up
// to m^(1/4) too large.  (Eight steps of minimax polynomials whose bound stays below 2.1 ran up to 3352 without it, and 512 x 1024 was off
// by 2e-5 in single steps, 2e-4 in groups and 0.1 in the groups of a bf16 set, of the result's norm; with it 8e-7, 9e-6 and 5e-5.
// Float32 products: 9e-7.)
struct StepArgs {
  float a, b, c;
  float q;  // a's of the group's earlier steps, multiplied
  double before_most, after_most;  // what the steps before it, and it as well, make of singular values up to 1, at most
  int32_t first, last;
  // of R = b A + c A A; of Q = a Q + q R + R Q; of S = a A + R A; of the next A = a S + R S; of X = q a X + Q X; of A = X X^T
  Factors *square, *join, *half, *next, *update, *gram;
  const Bound* before;
  Bound* after;
};
// The factors of matrix w, by one wave: returns those of R, and the first of the matrix's waves stores all of them.
__device__ __forceinline__ Factors step_factors(const StepArgs& f, int w, const float* squares, int tiles, bool store) {
  Bound t = f.before[w];
  double v = 0;
  for (int i = threadIdx.x & 63; i < tiles; i += 64) v += squares[i];
  for (int k = 32; k; k >>= 1) v += __shfl_xor(v, k, 64);
  const double a = f.a, b = f.b, c = f.c, qa = f.first ? a : f.q * a;
  t.x = fmin(fmin(t.x, sqrt(sqrt(v) / t.in_a) * 1.01), f.before_most * 1.01);
  const double x2 = t.x * t.x, r = fabs(b) * x2 + fabs(c) * x2 * x2, x = fmin(quintic_bound(a, b, c, t.x), f.after_most) * 1.01;
  t.in_r = store_scale(r);
  const Factors square = {(float)(c * t.in_r / (t.in_a * t.in_a)), (float)(b * t.in_r / t.in_a), 0.f};
  if (!store) return square;
  f.square[w] = square;
  if (f.first) {
    t.q = r;
    t.in_q = t.in_r;
  } else {
    t.q = fabs(a) * t.q + fabs((double)f.q) * r + r * t.q;
    const double in_q = store_scale(t.q);
    f.join[w] = {(float)(in_q / (t.in_r * t.in_q)), (float)(a * in_q / t.in_q), (float)(f.q * in_q / t.in_r)};
    t.in_q = in_q;
  }
  if (f.last) {
    const double in_x = store_scale(x);
    f.update[w] = {(float)(in_x / (t.in_q * t.in_x)), (float)(qa * in_x / t.in_x), 0.f};
    t.in_x = in_x;
    t.in_a = store_scale(x * x);
    t.out = (float)(1 / in_x);
    f.gram[w] = {(float)(t.in_a / (in_x * in_x)), 0.f, 0.f};
  } else {
    const double in_s = store_scale(t.x * x), in_a = store_scale(x * x);
    f.half[w] = {(float)(in_s / (t.in_r * t.in_a)), (float)(a * in_s / t.in_a), 0.f};
    f.next[w] = {(float)(in_a / (t.in_r * in_s)), (float)(a * in_a / in_s), 0.f};
    t.in_a = in_a;
  }
  t.x = x;
  f.after[w] = t;
  return square;
}
// With tiles of 64 the workgroups of R find their factors themselves: 24
// matrices of 256 x 128..384 162 -> 150 us, of 512 x 300..1200 496 -> 485.  With tiles of 128 it is a launch of its own,
// one wave per matrix, 5 us.  (In the launch that makes A, by the last of the matrix's workgroups: what it needs of the others has to
// leave their caches first, 6 us.)
__global__ __launch_bounds__(64) void ortho_factors_kernel(const Mat* __restrict__ table, const float* __restrict__ squares, int tile, StepArgs f) {
  const Mat& m = table[blockIdx.x];
  const int mt = (m.m + tile - 1) / tile;
  step_factors(f, blockIdx.x, squares + m.square_tile, mt * (mt + 1) / 2, threadIdx.x == 0);
}

__device__ __forceinline__ void store_pair(char* p, const f32x4& v) {  // four values of a block
  half4 hi, lo;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    hi[j] = (half_t)v[j];
    lo[j] = (half_t)(v[j] - (float)hi[j]);
  }
  *reinterpret_cast<half4*>(p) = hi;
  *reinterpret_cast<half4*>(p + 64) = lo;
}
struct Eight {  // neighbouring values of a row
  float v[8];
  __device__ __forceinline__ float& operator[](int k) { return v[k]; }
  __device__ __forceinline__ float operator[](int k) const { return v[k]; }
};
__device__ __forceinline__ void store_pair(char* p, const Eight& v) {
  half8 hi, lo;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    hi[j] = (half_t)v[j];
    lo[j] = (half_t)(v[j] - (float)hi[j]);
  }
  *reinterpret_cast<half8*>(p) = hi;
  *reinterpret_cast<half8*>(p + 64) = lo;
}
// byte of the hi part of column c of a row
__device__ __forceinline__ int pair_byte(int c) { return (c >> 5) * 128 + (c & 31) * 2; }

// X = G / (|G| + eps): 64 x 64 of a matrix per block, padding included, through LDS where the matrix is stored transposed.  As many
// bytes go out as come in: a full layer's 2.2 GB take 436 us, 5.1 TB/s.  Every block adds up the norm for itself, and a matrix's first
// one also makes its tile lists and the factor of the first product (in a launch of their own they took 4 to 15 us).
__global__ __launch_bounds__(256) void ortho_start_kernel(const Mat* __restrict__ table, const double* __restrict__ sums, float eps,
                                                          Bound* __restrict__ bounds, Factors* __restrict__ gram, int side,
                                                          Mat* __restrict__ square_list, Mat* __restrict__ update_list) {
  __shared__ float s[64][65];
  __shared__ double s_sum[4];
  const Mat& m = table[blockIdx.y];
  const bool tall = m.rows > m.cols;
  const int nt = m.np / 64, tiles = m.mp / 64 * nt;
  if (blockIdx.x >= tiles) return;
  double v = 0;
  for (int i = threadIdx.x; i < m.parts; i += 256) v += sums[m.part + i];
  for (int b = 32; b; b >>= 1) v += __shfl_xor(v, b, 64);
  if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = v;
  __syncthreads();
  const double norm = sqrt((s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]));
  const double inv = norm == 0 ? 0 : 1 / (norm + eps);
  // singular values of X are at most its norm; 1 % for what rounding adds
  const double most = norm == 0 ? 1 : fmin(norm * inv, 1.0) * 1.01;
  const double in_x = store_scale(most), in = inv * in_x;
  if (blockIdx.x == 0) {
    const int mt = (m.m + side - 1) / side, nt = (m.n + side - 1) / side;
    Mat t = m;
    for (int i = threadIdx.x; i < mt * (mt + 1) / 2; i += 256) {  // row by row of the triangle
      t.mt = (int)((sqrtf(8.f * i + 1.f) - 1.f) * 0.5f);
      while ((t.mt + 1) * (t.mt + 2) / 2 <= i) ++t.mt;
      while (t.mt * (t.mt + 1) / 2 > i) --t.mt;
      t.nt = i - t.mt * (t.mt + 1) / 2;
      square_list[m.square_tile + i] = t;
    }
    for (int i = threadIdx.x; i < mt * nt; i += 256) {  // columns of eight tiles
      const int group = i / (8 * nt), height = min(8, mt - group * 8), in_group = i - group * 8 * nt;
      t.mt = group * 8 + in_group % height;
      t.nt = in_group / height;
      update_list[m.update_tile + i] = t;
    }
    if (threadIdx.x == 0) {
      const double in_a = store_scale(most * most);
      bounds[blockIdx.y] = {most, 0, in_x, in_a, 0, 0, 0.f, 0.f};
      gram[blockIdx.y] = {(float)(in_a / (in_x * in_x)), 0.f, 0.f};
    }
  }
  for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int m0 = tile / nt * 64, n0 = tile % nt * 64;
    const int r0 = tall ? n0 : m0, c0 = tall ? m0 : n0;
    const int at = threadIdx.x & 15;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = (threadIdx.x >> 4) + 16 * i;
      f32x4 g = {0.f, 0.f, 0.f, 0.f};
      const int64_t first = (int64_t)(r0 + r) * m.cols + c0 + at * 4;
      if (r0 + r < m.rows) {
        if (c0 + at * 4 + 4 <= m.cols) {
          g = *reinterpret_cast<const Vec<float>::V_u*>(m.G + first);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (c0 + at * 4 + j < m.cols) g[j] = m.G[first + j];
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float v = (float)(g[j] * in);
        if (tall) s[at * 4 + j][r] = v;
        else s[r][at * 4 + j] = v;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = (threadIdx.x >> 4) + 16 * i;
      f32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = s[r][at * 4 + j];
      store_pair(m.X[0] + (size_t)(m0 + r) * m.np * 4 + pair_byte(n0 + at * 4), v);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------- products
// C = product P Q + first E + second F over TILE x TILE tiles, four waves, a quarter of the tile each.
//   SQUARES: C, E, F are [mp, mp] slots, and so are P and Q (symmetric), or both are X (A = X X^T, K = n): operands along K (TILE 128:
//            a slot's up to its diagonal)
//   else:    P is a slot along K, Q = X [mp, np] across it, E = X, C the other X or, in the last step, U (OUT)
//
// A step is 32 of K: a panel row is 64 bytes of hi and 64 of lo, and every fragment feeds two or one of the three products: 192
// matrix instructions of 16 x 16 x 32 per 32 KiB of panels (TILE 128), two thirds of the loads per instruction that a plain 16-bit
// product of this tile has.  Two workgroups share a CU (TILE 128, two stages of panels), so that one multiplies while the other
// waits.  Sets with few tiles take TILE 64 and five stages: there is nothing else on the CU then, and a step lasts as long
// as its loads unless they are under way early.
//
// Measured, tiles of 128: Q X of a full layer (24 matrices, 2048 x 2816..8448: 1.13e12 operations, three times as many in 16 bits) takes
// 2.8 to 2.9 ms, 1.2e15 16-bit operations a second where plain 16-bit products of 8192 x 8192 x 8192 reach 1.1e15 to 1.5e15 by card; A A takes 0.54 to
// 0.6 ms, 1.1e15.  The matrix pipes are busy 62 to 66 % of the time at 1.6 GHz, which is what the card's power leaves.  Squares of 352 to 1056
// take 0.3 ms for 192 of them, 0.75e15: 44 % at 1.9 GHz, a step of two workgroups 2600 clocks where its instructions take 1540; a quarter of
// a tile's time is its opening and its result, which the other workgroup's steps fill (E brought into the cache during the last step: 7960 -> 8080 us).  A tile of 256 x 256
// halves the reads of LDS and has one workgroup on a CU: all of them store at once, and narrow matrices do not fill it (before the steps
// that follow it, 64 narrow experts 10.0 -> 12.4 ms, a full layer 19.7 -> 18.6).  Loads two steps ahead, with a second barrier a step: a full layer 16.6
// -> 17.3 ms, 12 of 1024 x 1408..4224 1480 -> 1440 us.  Tiles of 64: a product of 24 matrices of at most 256 x 384 takes 8 to 9 us, four
// round trips to memory.
enum Out { OUT_PAIRS, OUT_F32, OUT_BF16 };
constexpr int BK = 32;
// Steps that are summed in one register.  A matrix instruction loses what lies 2^-26 below the sum that it adds to, so that shorter sums
// are nearer.  Errors of five steps in units of 2^-24, 512 x 1024, and us of 64 narrow experts / a full layer, 16 steps: 23, 7920 / 17000; 8: 16,
// 8040 / 17290; 4: 13, 8090 / 17670; 2: 12, 8230 / 18230.  (Float32 products: 17.)
constexpr int JOIN = 8;
// Neighbouring tiles that an XCD gets, of every 8 times as many: they share panels in its L2.  us, runs of 4 / 16 / 32 / 64: a full layer
// 17510 / 17080 / 16710 / 16920, 64 narrow experts 8550 / 7920 / 7800 / 7805; tiles of 64, runs of 4 / 8 / 16 / 32: 24 matrices of 512 x
// 300..1200 483 / 499 / 498 / 629, 12 of 512 x 500..1200 364 / 336 / 322 / 318, 6 of 768 x 700..1500 434 / 432 / 389 / 381.
constexpr int run_of(int tile) { return tile == 64 ? 16 : 32; }
struct SquareOp {
  const Factors* factors;
  int32_t p, q, e, f, c;  // slots; p < 0: X, e and f < 0: none
  int32_t sum;            // the squares of C are summed
  int32_t step;           // R: its factors come from StepArgs
};
struct ProductArgs {
  const Mat* list;
  SquareOp op[2];         // blockIdx.y
  const Bound* bounds;
  float* squares;         // sums of the squares of a result's tiles, as stored
  int32_t x;              // X[x] is the present one
  int32_t tiles;
  StepArgs step;
};

// What a workgroup has to do.  (All of it is read at once: what is read through a reference later is read again behind every
// barrier, one round trip after the other.)
template <int TILE, bool SQUARES, Out OUT>
struct Job {
  const char *P, *Q, *E, *F;
  char* C;
  void* U;
  int which, rows, cols, m0, n0, K, ldp, ldq, ldc;  // (distances of rows in bytes)
  float f_product, f_first, f_second, out;
  int square_tile;
  bool step;  // the factors are still to be found
  bool square, mirror, sum;  // P (and Q) are squares; C is off the diagonal
  __device__ __forceinline__ void load(const ProductArgs& a, int tile) {
    const SquareOp& o = a.op[SQUARES ? blockIdx.y : 0];
    const int op_p = o.p, op_q = o.q, op_e = o.e, op_f = o.f, op_c = o.c;
    const Mat& m = a.list[tile];
    const int mp = m.mp, np = m.np, mt = m.mt, nt = m.nt;
    char *const X0 = m.X[0], *const X1 = m.X[1], *const slots = m.slot;
    which = m.which;
    rows = m.rows;
    cols = m.cols;
    U = m.U;
    sum = o.sum;
    square_tile = m.square_tile;
    step = o.step;
    if (!step) {
      const Factors* const f = o.factors + which;
      f_product = f->product;
      f_first = f->first;
      f_second = f->second;
    }
    out = OUT == OUT_PAIRS ? 1.f : a.bounds[which].out;
    const char* const X = a.x ? X1 : X0;
    const size_t slot = (size_t)mp * mp * 4;
    const bool gram = SQUARES && op_p < 0;
    square = !gram;
    m0 = mt * TILE;
    n0 = nt * TILE;
    K = gram ? max(rows, cols) : min(rows, cols);
    ldp = (gram ? np : mp) * 4;
    ldq = (gram || !SQUARES ? np : mp) * 4;
    ldc = (SQUARES ? mp : np) * 4;
    P = gram ? X : slots + op_p * slot;
    Q = gram || !SQUARES ? X : slots + op_q * slot;
    E = SQUARES ? (op_e >= 0 ? slots + op_e * slot : nullptr) : X;
    F = SQUARES && op_f >= 0 ? slots + op_f * slot : nullptr;
    C = SQUARES ? slots + op_c * slot : a.x ? X0 : X1;
    mirror = SQUARES && mt != nt;
  }
  // eight neighbouring values of a row of the last step's result
  __device__ __forceinline__ void give(int r, int c, const Eight& v) const {
    typedef std::conditional_t<OUT == OUT_F32, float, bf16_t> T;
    typedef T T4 __attribute__((ext_vector_type(4)));
    typedef T4 T4_u __attribute__((aligned(sizeof(T))));
    T4 u[2];
#pragma unroll
    for (int k = 0; k < 8; ++k) u[k >> 2][k & 3] = (T)(v[k] * out);
    if (r >= rows) return;
    T* const to = static_cast<T*>(U) + (int64_t)r * cols + c;
    if (c + 8 <= cols) {
      reinterpret_cast<T4_u*>(to)[0] = u[0];
      reinterpret_cast<T4_u*>(to)[1] = u[1];
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (c + k < cols) to[k] = u[k >> 2][k & 3];
    }
  }
};
// (workgroups go to the XCDs in turn)
template <int TILE>
__device__ __forceinline__ int tile_of_workgroup() {
  constexpr int RUN = run_of(TILE);
  const int i = blockIdx.x / 8;
  return (i / RUN * 8 + (int)(blockIdx.x % 8)) * RUN + i % RUN;
}
// the 16-byte chunk of a panel row whose data lies in chunk `lane`: a row along K (eight chunks), row k of K across it
__device__ __forceinline__ int along_chunk(int r, int chunk) { return chunk ^ ((r >> 1) & 7); }
__device__ __forceinline__ int across_chunk(int k, int chunk) { return chunk ^ (4 * (k & 3) + 2 * (k >> 3 & 1)); }
// fragments of 16 rows (or columns): 8 K per lane from 8 (lane >> 4) on, hi (part 0) or lo (1)
__device__ __forceinline__ half8 along_fragment(const char* panel, int row, int part, int lane) {
  const int kq = lane >> 4, l16 = lane & 15;
  return *reinterpret_cast<const half8*>(panel + (row + l16) * 128 + (along_chunk(l16, part * 4 + kq) << 4));
}
template <int TILE>
__device__ __forceinline__ half8 across_fragment(const char* panel, int col, int part, int lane) {
  // lane 16 kq + s reads 8 bytes at row 8 kq + h + (s >> 2) of K, columns col + 4 (s & 3) on, and gets four K of column col + s
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  typedef __attribute__((address_space(3))) s16x4* lds_s16x4_ptr;
  const int kq = lane >> 4, l16 = lane & 15, r = l16 >> 2;
  const int c16 = (col >> 5) * 8 + part * 4 + (col >> 4 & 1) * 2 + ((l16 & 3) >> 1);
  const char* const at = panel + (kq * 8 + r) * (TILE * 4) + (across_chunk(kq * 8 + r, c16) << 4) + (l16 & 1) * 8;
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(at));
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(at + 4 * (TILE * 4)));
  const s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_bit_cast(half8, v);
}

template <int TILE, int STAGES, bool SQUARES, Out OUT>
__global__ __launch_bounds__(256, 2) void ortho_product_kernel(ProductArgs a) {
  constexpr int PANEL = TILE * 128, UNITS = TILE / 32;  // bytes of a panel; its 1 KiB units per wave
  constexpr int W = TILE / 2, NB = W / 16;              // a wave's part: NB x NB blocks of 16 x 16
  constexpr int RING = STAGES * 2 * PANEL;
  static_assert(RING >= TILE * TILE * 4, "the result's tile fits the ring");
  __shared__ __align__(1024) char s_ring[RING];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int tile = tile_of_workgroup<TILE>();
  if (tile >= a.tiles) return;
  Job<TILE, SQUARES, OUT> job;
  job.load(a, tile);
  const int steps = (job.K + BK - 1) / BK;

  // A square's panel comes along its rows up to the diagonal, which rows m0 (n0) meet in step p_turn (q_turn), and from there on across
  // them, as columns: what lies above is not stored.
  constexpr bool HALF = TILE == 128;
  const int p_turn = HALF && job.square ? (job.m0 + TILE) / BK : steps, q_turn = HALF && SQUARES && job.square ? (job.n0 + TILE) / BK : steps;

  // ---- loads: units of 1 KiB, landing swizzled (16-byte chunks of a row XOR-ed)
  struct Loads {
    const char* at;
    size_t step;  // bytes
    uint32_t off[UNITS];
    __device__ __forceinline__ void along(const char* from, int first, int ld, int unit, int lane) {
      at = from + (size_t)first * ld;
      step = 128;
#pragma unroll
      for (int i = 0; i < UNITS; ++i) {
        const int r = (unit + i) * 8 + (lane >> 3);
        off[i] = r * ld + along_chunk(r, lane & 7) * 16;
      }
    }
    __device__ __forceinline__ void across(const char* from, int first, int k0, int ld, int unit, int lane) {
      constexpr int CHUNKS = TILE / 4;  // of a row of K
      at = from + (size_t)k0 * ld + (size_t)first * 4;
      step = (size_t)BK * ld;
#pragma unroll
      for (int i = 0; i < UNITS; ++i) {
        const int k = (unit + i) * (64 / CHUNKS) + lane / CHUNKS;
        off[i] = k * ld + across_chunk(k, lane % CHUNKS) * 16;
      }
    }
  };
  Loads p, q;
  p.along(job.P, job.m0, job.ldp, wave * UNITS, lane);
  if (SQUARES) q.along(job.Q, job.n0, job.ldq, wave * UNITS, lane);
  else q.across(job.Q, job.n0, 0, job.ldq, wave * UNITS, lane);
  const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_address(s_ring));
  auto issue = [&](int stage, int g) {
    if (HALF && g == p_turn) p.across(job.P, job.m0, g * BK, job.ldp, wave * UNITS, lane);
    if (HALF && SQUARES && g == q_turn) q.across(job.Q, job.n0, g * BK, job.ldq, wave * UNITS, lane);
    const uint32_t dst = lds + stage * 2 * PANEL + wave * (UNITS * 1024);
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      dma_b128_s(p.at, p.off[i], dst + i * 1024);
      dma_b128_s(q.at, q.off[i], dst + PANEL + i * 1024);
    }
    p.at += p.step;
    q.at += q.step;
  };
  const int kq = lane >> 4, l16 = lane & 15;
  f32x4 total[NB][NB], acc[NB][NB];
  // acc joins total and starts again
  auto join = [&](bool first) {
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          total[i][j][r] = first ? 0.f : total[i][j][r] + acc[i][j][r];
          acc[i][j][r] = 0.f;
        }
  };
  join(true);

  // In the result a lane holds eight neighbouring columns of a row, by way of LDS, and a wave's access lies in as few cache lines as there
  // are.  (As the matrix instructions leave it a lane has four columns and the next lane another row: 64 narrow experts 8830 us where
  // this takes 7980, a full layer 17830 and 16950, 24 matrices of 256 x 128..384 174 and 161.)
  constexpr int LANES = W / 8, ROWS = 64 / LANES, TURNS = W / ROWS;
  const int at_row = lane / LANES, at_col = lane % LANES * 8;
  const size_t corner = (size_t)(job.m0 + wm * W) * job.ldc + pair_byte(job.n0 + wn * W);
  auto at = [&](int turn) { return (uint32_t)((turn * ROWS + at_row) * job.ldc + pair_byte(at_col)); };
  // what is added to the product: all its loads together (one after the other they took 0.7 us each, 11 us of a tile), and with
  // small tiles, which have the registers, in front of everything else
  half8 hi[TURNS], lo[TURNS];
  auto fetch = [&](const char* from) {
#pragma unroll
    for (int t = 0; t < TURNS; ++t) {
      hi[t] = *reinterpret_cast<const half8*>(from + corner + at(t));
      lo[t] = *reinterpret_cast<const half8*>(from + corner + at(t) + 64);
    }
  };
  constexpr bool EARLY = TILE == 64;
  // Waves whose part lies beyond the matrix, and the upper right one of a tile on the diagonal, whose part is the transpose of the lower
  // left one's, leave the matrix pipe to the others (and meet them at the barriers): 64 narrow experts 10083 -> 9836 us.  (With small
  // tiles they multiply, and what they make is not stored: the branch costs more.)
  const int last_row = min(job.rows, job.cols), last_col = SQUARES ? last_row : max(job.rows, job.cols);
  const bool diagonal = SQUARES && !job.mirror;
  const bool idle = job.m0 + wm * W >= last_row || job.n0 + wn * W >= last_col || (diagonal && wm < wn);
  const bool twice = job.mirror || (diagonal && wm > wn);            // what this wave makes stands for two places,
  const bool mirrored = HALF ? diagonal && wm > wn : twice;          // and goes there
  if (EARLY && job.E && !idle) fetch(job.E);

  auto panel = [&](int stage) -> const char* { return s_ring + stage * 2 * PANEL; };
  struct Fragments {
    half8 p[NB][2], q[NB][2];
  };
  auto read = [&](Fragments& f, int stage, auto p_across, auto q_across) {
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        if constexpr (p_across.value) f.p[i][part] = across_fragment<TILE>(panel(stage), wm * W + i * 16, part, lane);
        else f.p[i][part] = along_fragment(panel(stage), wm * W + i * 16, part, lane);
        if constexpr (q_across.value) f.q[i][part] = across_fragment<TILE>(panel(stage) + PANEL, wn * W + i * 16, part, lane);
        else f.q[i][part] = along_fragment(panel(stage) + PANEL, wn * W + i * 16, part, lane);
      }
  };
  auto multiply = [&](const Fragments& f) {
    // (Q's fragment is the first operand: a lane then holds four neighbouring columns of C.  The blocks are walked to and fro.  hi hi
    // first, which needs half of the fragments: a full layer 19409 -> 19053 us; in front of the other wave's reads: 64 narrow experts 7854 -> 7800.)
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int t = 0; t < 3; ++t)
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int jj = 0; jj < NB; ++jj) {
          const int j = i % 2 ? NB - 1 - jj : jj;
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f.q[j][t == 1], f.p[i][t == 2], acc[i][j], 0, 0, 0);
        }
    __builtin_amdgcn_s_setprio(0);
  };
  // everybody's loads but those of the YOUNGER youngest stages have landed, and everybody's reads of LDS have returned
  auto meet = [&](auto younger, bool all_issued) {
    constexpr int LOADS = decltype(younger)::value * 2 * UNITS;
    static_assert(LOADS < 64, "vmcnt field");
    if (LOADS > 0 && all_issued) __builtin_amdgcn_s_waitcnt(0x0070 | (LOADS & 15) | (LOADS >> 4) << 14);
    else __builtin_amdgcn_s_waitcnt(0x0070);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  auto next = [](int stage) { return stage + 1 == STAGES ? 0 : stage + 1; };
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i)
    if (i < steps) issue(i, i);
  if constexpr (SQUARES && EARLY) {
    if (job.step) {
      const int mt = (last_row + TILE - 1) / TILE;
      const Factors f = step_factors(a.step, job.which, a.squares + job.square_tile, mt * (mt + 1) / 2, job.m0 + tid == 0);
      job.f_product = f.product;
      job.f_first = f.first;
    }
  }
  int stage = 0;
  constexpr std::false_type ALONG;
  constexpr std::bool_constant<!SQUARES> Q_FIRST;
  if constexpr (EARLY) {
    // One wave per SIMD: the next step's fragments are read while this one's are multiplied.
    Fragments f[2];
    meet(std::integral_constant<int, STAGES - 2>{}, STAGES - 2 < steps);
    read(f[0], 0, ALONG, Q_FIRST);
    auto body = [&](auto set, int g) {
      constexpr int SET = decltype(set)::value;
      if (g + 1 < steps) {
        meet(std::integral_constant<int, STAGES - 3>{}, g + STAGES - 2 < steps);
        if (g + STAGES - 1 < steps) issue(stage == 0 ? STAGES - 1 : stage - 1, g + STAGES - 1);
        stage = next(stage);
        read(f[1 - SET], stage, ALONG, Q_FIRST);
      }
      multiply(f[SET]);
      if (g % JOIN == JOIN - 1) join(false);
    };
#pragma unroll 1
    for (int g = 0; g < steps; g += 2) {
      body(std::integral_constant<int, 0>{}, g);
      if (g + 1 < steps) body(std::integral_constant<int, 1>{}, g + 1);
    }
  } else {
    int g = 0;
    auto run = [&](int end, auto p_across, auto q_across) {
#pragma unroll 1
      for (; g < end; ++g) {
        meet(std::integral_constant<int, STAGES - 2>{}, g + STAGES - 2 < steps);
        if (g + STAGES - 1 < steps) issue(stage == 0 ? STAGES - 1 : stage - 1, g + STAGES - 1);
        if (!idle) {
          Fragments f;
          read(f, stage, p_across, q_across);
          multiply(f);
        }
        stage = next(stage);
        if (g % JOIN == JOIN - 1) join(false);
      }
    };
    constexpr std::true_type ACROSS;
    if constexpr (SQUARES) run(min(q_turn, steps), ALONG, ALONG);
    run(min(p_turn, steps), ALONG, ACROSS);
    run(steps, ACROSS, ACROSS);
  }
  join(false);

  // ---- result
  if (!EARLY && job.E && !idle) fetch(job.E);
  __syncthreads();  // the ring has been read: a wave's part of it holds the wave's part of the tile, chunks of four values XOR-ed with the row
  float sum = 0.f;
  if (!idle) {
    char* const mine = s_ring + wave * (W * W * 4);
    auto staged = [&](int r, int chunk) { return mine + r * (W * 4) + ((chunk ^ (r & (W / 4 - 1))) << 4); };
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) *reinterpret_cast<f32x4*>(staged(i * 16 + l16, j * 4 + kq)) = total[i][j];
    wave_lds_order();
    Eight v[TURNS];
#pragma unroll
    for (int t = 0; t < TURNS; ++t)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const f32x4 u = *reinterpret_cast<const f32x4*>(staged(t * ROWS + at_row, at_col / 4 + k));
#pragma unroll
        for (int j = 0; j < 4; ++j) v[t][4 * k + j] = u[j] * job.f_product;
      }
    auto add = [&](float factor) {
#pragma unroll
      for (int t = 0; t < TURNS; ++t)
#pragma unroll
        for (int k = 0; k < 8; ++k) v[t][k] += factor * ((float)hi[t][k] + (float)lo[t][k]);
    };
    if (job.E) add(job.f_first);
    if (job.F) {
      fetch(job.F);
      add(job.f_second);
    }
    const int r0 = job.m0 + wm * W, c0 = job.n0 + wn * W;
    const bool turned = OUT == OUT_PAIRS ? mirrored : job.rows > job.cols;  // goes out as columns
    if (OUT == OUT_PAIRS || !turned) {
#pragma unroll
      for (int t = 0; t < TURNS; ++t) {
        if constexpr (OUT == OUT_PAIRS) store_pair(job.C + corner + at(t), v[t]);
        else job.give(r0 + t * ROWS + at_row, c0 + at_col, v[t]);
      }
    }
    if (SQUARES && job.sum) {
#pragma unroll
      for (int t = 0; t < TURNS; ++t)
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += v[t][k] * v[t][k];
    }
    if (turned) {
#pragma unroll
      for (int t = 0; t < TURNS; ++t)
#pragma unroll
        for (int k = 0; k < 2; ++k) *reinterpret_cast<f32x4*>(staged(t * ROWS + at_row, at_col / 4 + k)) = f32x4{v[t][4 * k], v[t][4 * k + 1], v[t][4 * k + 2], v[t][4 * k + 3]};
      wave_lds_order();
#pragma unroll
      for (int t = 0; t < TURNS; ++t) {
        const int c = t * ROWS + at_row;
        Eight u;
#pragma unroll
        for (int k = 0; k < 8; ++k) u[k] = reinterpret_cast<const float*>(staged(at_col + k, c / 4))[c % 4];
        if constexpr (OUT == OUT_PAIRS) store_pair(job.C + (size_t)(c0 + c) * job.ldc + pair_byte(r0 + at_col), u);
        else job.give(c0 + c, r0 + at_col, u);
      }
    }
  }
  if constexpr (SQUARES) {
    if (job.sum) {
      __syncthreads();
      float* const part = reinterpret_cast<float*>(s_ring);
      sum = wave_sum(sum);
      if (lane == 0) part[wave] = twice ? 2.f * sum : sum;
      __syncthreads();
      if (tid == 0) a.squares[tile] = (part[0] + part[1]) + (part[2] + part[3]);
    }
  }
}

size_t align256(size_t v) { return (v + 255) / 256 * 256; }
size_t mat_bytes(int64_t mp, int64_t np, int slots) { return (size_t)(2 * mp * np + slots * mp * mp) * 4; }
int64_t tiles_of(int64_t v, int tile) { return (v + tile - 1) / tile; }
}  // namespace

// What a group's roundings have come to in the A of its last step, at most, in units of one of a value of 1: a step's own are those of
// terms up to (|a| + |b| x^2 + |c| x^4)^2 x^2 that all but cancel (x: the largest singular value), and what was there grows by the square
// of the polynomial's largest ratio.  Errors against float64 of 512 x 1024, of the result's norm, single steps / groups up to 2000 / up to
// 3e5 (float32 products): five steps of the usual coefficients, where singular values fall to a hundredth in equal ratios 1.2e-6 / 3.8e-6 /
// 4.1e-5 (2.6e-6), one value of 1 and 511 of 0.01 1.3e-6 / 1.6e-6 / 8.7e-4 (6.3e-6), strong directions in noise 1.0e-6 / 1.4e-6 / 1.6e-4
// (2.1e-6); six minimax steps, values as the first 1.5e-6 / 3.4e-6 / 2.0e-5 (3.3e-6), and 1.2e-4 in groups that went by the ratios alone; eight
// where they fall to 1e-4 1.6e-5 / 1.6e-5 / 9.6e-4 (3.4e-5).  bf16 results are rounded by 1.7e-3 behind that, 1.9e-3 with the worst of these, and
// 64 narrow experts into bf16 take 8.0 ms for it where groups up to 2000 take 9.1.
constexpr double F32_ROUNDINGS = 2000, BF16_ROUNDINGS = 3e5;

modse_status ortho_layout(const modse_matrix_set* set, const float* coeffs, int steps, OrthoLayout& w) {
  const int n = set->n_matrices;
  constexpr int SIDES[2] = {64, 128};
  int64_t square[2] = {0, 0}, update[2] = {0, 0}, parts = 0;
  double m3 = 0, m2n = 0;
  for (int i = 0; i < n; ++i) {
    const int r = set->rows[i], c = set->cols[i];
    if (r < 1 || c < 1) return MODSE_ERR_INVALID_ARG;
    if (r > 65536 || c > 65536) return MODSE_ERR_UNSUPPORTED;
    const int64_t sm = r < c ? r : c, sn = r < c ? c : r;
    for (int t = 0; t < 2; ++t) {
      const int64_t mt = tiles_of(sm, SIDES[t]);
      square[t] += mt * (mt + 1) / 2;
      update[t] += mt * tiles_of(sn, SIDES[t]);
    }
    parts += ((int64_t)r * c + PART - 1) / PART;
    m3 += (double)sm * sm * sm;
    m2n += (double)sm * sm * sn;
  }
  if (update[0] >= (int64_t)1 << 23) return MODSE_ERR_UNSUPPORTED;  // (a launch has fewer than 2^32 threads)
  // Tiles of 64 where those of 128 leave a quarter of the CUs without one.  us, 64 / 128: 24 matrices of 256 x 128..384 146 / 253, 48 of
  // 256 x 100..700 (144 tiles of 128) 235 / 319, 3 of 1100 x 1500 (135) 636 / 660, 24 of 512 x 300..1200 (190) 467 / 470, into bf16 448 / 433,
  // 6 of 1024 x 1024 (216) 678 / 631, 6 of 1024 x 1408..4224 (216) 1050 / 928, 12 of 768 x 700..2100 (252) 744 / 642, 12 of 1024 x
  // 1408..4224 (432) 2037 / 1492.
  const int side = square[1] <= 192 ? 0 : 1;
  w.tile = SIDES[side];
  w.square_tiles = (int32_t)square[side];
  w.update_tiles = (int32_t)update[side];
  w.parts = (int32_t)parts;
  // Groups of steps where the products are what counts, and X is longer than it is wide.  us, single steps / groups: 24 matrices of
  // 256 x 128..384 146 / 150, 3 of 256 x 256 110 / 128, 6 of 512 x 700..1200 249 / 222, 24 of 512 x 300..1200 491 / 468, 12 of 1000 x
  // 333..1999 into bf16 926 / 787, 12 of 1024 x 1408..4224 2061 / 1492; squares, 3 of 2048 x 2048 1630 / 1738, 3 of 1111 x 1500 636 / 650.
  const bool grouped = m2n >= 6e8 && m2n >= 1.4 * m3;
  w.slots = grouped ? N_SLOTS : SLOT_R + 1;  // (a step alone has A and R)
  size_t data = 0;
  for (int i = 0; i < n; ++i) {
    const int r = set->rows[i], c = set->cols[i];
    data += mat_bytes(padded(r < c ? r : c), padded(r < c ? c : r), w.slots);
  }
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off = align256(off + bytes);
    return o;
  };
  w.mats = take(n * sizeof(Mat));
  w.bounds = take(2 * n * sizeof(Bound));
  w.factors = take((size_t)n * 6 * sizeof(Factors));
  w.squares = take((size_t)w.square_tiles * 4);
  w.sums = take((size_t)parts * sizeof(double));
  w.square_list = take((size_t)w.square_tiles * sizeof(Mat));
  w.update_list = take((size_t)w.update_tiles * sizeof(Mat));
  w.data = take(data);
  w.total = n ? off : 0;
  w.n_groups = 0;
  const double most = set->dtype == MODSE_F32 ? F32_ROUNDINGS : BF16_ROUNDINGS;
  double top = 1;
  w.most[0] = top;
  for (int i = 0; coeffs && i < steps;) {
    double roundings = top * top;
    int g = 0;
    do {
      const float* const c = coeffs + 3 * (i + g);
      const double slope = ratio_bound(c[0], c[1], c[2], top), x2 = top * top, term = fabs(c[0]) + (fabs(c[1]) + fabs(c[2]) * x2) * x2;
      roundings = roundings * (slope > 1 ? slope * slope : 1) + term * term * x2;
      top = quintic_bound(c[0], c[1], c[2], top);
      ++g;
      w.most[i + g] = top;
    } while (grouped && i + g < steps && roundings <= most);
    w.group[w.n_groups++] = g;
    i += g;
  }
  return MODSE_OK;
}

hipError_t launch_orthogonalize(const modse_matrix_set* set, const OrthoLayout& w, const float* coeffs, float eps, char* ws, hipStream_t s) {
  const int n = set->n_matrices, tile = w.tile;
  Mat* const table = reinterpret_cast<Mat*>(ws + w.mats);
  Bound* const bounds = reinterpret_cast<Bound*>(ws + w.bounds);
  Factors* const factors = reinterpret_cast<Factors*>(ws + w.factors);
  Factors *const f_gram = factors, *const f_square = factors + n, *const f_join = factors + 2 * n, *const f_half = factors + 3 * n,
          *const f_next = factors + 4 * n, *const f_update = factors + 5 * n;
  float* const squares = reinterpret_cast<float*>(ws + w.squares);
  double* const sums = reinterpret_cast<double*>(ws + w.sums);
  Mat* const square_list = reinterpret_cast<Mat*>(ws + w.square_list);
  Mat* const update_list = reinterpret_cast<Mat*>(ws + w.update_list);
  // the matrices with the longest products first: 12 of 1000 x 333..1999 into bf16 1059 -> 995 us, a full layer 19053 -> 18825
  int32_t order[MAX_MATS];
  for (int i = 0; i < n; ++i) order[i] = i;
  std::sort(order, order + n, [&](int i, int j) {
    const int a = std::max(set->rows[i], set->cols[i]), b = std::max(set->rows[j], set->cols[j]);
    return a != b ? a > b : i < j;
  });
  int32_t square = 0, update = 0, part = 0, most_parts = 0, most_tiles = 0;
  int64_t data = 0;
  hipError_t e;
  for (int first = 0; first < n; first += MATS_PER_LAUNCH) {
    MatArgs a;
    a.table = table;
    a.data = ws + w.data;
    a.first = first;
    a.count = n - first < MATS_PER_LAUNCH ? n - first : MATS_PER_LAUNCH;
    most_parts = 0;
    for (int i = 0; i < a.count; ++i) {
      const int k = order[first + i], r = set->rows[k], c = set->cols[k];
      const int64_t sm = r < c ? r : c, sn = r < c ? c : r, mt = tiles_of(sm, tile);
      const int parts = (int)(((int64_t)r * c + PART - 1) / PART), mp = padded(sm), np = padded(sn), blocks = mp / 64 * (np / 64);
      a.mat[i] = {set->G[k], set->U[k], data, r, c, square, update, part, parts};
      square += (int32_t)(mt * (mt + 1) / 2);
      update += (int32_t)(mt * tiles_of(sn, tile));
      part += parts;
      data += (int64_t)mat_bytes(mp, np, w.slots);
      if (parts > most_parts) most_parts = parts;
      if (blocks > most_tiles) most_tiles = blocks;
    }
    hipLaunchKernelGGL(ortho_squares_kernel, dim3(most_parts < 1024 ? most_parts : 1024, a.count), dim3(256), 0, s, a, sums);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  hipLaunchKernelGGL(ortho_start_kernel, dim3(std::min(most_tiles, std::max(8, 16384 / n)), n), dim3(256), 0, s, table, sums, eps, bounds, f_gram,
                     tile, square_list, update_list);
  if ((e = hipGetLastError()) != hipSuccess) return e;

  ProductArgs a = {square_list, {}, bounds, squares, 0, w.square_tiles, {}};
  const bool in_products = tile == 64;  // R's launches find their factors
  const int span = 8 * run_of(tile);
  auto grid = [span](int tiles, int ops) { return dim3((tiles + span - 1) / span * span, ops); };
  auto squares_of = [&](const SquareOp& one, const SquareOp* two) {
    a.list = square_list;
    a.tiles = w.square_tiles;
    a.op[0] = one;
    if (two) a.op[1] = *two;
    const dim3 g = grid(a.tiles, two ? 2 : 1);
    if (tile == 128) hipLaunchKernelGGL((ortho_product_kernel<128, 2, true, OUT_PAIRS>), g, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((ortho_product_kernel<64, 5, true, OUT_PAIRS>), g, dim3(256), 0, s, a);
    return hipGetLastError();
  };
  auto update_by = [&](int q, auto out) {
    constexpr Out OUT = decltype(out)::value;
    a.list = update_list;
    a.tiles = w.update_tiles;
    a.op[0] = {f_update, q, -1, -1, -1, -1, 0, 0};
    const dim3 g = grid(a.tiles, 1);
    if (tile == 128) hipLaunchKernelGGL((ortho_product_kernel<128, 2, false, OUT>), g, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((ortho_product_kernel<64, 5, false, OUT>), g, dim3(256), 0, s, a);
    return hipGetLastError();
  };
  int step = 0;
  for (int k = 0; k < w.n_groups; ++k) {
    int A = SLOT_A, Q = SLOT_R;
    float qa = 0.f;
    // the factors that the A of the group's step i brings
    auto factors_of = [&](int i) {
      const float* const c = coeffs + 3 * (step + i);
      Bound* const after = bounds + n - (a.bounds - bounds);  // (the two take turns)
      a.step = {c[0], c[1], c[2], qa, w.most[step + i], w.most[step + i + 1], i == 0, i + 1 == w.group[k], f_square, f_join, f_half, f_next, f_update, f_gram, a.bounds, after};
      a.bounds = after;
      if (in_products) return hipSuccess;
      hipLaunchKernelGGL(ortho_factors_kernel, dim3(n), dim3(64), 0, s, table, squares, tile, a.step);
      return hipGetLastError();
    };
    if ((e = squares_of({f_gram, -1, -1, -1, -1, SLOT_A, 1, 0}, nullptr)) != hipSuccess) return e;
    if ((e = factors_of(0)) != hipSuccess) return e;
    for (int i = 0; i < w.group[k]; ++i) {
      const float first = coeffs[3 * (step + i)];
      const bool last = i + 1 == w.group[k];
      const int R = i == 1 ? SLOT_R2 : SLOT_R;  // (the first one is Q in the second step)
      if ((e = squares_of({f_square, A, A, A, -1, R, 0, in_products}, nullptr)) != hipSuccess) return e;
      const int Q2 = i == 0 ? R : Q == SLOT_Q ? SLOT_R2 : SLOT_Q;
      const SquareOp join = {f_join, R, Q, Q, R, Q2, 0, 0}, half = {f_half, R, A, A, -1, SLOT_S, 0, 0};
      if (i > 0 || !last) {
        if ((e = i == 0 ? squares_of(half, nullptr) : last ? squares_of(join, nullptr) : squares_of(join, &half)) != hipSuccess) return e;
      }
      Q = Q2;
      qa = i == 0 ? first : qa * first;
      if (!last) {
        A = A == SLOT_A ? SLOT_A2 : SLOT_A;
        if ((e = squares_of({f_next, R, SLOT_S, SLOT_S, -1, A, 1, 0}, nullptr)) != hipSuccess) return e;
        if ((e = factors_of(i + 1)) != hipSuccess) return e;
      }
    }
    step += w.group[k];
    if (k + 1 < w.n_groups) e = update_by(Q, std::integral_constant<Out, OUT_PAIRS>{});
    else if (set->dtype == MODSE_F32) e = update_by(Q, std::integral_constant<Out, OUT_F32>{});
    else e = update_by(Q, std::integral_constant<Out, OUT_BF16>{});
    if (e != hipSuccess) return e;
    a.x = 1 - a.x;
  }
  return hipSuccess;
}
