// The orthogonalised update: X = G / (|G| + eps), then X <- a X + (b A + c A^2) X with A = X X^T, for every matrix of a set.
//
// All of it is matrix products: for an m x n matrix (m the shorter side; a tall one is stored transposed) X X^T, A A and R X.
// The iteration enlarges small singular values by up to a per step, and with them the rounding errors of the large ones, so the
// products need float32 precision.  They get it from the 16-bit matrix instructions, whose rate is sixteen times that of the
// float32 ones: a value is stored as hi + lo, two float16 numbers with 11 bits each, times a power of two that keeps the
// largest value that the matrix can have (a bound on its singular values) below 2^15, and a product is hi hi + hi lo + lo hi,
// summed in float32.  What is left out, lo lo, is 2^-24 of the product in the mean, as a float32 rounding is.  Simulated on the
// CPU, and measured: errors against float64 as those of float32 products (1.3e-6 and 1.4e-6 after five steps).
//
// Storage: rows of blocks of 32 values, 64 bytes of hi and then 64 of lo, so that a cache line feeds one step of a product.
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

__global__ __launch_bounds__(64) void ortho_table_kernel(MatArgs a) {
  const int i = threadIdx.x;
  if (i >= a.count) return;
  const MatArg& t = a.mat[i];
  Mat m;
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
  a.table[a.first + i] = m;
}

constexpr int PART = 1 << 15;  // elements of a partial sum of squares
// (float64: no overflow, and the order of the additions is of no account)
__global__ __launch_bounds__(256) void ortho_squares_kernel(const Mat* __restrict__ table, double* __restrict__ sums) {
  __shared__ double s[4];
  const Mat& m = table[blockIdx.y];
  const int64_t n = (int64_t)m.rows * m.cols;
  const float* const G = m.G;
  for (int part = blockIdx.x; part < m.parts; part += gridDim.x) {
    const int64_t end = min(n, ((int64_t)part + 1) * PART);
    double v = 0;
    for (int64_t i = (int64_t)part * PART + threadIdx.x * 4; i < end; i += 1024) {
      if (i + 4 <= end) {
        const f32x4 g = *reinterpret_cast<const f32x4_u*>(G + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) v += (double)g[j] * g[j];
      } else {
        for (int64_t j = i; j < end; ++j) v += (double)G[j] * G[j];
      }
    }
    for (int b = 32; b; b >>= 1) v += __shfl_xor(v, b, 64);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0) sums[m.part + part] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
  }
}

// the power of two that takes what is at most `bound` to at most 2^15 (twice that in error)
__device__ inline double store_scale(double bound) {
  int e = 0;
  if (bound > 0 && bound < 1e300) frexp(bound, &e);
  return ldexp(1.0, 15 - e);
}

// What is known of a matrix on its way through the steps.
struct Bound {
  double x;              // singular values of the present X are at most this
  double in_x, in_a;     // the factors that X and A are stored with
  double start;          // G's
  float out;             // 1 / in_x, of the result
  float pad;
};

// One block per matrix: the norm, the factor of the first product, the matrix's part of the tile lists.
__global__ __launch_bounds__(256) void ortho_prepare_kernel(const Mat* __restrict__ table, const double* __restrict__ sums, float eps,
                                                            Bound* __restrict__ bounds, Factors* __restrict__ gram,
                                                            int32_t* __restrict__ square_map, int32_t* __restrict__ update_map) {
  __shared__ double s[4];
  const Mat& m = table[blockIdx.x];
  double v = 0;
  for (int i = threadIdx.x; i < m.parts; i += 256) v += sums[m.part + i];
  for (int b = 32; b; b >>= 1) v += __shfl_xor(v, b, 64);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  const int mt = m.mp / PAD, nt = m.np / PAD;
  for (int i = threadIdx.x; i < mt * mt; i += 256) square_map[m.square_tile + i] = blockIdx.x;
  for (int i = threadIdx.x; i < mt * nt; i += 256) update_map[m.update_tile + i] = blockIdx.x;
  if (threadIdx.x != 0) return;
  const double norm = sqrt((s[0] + s[1]) + (s[2] + s[3]));
  const double inv = norm == 0 ? 0 : 1 / (norm + eps);
  Bound b;
  // singular values of X are at most its norm; 1 % for what rounding adds
  b.x = norm == 0 ? 1 : fmin(norm * inv, 1.0) * 1.01;
  b.in_x = store_scale(b.x);
  b.in_a = store_scale(b.x * b.x);
  b.start = inv * b.in_x;
  b.out = 0.f;
  b.pad = 0.f;
  bounds[blockIdx.x] = b;
  gram[blockIdx.x] = {(float)(b.in_a / (b.in_x * b.in_x)), 0.f};
}

// One wave per matrix, behind every A = X X^T: the largest singular value of X is at most the root of A's Frobenius norm, which
// is what the factors of the step's other products and of the next A go by.  (Bounds that come from the polynomials alone lag
// behind values that shrink, and what is stored loses bits.)
__global__ __launch_bounds__(64) void ortho_factors_kernel(const Mat* __restrict__ table, const float* __restrict__ squares, float a, float b, float c,
                                                           Bound* __restrict__ bounds, Factors* __restrict__ square, Factors* __restrict__ update,
                                                           Factors* __restrict__ gram) {
  const Mat& m = table[blockIdx.x];
  const int mt = m.mp / PAD;
  double v = 0;
  for (int i = threadIdx.x; i < mt * mt; i += 64) v += squares[m.square_tile + i];
  for (int k = 32; k; k >>= 1) v += __shfl_xor(v, k, 64);
  if (threadIdx.x != 0) return;
  Bound t = bounds[blockIdx.x];
  t.x = fmin(t.x, sqrt(sqrt(v) / t.in_a) * 1.01);
  const double x2 = t.x * t.x, in_r = store_scale(fabs(b) * x2 + fabs(c) * x2 * x2);
  square[blockIdx.x] = {(float)(c * in_r / (t.in_a * t.in_a)), (float)(b * in_r / t.in_a)};
  t.x = quintic_bound(a, b, c, t.x) * 1.01;
  const double next = store_scale(t.x);
  update[blockIdx.x] = {(float)(next / (in_r * t.in_x)), (float)(a * next / t.in_x)};
  t.in_x = next;
  t.in_a = store_scale(t.x * t.x);
  t.out = (float)(1 / next);
  gram[blockIdx.x] = {(float)(t.in_a / (next * next)), 0.f};
  bounds[blockIdx.x] = t;
}

__device__ __forceinline__ void store_pair(char* p, const float (&v)[4]) {  // four values of a block
  half4 hi, lo;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    hi[j] = (half_t)v[j];
    lo[j] = (half_t)(v[j] - (float)hi[j]);
  }
  *reinterpret_cast<half4*>(p) = hi;
  *reinterpret_cast<half4*>(p + 64) = lo;
}
__device__ __forceinline__ void load_pair(const char* p, float (&v)[4]) {
  const half4 hi = *reinterpret_cast<const half4*>(p), lo = *reinterpret_cast<const half4*>(p + 64);
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = (float)hi[j] + (float)lo[j];
}
// byte of the hi part of column c of a row
__device__ __forceinline__ int pair_byte(int c) { return (c >> 5) * 128 + (c & 31) * 2; }

// X = G / (|G| + eps): 64 x 64 of a matrix per block, padding included
__global__ __launch_bounds__(256) void ortho_start_kernel(const Mat* __restrict__ table, const Bound* __restrict__ bounds) {
  __shared__ float s[64][65];
  const Mat& m = table[blockIdx.y];
  const double in = bounds[blockIdx.y].start;
  const bool tall = m.rows > m.cols;
  const int nt = m.np / 64, tiles = m.mp / 64 * nt;
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
          g = *reinterpret_cast<const f32x4_u*>(m.G + first);
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
      float v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = s[r][at * 4 + j];
      store_pair(m.X[0] + (size_t)(m0 + r) * m.np * 4 + pair_byte(n0 + at * 4), v);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------- products
// C = first E + product P Q over 128 x 128 tiles, four waves of 64 x 64 each.
//   SQUARES: C, E, P and Q are [mp, mp] slots (P = Q = X for A = X X^T, then K = n and there is no E); Q is symmetric or
//            transposed, so both operands are read along K
//   else:    P = R [mp, mp] along K, Q = X [mp, np] across it, E = X, C the other X or, in the last step, U (OUT)
enum Out { OUT_PAIRS, OUT_F32, OUT_BF16 };
constexpr int BK = 32;               // a row of a panel: 64 bytes of hi, 64 of lo
constexpr int PANEL = PAD * 128;     // bytes
constexpr int JOIN = 16;             // steps that are summed in one register
struct ProductArgs {
  const Mat* table;
  const Factors* factors;
  const Bound* bounds;
  float* squares;  // sums of the squares of A's tiles, as stored
  const int32_t* map;
  OpKind kind;
  int32_t x;  // X[x] is the present one
};

template <bool SQUARES, Out OUT>
__global__ __launch_bounds__(256, 2) void ortho_product_kernel(ProductArgs a) {
  __shared__ __align__(1024) char s_ring[4 * PANEL];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int which = uniform_int(a.map[blockIdx.x]);
  const Mat& m = a.table[which];
  const int mp = m.mp, np = m.np;
  const size_t slot = (size_t)mp * mp * 4;
  const bool gram = SQUARES && a.kind == OP_GRAM;
  const int local = blockIdx.x - (SQUARES ? m.square_tile : m.update_tile);
  const int nt = (SQUARES ? mp : np) / PAD;
  const int m0 = local / nt * PAD, n0 = local % nt * PAD;
  const int K = gram ? m.n : m.m, steps = (K + BK - 1) / BK;
  const char* const X = m.X[a.x];
  const int ldp = (gram ? np : mp) * 4, ldq = (gram || !SQUARES ? np : mp) * 4;  // bytes
  const char* const P = gram ? X : SQUARES ? m.slot + SLOT_A * slot : m.slot + SLOT_R * slot;
  const char* const Q = gram || !SQUARES ? X : m.slot + SLOT_A * slot;

  // ---- loads: units of 1 KiB, four of each panel per wave, landing swizzled (16-byte chunks of a row XOR-ed)
  uint32_t offp[4], offq[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int u = wave * 4 + i;
    const int r = u * 8 + (lane >> 3), c = (lane & 7) ^ ((r >> 1) & 7);
    offp[i] = r * ldp + c * 16;
    if (SQUARES) {
      offq[i] = r * ldq + c * 16;
    } else {
      const int k = u * 2 + (lane >> 5);
      offq[i] = k * ldq + ((lane & 31) ^ (4 * (k & 3))) * 16;
    }
  }
  const char* p = P + (size_t)m0 * ldp;
  const char* q = SQUARES ? Q + (size_t)n0 * ldq : Q + n0 * 4;
  const size_t q_step = SQUARES ? 128 : (size_t)BK * ldq;
  const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_address(s_ring));
  auto issue = [&](int stage) {
    const uint32_t dst = lds + stage * 2 * PANEL + wave * 4096;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      dma_b128_s(p, offp[i], dst + i * 1024);
      dma_b128_s(q, offq[i], dst + PANEL + i * 1024);
    }
    p += 128;
    q += q_step;
  };
  // ---- fragments: 32 rows, slice kk of 16 K, hi (part 0) or lo (1)
  const int khalf = lane >> 5, lsw = (lane >> 1) & 7;
  auto along = [&](const char* panel, int row, int kk, int part) {
    return *reinterpret_cast<const half8*>(panel + (row + (lane & 31)) * 128 + (((part * 4 + kk * 2 + khalf) ^ lsw) << 4));
  };
  auto across = [&](const char* panel, int col, int kk, int part) -> half8 {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    typedef __attribute__((address_space(3))) s16x4* lds_s16x4_ptr;
    const int blk = lane >> 4, sl = lane & 15, kq = sl >> 2;
    const int c16 = (col >> 5) * 8 + part * 4 + (blk & 1) * 2 + ((sl & 3) >> 1);
    const char* const at = panel + (kk * 16 + (blk >> 1) * 8 + kq) * 512 + ((c16 ^ (4 * kq)) << 4) + (sl & 1) * 8;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(at));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(at + 4 * 512));
    const s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(half8, v);
  };
  f32x16 total[2][2], acc[2][2];
  // acc joins total and starts again.  (A sum of K terms of one sign in one register is off by up to K / 16 * 3 roundings, the
  // diagonal of X X^T at K = 3000 by 1e-6; in parts of 512 it is as good as one of 512.)
  auto join = [&](bool first) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          total[i][j][r] = first ? 0.f : total[i][j][r] + acc[i][j][r];
          acc[i][j][r] = 0.f;
        }
  };
  join(true);

  issue(0);
#pragma unroll 1
  for (int g = 0; g < steps; ++g) {
    __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0): this step's panels are there, the last one's have been read
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (g + 1 < steps) issue((g + 1) & 1);
    const char* const pp = s_ring + (g & 1) * 2 * PANEL;
    const char* const pq = pp + PANEL;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      half8 fp[2][2], fq[2][2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          fp[i][part] = along(pp, wm * 64 + i * 32, kk, part);
          fq[i][part] = SQUARES ? along(pq, wn * 64 + i * 32, kk, part) : across(pq, wn * 64 + i * 32, kk, part);
        }
      // (Q's fragment is the first operand: a lane then holds four neighbouring columns of C)
#pragma unroll
      for (int t = 0; t < 3; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fq[j][t == 0], fp[i][t == 1], acc[i][j], 0, 0, 0);
    }
    if (g % JOIN == JOIN - 1) join(false);
  }
  join(false);

  // ---- result: a lane holds row (lane & 31) and columns 8 b + 4 (lane >> 5) + 0..3, b = 0..3, of every 32 x 32 block
  const Factors f = a.factors[which];
  const char* const E = gram ? nullptr : SQUARES ? m.slot + SLOT_A * slot : X;
  const int ldc = (SQUARES ? mp : np) * 4;
  char* const C = SQUARES ? m.slot + (gram ? SLOT_A : SLOT_R) * slot : m.X[1 - a.x];
  const float out = OUT == OUT_PAIRS ? 1.f : a.bounds[which].out;
  const bool tall = m.rows > m.cols;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int row = m0 + wm * 64 + i * 32 + (lane & 31);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int col = n0 + wn * 64 + j * 32 + b * 8 + khalf * 4;
        const size_t byte = (size_t)row * ldc + pair_byte(col);
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        if (E) load_pair(E + byte, v);
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = f.first * v[r] + f.product * total[i][j][b * 4 + r];
        if constexpr (OUT == OUT_PAIRS) {
          store_pair(C + byte, v);
          if (SQUARES)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum += v[r] * v[r];
        } else {
          typedef std::conditional_t<OUT == OUT_F32, float, bf16_t> T;
          T* const U = static_cast<T*>(m.U);
          if (row < m.m) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (col + r < m.n) U[tall ? (int64_t)(col + r) * m.cols + row : (int64_t)row * m.cols + col + r] = (T)(v[r] * out);
          }
        }
      }
    }
  if (gram) {
    sum = wave_sum(sum);
    __syncthreads();
    float* const part = reinterpret_cast<float*>(s_ring);
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    if (tid == 0) a.squares[blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
  }
}

constexpr size_t align256(size_t v) { return (v + 255) / 256 * 256; }
size_t mat_bytes(int64_t mp, int64_t np) { return (size_t)(2 * mp * np + N_SLOTS * mp * mp) * 4; }
}  // namespace

modse_status ortho_layout(const modse_matrix_set* set, OrthoLayout& w) {
  const int n = set->n_matrices;
  int64_t square = 0, update = 0, parts = 0;
  size_t data = 0;
  for (int i = 0; i < n; ++i) {
    const int r = set->rows[i], c = set->cols[i];
    if (r < 1 || c < 1) return MODSE_ERR_INVALID_ARG;
    if (r > 65536 || c > 65536) return MODSE_ERR_UNSUPPORTED;
    const int64_t mp = padded(r < c ? r : c), np = padded(r < c ? c : r);
    square += mp / PAD * (mp / PAD);
    update += mp / PAD * (np / PAD);
    parts += ((int64_t)r * c + PART - 1) / PART;
    data += mat_bytes(mp, np);
  }
  if (update >= (int64_t)1 << 24) return MODSE_ERR_UNSUPPORTED;  // (a launch has fewer than 2^32 threads)
  w.square_tiles = (int32_t)square;
  w.update_tiles = (int32_t)update;
  w.parts = (int32_t)parts;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off = align256(off + bytes);
    return o;
  };
  w.mats = take(n * sizeof(Mat));
  w.bounds = take(n * sizeof(Bound));
  w.factors = take((size_t)n * 3 * sizeof(Factors));
  w.squares = take((size_t)square * 4);
  w.sums = take((size_t)parts * sizeof(double));
  w.square_map = take((size_t)square * 4);
  w.update_map = take((size_t)update * 4);
  w.data = take(data);
  w.total = n ? off : 0;
  return MODSE_OK;
}

hipError_t launch_orthogonalize(const modse_matrix_set* set, const OrthoLayout& w, const float* coeffs, int steps, float eps, char* ws,
                               hipStream_t s) {
  const int n = set->n_matrices;
  Mat* const table = reinterpret_cast<Mat*>(ws + w.mats);
  Bound* const bounds = reinterpret_cast<Bound*>(ws + w.bounds);
  Factors* const factors = reinterpret_cast<Factors*>(ws + w.factors);  // of the three kinds of products
  Factors *const f_gram = factors, *const f_square = factors + n, *const f_update = factors + 2 * n;
  float* const squares = reinterpret_cast<float*>(ws + w.squares);
  double* const sums = reinterpret_cast<double*>(ws + w.sums);
  int32_t* const square_map = reinterpret_cast<int32_t*>(ws + w.square_map);
  int32_t* const update_map = reinterpret_cast<int32_t*>(ws + w.update_map);
  int32_t square = 0, update = 0, part = 0, most_parts = 0, most_tiles = 0;
  int64_t data = 0;
  hipError_t e;
  for (int first = 0; first < n; first += MATS_PER_LAUNCH) {
    MatArgs a;
    a.table = table;
    a.data = ws + w.data;
    a.first = first;
    a.count = n - first < MATS_PER_LAUNCH ? n - first : MATS_PER_LAUNCH;
    for (int i = 0; i < a.count; ++i) {
      const int r = set->rows[first + i], c = set->cols[first + i];
      const int mp = padded(r < c ? r : c), np = padded(r < c ? c : r);
      const int parts = (int)(((int64_t)r * c + PART - 1) / PART);
      a.mat[i] = {set->G[first + i], set->U[first + i], data, r, c, square, update, part, parts};
      square += mp / PAD * (mp / PAD);
      update += mp / PAD * (np / PAD);
      part += parts;
      data += (int64_t)mat_bytes(mp, np);
      if (parts > most_parts) most_parts = parts;
      if (mp / 64 * (np / 64) > most_tiles) most_tiles = mp / 64 * (np / 64);
    }
    hipLaunchKernelGGL(ortho_table_kernel, dim3(1), dim3(64), 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  hipLaunchKernelGGL(ortho_squares_kernel, dim3(most_parts < 1024 ? most_parts : 1024, n), dim3(256), 0, s, table, sums);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL(ortho_prepare_kernel, dim3(n), dim3(256), 0, s, table, sums, eps, bounds, f_gram, square_map, update_map);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL(ortho_start_kernel, dim3(most_tiles < 2048 ? most_tiles : 2048, n), dim3(256), 0, s, table, bounds);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  for (int i = 0; i < steps; ++i) {
    ProductArgs a = {table, f_gram, bounds, squares, square_map, OP_GRAM, i & 1};
    const dim3 block(256);
    const float* const c = coeffs + 3 * i;
    hipLaunchKernelGGL((ortho_product_kernel<true, OUT_PAIRS>), dim3(w.square_tiles), block, 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(ortho_factors_kernel, dim3(n), dim3(64), 0, s, table, squares, c[0], c[1], c[2], bounds, f_square, f_update, f_gram);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    a.kind = OP_SQUARE;
    a.factors = f_square;
    hipLaunchKernelGGL((ortho_product_kernel<true, OUT_PAIRS>), dim3(w.square_tiles), block, 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    a.kind = OP_UPDATE;
    a.factors = f_update;
    a.map = update_map;
    const dim3 grid(w.update_tiles);
    if (i + 1 < steps) hipLaunchKernelGGL((ortho_product_kernel<false, OUT_PAIRS>), grid, block, 0, s, a);
    else if (set->dtype == MODSE_F32) hipLaunchKernelGGL((ortho_product_kernel<false, OUT_F32>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((ortho_product_kernel<false, OUT_BF16>), grid, block, 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  return hipSuccess;
}
