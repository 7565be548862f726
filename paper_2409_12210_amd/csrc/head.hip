// Log probabilities of the next tokens from the last hidden rows and the output matrix, without the logits of a whole batch, and their
// gradients.
//
//   l = x W^T,  log Z_t = log sum_v e^l_tv,  logp_t = l_t,target - log Z_t
//   G_tv = w_t (1[v = target_t] - e^(l_tv - log Z_t)),  dX = G W,  dW = G^T x
//
// The batch is taken in pieces of rows whose G fits a workspace that stops growing with the batch.  The products are those of the grouped GEMM kernels,
// whose problem tables one launch makes for sixteen pieces.  dX is a product over the whole vocabulary with few columns, so its
// sum is cut into parts that fill the chip; the parts are float32 slabs that a last launch adds up in order.
//
// The product of the logits leaves, for every row and 32 to 128 columns, their maximum and sum of exponentials, and the target's logit
// (EPI_LOGITS); one launch joins them.  Without gradients no logit is stored.  With gradients the logits are, in float32, and another
// launch turns them into G.
//
// float32 from some hundred rows on: x, W and G are held as the sums of two float16 matrices, hi + lo, times powers of two (see HeadRange)
// that bring the largest value below 2^15.  Three products of float16 matrices, hi hi' + hi lo' + lo hi', in one accumulator leave
// out 2^-22 of a product; they take 3 of the 16-bit matrix rate where float32 instructions take 16 (1021 x 256 x 50257 with gradients:
// 450 us in place of 731).  Fewer rows, or a W of more than 2^28 elements: products in float32, and G in the place of the logits.  Where the device finds
// values in W that its parts would lose, the products with W are in float32, too: by a second list of tiles, of which one is empty.
//
// Up to 64 rows (small vocabularies: more) a stream over W makes the logits, see "few rows".  dW of a small vocabulary has few tiles,
// so its sum over the tokens is cut into parts as well (float32, 1000 x 512, 4096 rows: with the stream 150 us in place of 337 for the whole call).
//
// dX of a bf16 layer takes G as the sum of two bf16 numbers, which hold 16 bits, in two passes over W; what they lose lies below the rounding
// of the result.  (One number, with what it loses of the target's entry put back in float32: 2 T V d operations less, but where another token
// has most of the probability an error of 2.0e-3 of the norm, of which the rounding of the result is 1.65e-3.)  Up to 128 rows, which fill half a
// tile, the second numbers are rows of their own.  dW is float32, and takes G as the sum of two float16 numbers, hi + lo, which hold 22
// bits, times float16 copies of the rows of x, so that what is rounded or lost lies below 2^-39 of the largest product of a row's two factors.
// (Two bf16 numbers, 16 bits, left an error of 2.7e-6 of dW where float32 products have 0.7e-6 to 2e-6; the rest takes as long.)
#include <cmath>
#include <cstddef>

#include "ops.h"

#include "gemm_bf16_util.h"
#include "gemm_plan.h"

namespace {
using namespace modse_gemm;

constexpr int64_t GRAD_CELLS = (int64_t)1 << 28;   // values of G in the workspace (float32: of logits)
constexpr int64_t PAIR_W = (int64_t)1 << 28;       // elements of W of which the parts are kept
constexpr int64_t PAIR_CELLS = (int64_t)1 << 27;   // pairs of 128 columns in it (float32: of 32)
constexpr int64_t W_PART = (int64_t)1 << 30;       // elements of W that one problem reads (kernels count them in 32 bits)
constexpr size_t ALIGN = 256;                      // of what is in the workspace, which itself may lie at any sixteen bytes
constexpr int64_t SLAB_CELLS = (int64_t)1 << 26;   // values of all parts of dX together, unless one part has more
constexpr int64_t STACK_ROWS = 128;                // of bf16 layers up to which the second numbers of G are rows of their own in the product of dX
constexpr int PLAN_PIECES = 16;                    // of which the problem tables, 25 KB a product, are there at a time
constexpr int MAX_PARTS = 128;                     // of dX, of dW (problems of a product: fewer than 192)
static_assert(MAX_PARTS <= MODSE_MAX_PROBLEMS, "a problem for each");

struct HeadShape {
  int64_t T;
  int32_t d, vocab, ldv;   // ldv: distance of rows of logits and G
  int32_t rows, pieces;    // rows of a piece (the last one may have fewer)
  int32_t w_parts, w_rows; // problems of the logits, rows of W in each
  int32_t dx_rows;         // rows of the product of dX: those of a piece, or twice as many
  int32_t k_parts, k_len;  // problems of dX, columns of G in each
  int32_t w_split, w_len;  // problems of dW, rows in each
  int32_t bf16, grad;
  int32_t pairs;           // float32, and the matrices are held as pairs of float16 ones
  int32_t wide;            // either of them: 16-bit products, tiles of 256 or 128
  TileShape logits_tile, dx_tile, dw_tile;
  __host__ __device__ int pair_cols() const { return logits_tile.bn / 2; }  // columns of a pair of maximum and sum
};

int32_t padded_rows(int64_t n) { return (int32_t)align_up((size_t)n, 32); }
// the most rows of a buffer of so many cells, `per_row` of them a row: a power of two from 256 to 65536
int64_t rows_in(int64_t cells, int64_t per_row) {
  int64_t r = 256;
  while (r < 65536 && 2 * r * per_row <= cells) r *= 2;
  return r;
}
int64_t most_rows(int32_t vocab, bool bf16, bool pairs, bool grad) {
  if (grad || !(bf16 || pairs)) return rows_in(GRAD_CELLS, (int64_t)align_up(vocab, 64));
  return bf16 ? rows_in(PAIR_CELLS, (vocab + 127) / 128) : rows_in(PAIR_CELLS, (vocab + 31) / 32);
}
// Float32 layers: the rows from which on products of pairs of float16 numbers are faster, three 16-bit products in place of one of float32,
// with the largest values and the parts of W (and some launches) before them.  At 105 and 1150 TFLOP/s, 5 TB/s and tiles that are 128 rows too
// high on average.  Float32 / pairs, us: gradients with 32000 x 2048, 256 rows 828 / 567, 1024 3045 / 1189; with 50257 x 256, 256 rows 217 / 187,
// 1024 721 / 448; with 4097 x 64, 5000 rows 222 / 200; scoring with 32000 x 2048, 256 rows 264 / 277, 512 514 / 320; with 50257 x 256, 300 rows 81 / 90,
// 400 106 / 103.
int64_t pairs_from(int32_t d, int32_t vocab, bool grad) {
  const double cells = (double)vocab * d, products = grad ? 6 : 2;
  const double fixed = 3 * products * 128 * cells / 1.15e9 + 12 * cells / 5e6 + (grad ? 50 : 35);
  return std::max<int64_t>(129, (int64_t)std::ceil(fixed / (products * cells * (1 / 1.05e8 - 3 / 1.15e9))));
}
bool takes_pairs(int64_t T, int32_t d, int32_t vocab, modse_dtype dt, bool grad) {
  return dt == MODSE_F32 && (int64_t)vocab * d <= PAIR_W && T >= pairs_from(d, vocab, grad);
}
// Up to so many rows the logits are made by a stream over W (below): blocks of 64 rows of each, while there are two for every CU at the most, or
// one block of rows.
constexpr int STREAM_W = 64;
int64_t stream_rows(int32_t vocab) { return std::max<int64_t>(1, 512 / ((vocab + STREAM_W - 1) / STREAM_W)) * 64; }
int64_t tiles(int64_t m, int64_t n, int b) { return ((m + b - 1) / b) * ((n + b - 1) / b); }
// 16-bit products: the logits take tiles of 128, two of which share a CU, where tiles of 256 are few or a tile is but a few steps of K.  Tiles of
// 256 / 128, us: 128 rows with 32000 x 2048 54 / 36, 131072 x 128 41 / 22; 229 rows with 32000 x 2048 55 / 51, 50257 x 2048 69 / 88, 131072 x
// 128 35 / 30; 512 rows with 32000 x 1024 44 / 53, 131072 x 512 86 / 88, 50257 x 256 38 / 33, 4096 rows 177 / 157; with gradients 512
// rows x 50257 x 256 221 / 210, 2048 rows 631 / 642.  Float32 by pairs, gradients: 300 rows with 8000 x 1024 202 / 171, 1021 rows 275 / 257, 2048
// rows 372 / 399, 1021 rows with 50257 x 256 478 / 449, 2048 rows 768 / 768, scored 4096 rows 415 / 443.
constexpr int64_t BLOCK_ROWS = 256, BLOCK_ROWS_MOST = 1024, FEW_TILES = 128;
bool logits_take_blocks(int64_t T, int32_t d, int32_t vocab, bool all_rows) {
  return T <= 128 || tiles(T, vocab, 256) <= FEW_TILES || (d <= 256 && (all_rows || T <= BLOCK_ROWS_MOST));
}
// dX takes them up to 256 rows, and with short rows up to 1024 (one row with 32000 x 2048 167 / 137, 50257 x 256 78 / 56; 229 rows 287 / 292, 140 / 122;
// 512 rows 405 / 464, 217 / 204; float32, 512 rows with 32000 x 512 302 / 278, 1021 rows 427 / 482, 512 rows with 32000 x 2048 745 / 862), dW
// of bf16 layers up to 64 rows and where tiles of 256 do not fill the chip and are a few steps of K each: one row with 32000 x 2048 135 / 122, 128 rows
// with 131072 x 512 252 / 267; 1024 rows with 1000 x 1024 97 / 80, 4000 x 512 105 / 98, 8000 x 1024 168 / 178.
bool dx_takes_blocks(int64_t T, int32_t d, bool pairs) {
  return pairs ? T <= 512 && d <= 512 : T <= BLOCK_ROWS || (d <= 256 && T <= BLOCK_ROWS_MOST);
}
bool dw_takes_blocks(int64_t T, int64_t tiles_256) { return T <= 64 || (tiles_256 <= FEW_TILES && T * tiles_256 <= 256 * FEW_TILES); }
// pairs of maximum and sum for so many rows of any batch
size_t pair_cells(int64_t rows, int32_t d, int32_t vocab, bool bf16) {
  auto of = [&](int64_t n, int cols) { return (size_t)n * ((vocab + cols - 1) / cols); };
  const int64_t block_rows = d > 256 ? std::max<int64_t>(128, FEW_TILES / tiles(1, vocab, 256) * 256) : rows;
  return bf16 ? std::max(of(rows, 128), of(std::min(rows, block_rows), 64)) : of(rows, 32);
}
// Parts of dW's sum over the tokens, where it has too few tiles for the chip: slabs like those of dX, added up behind it.
int64_t dw_most_parts(int32_t d, int32_t vocab, bool wide) {
  const int64_t tiles = (int64_t)((vocab + 255) / 256) * ((d + 255) / 256);
  return wide && tiles <= 128 ? std::min<int64_t>(MAX_PARTS, 256 / tiles) : 1;
}

// (plain: the products in float32 of a call that takes pairs)
HeadShape head_shape(int64_t T, int32_t d, int32_t vocab, modse_dtype dt, bool grad, bool plain = false) {
  HeadShape h = {};
  h.T = T;
  h.d = d;
  h.vocab = vocab;
  h.bf16 = dt == MODSE_BF16;
  h.grad = grad;
  const bool pairs = takes_pairs(T, d, vocab, dt, grad);
  h.pairs = pairs && !plain;
  h.wide = h.bf16 || h.pairs;
  h.ldv = (int32_t)align_up(vocab, 64);
  // Pieces of about one size, whole tiles of 256: a last one of a few rows would go over all of W and dW for them.  Gradients of 8193 rows with
  // 32000 x 2048, as 8192 + 1 / 4352 + 3841: bf16 5850 / 4975 us, float32 9870 / 8320; 2049 rows with
  // 131072 x 2048, 2048 + 1 / 1280 + 769: 6580 / 5660, 11170 / 9710.
  const int64_t most = most_rows(vocab, h.bf16, pairs, grad);
  h.pieces = (int32_t)((T + most - 1) / most);
  h.rows = h.pieces == 1 ? padded_rows(T) : (int32_t)align_up((size_t)((T + h.pieces - 1) / h.pieces), 256);
  h.pieces = (int32_t)((T + h.rows - 1) / h.rows);
  h.w_rows = (int32_t)std::min<int64_t>(vocab, W_PART / d / 256 * 256);
  h.w_parts = (vocab + h.w_rows - 1) / h.w_rows;
  // (float32: tiles of 128 from four rounds of the chip's 512 workgroups on.  50304 x 256, 1.5 rounds: 287 us with them, 258 with tiles of
  // 64; 1021 x 50257, 6.1 rounds: 251 and 261)
  auto tile = [&](int64_t m, int64_t n) { const int b = h.wide ? 256 : tiles(m, n, 128) >= 2048 ? 128 : 64; return TileShape{b, b}; };
  h.logits_tile = plain || (h.wide && logits_take_blocks(T, d, vocab, h.bf16 && !grad)) ? TileShape{128, 128} : tile(h.rows, vocab);
  h.dw_tile = h.bf16 && dw_takes_blocks(T, tiles(vocab, d, 256)) ? TileShape{128, 128} : tile(vocab, d);
  const int64_t w_steps = (h.rows + 63) / 64, w_split = std::min(dw_most_parts(d, vocab, h.wide), std::max<int64_t>(1, w_steps / 4));
  h.w_len = (int32_t)((w_steps + w_split - 1) / w_split) * 64;
  h.w_split = (h.rows + h.w_len - 1) / h.w_len;
  const int dx = h.wide && dx_takes_blocks(T, d, h.pairs) ? 128 : h.wide ? 256 : h.rows <= 64 ? 64 : 128;
  h.dx_tile = TileShape{dx, dx};
  // Parts of dX: whole rounds of workgroups over the chip, each part with six further steps for its opening and its end, and slabs that
  // are written and read.
  h.dx_rows = h.bf16 && T <= STACK_ROWS ? 2 * h.rows : h.rows;
  const int64_t out = tiles(h.dx_rows, d, h.dx_tile.bm), steps = (vocab + 63) / 64, slots = dx == 256 ? 256 : 512;
  const int64_t parts_most = std::min<int64_t>({MAX_PARTS, steps, std::max<int64_t>(1, SLAB_CELLS / ((int64_t)h.dx_rows * d))});
  double best = 0;
  for (int64_t n = 1; n <= parts_most; ++n) {
    const int64_t len = (steps + n - 1) / n, parts = (steps + len - 1) / len;
    const double step_us = h.wide ? (h.pairs ? 3 : 1) * (dx == 128 ? 1.0 : 1.6) : dx == 64 ? 3.0 : 8.0;
    const int64_t passes = h.bf16 && h.dx_rows == h.rows ? 2 : 1;  // (over K, of one length)
    const double us = (double)((out * parts + slots - 1) / slots) * (passes * len + 6) * step_us + parts * (double)h.dx_rows * d * 8 / 4e6;
    if (n == 1 || us < best) {
      best = us;
      h.k_parts = (int32_t)parts;
      h.k_len = (int32_t)len * 64;
    }
  }
  return h;
}

// Float16 numbers hold 2^15 to 2^-25, so what is taken in two of them goes by powers of two, of which the results are freed again.
// A row of x: by its largest value, for its logits (no row touches another).  W: by its largest value.  A row of G: by the most that an entry of it can be,
// |w| (1 - p_target), for dX and dW.  dW sums over the rows, so there the rows of x make up for those of G: row t of G times 2^r_t, row t of x
// times 2^(C - r_t), with one C from the largest |w_t| (1 - p_target) max|x_t| so far in the call.
constexpr int RANGE_BLOCKS = 512;
constexpr int NO_ROW = -(1 << 20);
constexpr int MOST_LINES = 64;  // that many blocks or rows change together, each in a line of its own (2048 rows one number: 15 us)
struct HeadRange {
  uint32_t w_of[RANGE_BLOCKS];  // the largest |W|, as the bits of a float, by block (of a NaN more than those of an infinity)
  int32_t counts[MOST_LINES][32];   // [i][0 .. 2], of every 64th block: values of W that are not 0, those below 2^-20 and 2^-30 of its largest
  int32_t w_exponent;  // W is taken times 2 to it
  int32_t plain;       // the products with W are in float32
  float undo_dw[2];    // 2^-C, in two factors
  int32_t most[MOST_LINES][32];  // [i][0]: exponent of the largest |w_t| (1 - p_target) max|x_t| so far of every 64th row, or NO_ROW
  float pad[3];
  float undo_w;  // right before the targets' logits (EPI_LOGITS_PAIRS)
};
static_assert(sizeof(HeadRange) == offsetof(HeadRange, undo_w) + 4 && sizeof(HeadRange) % 16 == 0, "laid out up to the targets' logits");
// floor(log2) of a float of so many bits; -127 of what is smaller than all normal ones
__device__ __forceinline__ int exponent_of(uint32_t bits) { return (int)(bits >> 23 & 255) - 127; }
// the power of two that brings values of at most this size below 2^15
__device__ __forceinline__ int scale_exponent(uint32_t bits) { return min(14 - exponent_of(bits), 120); }
__device__ __forceinline__ float power_of_two(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }
// Times 2^e, any e: of NaN and infinities what they are, 0 below the smallest number.
__device__ __forceinline__ float times_2(float x, int e) { return __builtin_amdgcn_ldexpf(x, e); }
// C.  An entry of G lies below 2^(e_t + 2), e_t as in row_exponent, and is taken times 2^(13 - e_t); one of x, below 2^(f_t + 1), times 2^(C - 13 + e_t):
// with C = 27 - max(e_t + f_t) both lie below 2^15.  (Where C would be more than 250, dW lies below the smallest float.)
__device__ __forceinline__ int common_exponent(const HeadRange* range) {  // (by a wave)
  int most = range->most[threadIdx.x % MOST_LINES][0];
#pragma unroll
  for (int o = 32; o; o >>= 1) most = max(most, __shfl_xor(most, o, 64));
  return most == NO_ROW ? 0 : min(27 - most, 250);
}

typedef _Float16 f16_t;
typedef f16_t f16x8 __attribute__((ext_vector_type(8)));

struct HeadBufs {
  GemmPlan* plans;   // logits of some pieces, then dX and dW of each of them
  float* logits;     // [rows, ldv]; float32 layers: then G
  float* pairs;      // [ceil(vocab / pair_cols)][rows] maximum and sum
  float* at_target;  // [rows] the target's logit, and behind them [rows] what undoes the scaling of a row of x (float32 by pairs)
  float* off;        // [rows][2] the row's maximum and log2 of its sum
  bf16_t* g;         // [2 rows, ldv] G, and behind its rows what bf16 lacks of them
  f16_t *hi, *lo;    // [rows, ldv] G in two parts, scaled
  f16_t *x16, *x16_lo;   // [rows, d] x in the same way, for dW; x16_lo: float32 layers, there for the logits before
  int32_t* exponents;    // [rows] rows of G are taken times 2 to it
  f16_t *w16, *w16_lo;   // [vocab, d] W, float32 layers
  float* x32;        // [rows, d] x, zeros in rows without a target: float32 layers that take no pairs
  HeadRange* range;
  float* slabs;      // [k_parts][dx_rows, d]
};

struct HeadPlanArgs {
  HeadShape h;
  HeadBufs b;
  const void *x, *W;
  const int32_t* targets;
  const float* d_logp;
  float* dW;
  HeadShape plain;     // of a call that takes pairs: its products with W in float32
  int32_t first, pieces, tables;  // pieces whose problems are made, the first of them; their products
  int32_t x_first, x_rows;        // rows of x that are split
  int32_t range_blocks;
};
enum HeadProduct { LOGITS, DX, DW, PLAIN_LOGITS, PLAIN_DX };
// The products of a piece that a call has tables for, and the i-th of them.
__host__ __device__ inline int head_products(const HeadShape& h) { return (h.grad ? 3 : 1) + (h.pairs ? h.grad ? 2 : 1 : 0); }
__host__ __device__ inline int head_product(const HeadShape& h, int i) { return h.grad || i == 0 ? i : PLAIN_LOGITS; }
__host__ __device__ inline int head_table(const HeadShape& h, int product) { return h.grad || product == LOGITS ? product : 1; }

// Infinities and NaN count as 0: they stay what they are in the parts, and the other values keep theirs.
__device__ __forceinline__ uint32_t finite(uint32_t bits) { return (bits & 0x7fffffffu) < 0x7f800000u ? bits & 0x7fffffffu : 0; }
__device__ __forceinline__ uint32_t largest(u32x4 v, bool bf16) {
  uint32_t most = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) most = max(most, bf16 ? max(finite(v[e] << 16), finite(v[e] & 0xffff0000u)) : finite(v[e]));
  return most;
}
// of sixteen-byte vectors, every `step`th from `first` on
__device__ __forceinline__ uint32_t largest(const u32x4* v16, int64_t vectors, bool bf16, int64_t first, int64_t step) {
  uint32_t most = 0;
  for (int64_t i = first; i < vectors; i += 4 * step) {
    u32x4 v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = v16[i + q * step < vectors ? i + q * step : i];
#pragma unroll
    for (int q = 0; q < 4; ++q) most = max(most, largest(v[q], bf16));
  }
  return most;
}
// lanes that share a row of so many vectors: a power of two
__device__ __forceinline__ int lanes_of(int vectors) { return vectors >= 64 ? 64 : 1 << (32 - __builtin_clz(max(vectors, 2) - 1)); }
__device__ __forceinline__ uint32_t wave_most(uint32_t v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  return v;
}
// float32 by pairs: W's largest value; clears the counts.
__global__ __launch_bounds__(1024) void head_range_kernel(const u32x4* W, int64_t vectors, HeadRange* range) {
  __shared__ uint32_t s_most[16];
  if (blockIdx.x == 0 && threadIdx.x < 3 * MOST_LINES) range->counts[threadIdx.x / 3][threadIdx.x % 3] = 0;
  uint32_t most = 0;
  for (int64_t i = (int64_t)blockIdx.x * 1024 + threadIdx.x; i < vectors; i += (int64_t)gridDim.x * 4096) {
    u32x4 v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t at = i + q * (int64_t)gridDim.x * 1024;
      v[q] = W[at < vectors ? at : i];
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e) most = max(most, v[q][e] & 0x7fffffffu);
  }
  most = wave_most(most);
  if ((threadIdx.x & 63) == 0) s_most[threadIdx.x >> 6] = most;
  __syncthreads();
  if (threadIdx.x > 0) return;
  for (int w = 1; w < 16; ++w) most = max(most, s_most[w]);
  range->w_of[blockIdx.x] = most;
}
// By a wave: the bits of the largest |W|, those of an infinity or more where not all values are finite.
__device__ __forceinline__ uint32_t largest_w(const HeadRange* range, int blocks) {
  uint32_t most = 0;
  for (int i = threadIdx.x & 63; i < blocks; i += 64) most = max(most, range->w_of[i]);
  return wave_most(most);
}
__device__ __forceinline__ int wave_total(int v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
// What lies 2^-40 below W's largest value is lost by pairs.  Where that is more than a rounding of values that count, as beside a few far larger rows (which
// keep columns out by a constant in x, say), the products with W are in float32 instead: where more than 1 of 256 values other than 0 are below 2^-20 of the largest,
// or more than 1 of 16384 below 2^-30 (normal values: below 1e-5 and 1e-8 of them), or not all are finite.  By a wave.
__device__ __forceinline__ bool w_takes_float32(const HeadRange* range, uint32_t most) {
  int n[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) n[k] = wave_total(range->counts[threadIdx.x % MOST_LINES][k]);
  return most >= 0x7f800000u || n[1] > n[0] / 256 || n[2] > n[0] / 16384;
}
// What a row's G and x are taken times, once its statistics are there: by the first wave of those that call it.  `largest_x`: of the row's finite values.
// (1 - p as it is computed, of a p that may be rounded to 1.)  Rows without a gradient have no part in C, and their copies of x are 0.
__device__ __forceinline__ int row_exponent(HeadRange* range, int row, float w, float p, uint32_t largest_x) {
  const uint32_t size = __builtin_bit_cast(uint32_t, w) & 0x7fffffffu;
  if (size == 0 || size >= 0x7f800000u) return -NO_ROW;
  const int e = exponent_of(size) + exponent_of(__builtin_bit_cast(uint32_t, fmaxf(1.f - p, 0x1p-23f)));
  atomicMax(&range->most[row % MOST_LINES][0], e + exponent_of(largest_x));  // (the order does not matter)
  return 13 - e;
}

// float32 by pairs: eight elements in two parts
__device__ __forceinline__ void put_parts(const f32x4 (&v)[2], int exponent, f16_t* hi, f16_t* lo) {
  f16x8 h, l;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float x = times_2(v[e >> 2][e & 3], exponent);
    h[e] = (f16_t)x;
    l[e] = (f16_t)(x - (float)h[e]);
  }
  *reinterpret_cast<f16x8*>(hi) = h;
  *reinterpret_cast<f16x8*>(lo) = l;
}
// W's parts, of n elements (a multiple of 8).  Every block joins the largest values for itself.
__global__ __launch_bounds__(256) void head_split_w_kernel(const float* W, int64_t n, f16_t* hi, f16_t* lo, HeadRange* range, int blocks) {
  __shared__ uint32_t s_most;
  __shared__ int s_n[3][4];
  if (threadIdx.x < 64) {
    const uint32_t most = largest_w(range, blocks);
    if (threadIdx.x == 0) s_most = most < 0x7f800000u ? most : 0;
  }
  __syncthreads();
  const int exponent = scale_exponent(s_most);
  const float most = __builtin_bit_cast(float, s_most), small = most * 0x1p-20f, smaller = most * 0x1p-30f;
  int count[3] = {};
  const int64_t step = (int64_t)gridDim.x * 2048;
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8; i < n; i += step) {
    const f32x4 v[2] = {__builtin_nontemporal_load(reinterpret_cast<const f32x4*>(W + i)),
                        __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(W + i + 4))};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float size = fabsf(v[e >> 2][e & 3]);
      count[0] += size > 0.f;
      count[1] += size > 0.f && size < small;
      count[2] += size > 0.f && size < smaller;
    }
    put_parts(v, exponent, hi + i, lo + i);
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    count[k] = wave_total(count[k]);
    if ((threadIdx.x & 63) == 0) s_n[k][threadIdx.x >> 6] = count[k];
  }
  __syncthreads();
  if (threadIdx.x >= 3) return;
  int sum = 0;
  for (int w = 0; w < 4; ++w) sum += s_n[threadIdx.x][w];
  if (sum) atomicAdd(&range->counts[blockIdx.x % MOST_LINES][threadIdx.x], sum);
}
// Rows of x of a piece, some lanes of a wave each, by their own largest values.
__device__ __forceinline__ void split_x(const HeadPlanArgs& a, int block) {
  const int d = a.h.d, lanes = lanes_of(d / 8), lane = threadIdx.x & (lanes - 1);
  const int64_t row = ((int64_t)block * 256 + threadIdx.x) / lanes;
  if (row >= a.x_rows) return;
  const int64_t at = row * d;
  const float* const x = static_cast<const float*>(a.x) + (int64_t)a.x_first * d;
  uint32_t most = largest(reinterpret_cast<const u32x4*>(x + at), d / 4, false, lane, lanes);
  for (int o = lanes / 2; o; o >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o, 64));
  const int e = scale_exponent(most);
  if (lane == 0) a.b.at_target[a.h.rows + row] = power_of_two(-e);
  for (int c = lane * 8; c < d; c += lanes * 8) {
    const f32x4 v[2] = {*reinterpret_cast<const f32x4*>(x + at + c), *reinterpret_cast<const f32x4*>(x + at + c + 4)};
    put_parts(v, e, a.b.x16 + at + c, a.b.x16_lo + at + c);
  }
}

// The problems of one product of one piece, by a block's first wave.  Of the products by pairs and those in float32 one has no tiles.  Blocks behind
// these split rows of x.
__global__ __launch_bounds__(256) void head_plan_kernel(HeadPlanArgs a) {
  __shared__ int s_tiles[MODSE_MAX_PROBLEMS];
  const HeadShape& h = a.h;
  if ((int)blockIdx.x >= a.tables) {
    split_x(a, blockIdx.x - a.tables);
    return;
  }
  if (threadIdx.x >= 64) return;
  const int lane = threadIdx.x;
  const uint32_t most = h.pairs ? largest_w(a.b.range, a.range_blocks) : 0;
  const bool takes_float32 = h.pairs && w_takes_float32(a.b.range, most);
  if (a.first == 0 && blockIdx.x == 0 && a.b.range) {
    a.b.range->most[lane][0] = NO_ROW;
    if (lane == 0) {
      a.b.range->w_exponent = scale_exponent(most);
      a.b.range->plain = takes_float32;
      a.b.range->undo_w = power_of_two(-scale_exponent(most));
    }
  }
  const int which = head_product(h, (int)blockIdx.x / a.pieces);
  const int64_t t0 = (int64_t)(a.first + (int)blockIdx.x % a.pieces) * h.rows;
  const size_t es = h.bf16 ? 2 : 4;
  const int m = (int)min((int64_t)h.rows, h.T - t0);
  const char* const x = cadd(a.x, (size_t)t0 * h.d * es);
  GemmPlan* const plan = a.b.plans + blockIdx.x;
  const bool plain = which == PLAIN_LOGITS || which == PLAIN_DX, active = which == DW || plain == takes_float32;
  const int n = which == LOGITS || which == PLAIN_LOGITS ? h.w_parts : which == DX ? h.k_parts : which == PLAIN_DX ? a.plain.k_parts : h.w_split;
  for (int p = lane; p < n; p += 64) {
    GemmProblem P = {};
    TileShape t;
    if (which == LOGITS || which == PLAIN_LOGITS) {
      const int v0 = p * h.w_rows;
      P.A = x;
      P.B = cadd(a.W, (size_t)v0 * h.d * es);
      if (h.pairs && !plain) {
        P.A = a.b.x16;
        P.A2 = a.b.x16_lo;
        P.B = a.b.w16 + (size_t)v0 * h.d;
        P.B2 = a.b.w16_lo + (size_t)v0 * h.d;
      }
      if (h.grad) P.C = a.b.logits + v0;
      P.C2 = a.b.pairs;
      P.C3 = a.b.at_target;
      P.E1 = a.targets + t0;
      P.E2 = reinterpret_cast<const void*>((uint64_t)h.rows << 32 | (uint32_t)v0);
      P.M = m; P.N = min(h.w_rows, h.vocab - v0); P.K = h.d;
      P.lda = h.d; P.ldb = h.d; P.ldc = h.ldv;
      t = plain ? a.plain.logits_tile : h.logits_tile;
    } else if (which == DX || which == PLAIN_DX) {
      const int k_len = plain ? a.plain.k_len : h.k_len, v0 = p * k_len;
      P.A = h.bf16 ? (const void*)(a.b.g + v0) : (const void*)(a.b.logits + v0);
      P.B = cadd(a.W, (size_t)v0 * h.d * es);
      if (h.pairs && !plain) {
        P.A = a.b.hi + v0;
        P.A2 = a.b.lo + v0;
        P.B = a.b.w16 + (size_t)v0 * h.d;
        P.B2 = a.b.w16_lo + (size_t)v0 * h.d;
      }
      if (h.bf16 && h.dx_rows == h.rows) {
        P.A2 = a.b.g + (size_t)h.rows * h.ldv + v0;
        P.B2 = P.B;
      }
      P.C = a.b.slabs + (size_t)p * h.dx_rows * h.d;
      P.M = h.dx_rows > h.rows ? h.dx_rows : m; P.N = h.d; P.K = min(k_len, h.vocab - v0);
      P.lda = h.ldv; P.ldb = h.d; P.ldc = h.d;
      t = plain ? a.plain.dx_tile : h.dx_tile;
    } else {
      const int r0 = p * h.w_len;  // (behind the last piece's rows: a part of zeros)
      const size_t g0 = (size_t)r0 * h.ldv, x0 = (size_t)r0 * h.d;
      P.A = h.wide ? (const void*)(a.b.hi + g0) : (const void*)a.b.logits;
      P.A2 = a.b.lo + g0;
      P.B = P.B2 = h.wide ? (const void*)(a.b.x16 + x0) : a.b.x32;
      if (h.pairs) P.B2 = a.b.x16_lo + x0;
      P.E1 = a.b.range ? a.b.range->undo_dw : nullptr;
      P.C = h.w_split > 1 ? a.b.slabs + (size_t)p * h.vocab * h.d : a.dW;
      P.E2 = reinterpret_cast<const void*>((intptr_t)h.vocab);
      P.M = (h.vocab + 31) / 32 * 32; P.N = h.d; P.K = max(min(h.w_len, m - r0), 0);
      P.lda = h.ldv; P.ldb = h.d; P.ldc = h.d;
      t = h.dw_tile;
    }
    const int tiles = set_tiles(P, t.bm, t.bn);
    s_tiles[p] = active ? tiles : 0;
    plan->prob[p] = P;
  }
  wave_lds_order();
  finish_plan(plan, lane, n, s_tiles);
}

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

struct HeadRowsArgs {
  const int32_t* targets;  // of the product's first row
  const float* d_logp;
  float *logp, *log_z;     // of the product's first row, either may be null
  float* logits;
  const float *pairs, *at_target;
  float* off;
  bf16_t *g, *g_rest;      // of the product's first row; null where there is no dX
  f16_t *hi, *lo;          // null where there is no dW
  HeadRange* range;        // (16-bit products) or null
  int32_t* exponents;
  const void* x;           // of the product's first row, and their copies for dW, with zeros in rows without a target
  f16_t *x16, *x16_lo;     // x16_lo: null of bf16 layers
  float* x32;              // (float32 layers) null where there is no dW
  int32_t rows, vocab, ldv, pair_rows, pair_cols, plain_cols, d;  // plain_cols: those of the products in float32 of a call that takes pairs, or 0
};
__device__ __forceinline__ float row_weight(int32_t target, int vocab, const float* d_logp) {
  return target < 0 ? 0.f : target >= vocab ? __builtin_nanf("") : *d_logp;
}
__device__ __forceinline__ uint32_t row_largest(const void* x, int64_t row, int d, bool bf16) {  // (by a wave)
  const int vectors = bf16 ? d / 8 : d / 4;
  return wave_most(largest(static_cast<const u32x4*>(x) + row * vectors, vectors, bf16, threadIdx.x & 63, 64));
}
// (by maximum and sum, not by log Z: of a row that is all but sure 1 - p is what counts, and log Z is rounded at the size of the logits)
__device__ __forceinline__ float probability(float logit, float top, float log2_sum) {
  return __builtin_amdgcn_exp2f(fmaf(logit - top, LOG2E, -log2_sum));
}
__device__ __forceinline__ float grad_of(float logit, float top, float log2_sum, float w, int32_t target, int c, int vocab) {
  const float p = probability(logit, top, log2_sum);
  return c >= vocab || target < 0 ? 0.f : c == target ? w * (1.f - p) : -w * p;
}
__device__ __forceinline__ void put_row(float* logp, float* log_z, int32_t target, int vocab, float at_target, float top, float log_sum) {
  if (logp) *logp = target < 0 ? 0.f : target >= vocab ? __builtin_nanf("") : at_target - top - log_sum;
  if (log_z) *log_z = top + log_sum;
}
__device__ __forceinline__ void put_row(const HeadRowsArgs& a, int row, int32_t target, float at_target, float top, float log_sum) {
  put_row(a.logp ? a.logp + row : nullptr, a.log_z ? a.log_z + row : nullptr, target, a.vocab, at_target, top, log_sum);
}

// Joins the pairs of sixteen rows.  Sixteen waves of four quarters, each quarter takes every 64th pair of the rows.  (A lane for each of 64 rows
// kept a call of 128 rows x 50257 waiting for two blocks: 42 us in place of 56.)
__global__ __launch_bounds__(1024) void head_stats_kernel(HeadRowsArgs a) {
  __shared__ float s_m[64][16], s_s[64][16];
  __shared__ uint32_t s_x[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, quarter = threadIdx.x >> 4;
  const int row = blockIdx.x * 16 + (lane & 15), pair_cols = a.plain_cols && a.range->plain ? a.plain_cols : a.pair_cols, n = (a.vocab + pair_cols - 1) / pair_cols;
  constexpr int AHEAD = 4;
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  float m = LOWEST, s = 0.f;
  if (row < a.rows) {
    for (int p = quarter; p < n; p += 64 * AHEAD) {
      f32x2 v[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        v[i] = *reinterpret_cast<const f32x2*>(a.pairs + ((int64_t)min(p + i * 64, n - 1) * a.pair_rows + row) * 2);
      float most = m;
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) most = fmaxf(most, v[i][0]);
      s *= __builtin_amdgcn_exp2f((m - most) * LOG2E);
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        if (p + i * 64 < n) s += v[i][1] * __builtin_amdgcn_exp2f((v[i][0] - most) * LOG2E);
      m = most;
    }
  }
  s_m[quarter][lane & 15] = m;
  s_s[quarter][lane & 15] = s;
  const bool exponents = a.range && a.d_logp;
  if (exponents && blockIdx.x * 16 + wave < a.rows) {  // (a row a wave)
    const uint32_t most = row_largest(a.x, blockIdx.x * 16 + wave, a.d, a.x16_lo == nullptr);
    if (lane == 0) s_x[wave] = most;
  }
  __syncthreads();
  if (wave > 0) return;
  // (a quarter of this wave joins sixteen of the sums)
  float top = LOWEST, sum = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) top = fmaxf(top, s_m[quarter * 16 + w][lane & 15]);
  top = fmaxf(top, __shfl_xor(top, 16, 64));
  top = fmaxf(top, __shfl_xor(top, 32, 64));
#pragma unroll
  for (int w = 0; w < 16; ++w) sum += s_s[quarter * 16 + w][lane & 15] * __builtin_amdgcn_exp2f((s_m[quarter * 16 + w][lane & 15] - top) * LOG2E);
  sum += __shfl_xor(sum, 16, 64);
  sum += __shfl_xor(sum, 32, 64);
  if (lane >= 16 || row >= a.rows) return;
  const float log2_sum = __builtin_amdgcn_logf(sum), log_sum = log2_sum * LN2;
  const int32_t target = a.targets[row];
  put_row(a, row, target, a.at_target[row], top, log_sum);
  a.off[2 * row] = top;
  a.off[2 * row + 1] = log2_sum;
  if (exponents)
    a.exponents[row] = row_exponent(a.range, row, row_weight(target, a.vocab, a.d_logp + row), probability(a.at_target[row], top, log2_sum), s_x[lane]);
}

// 16-bit products: G of a row's 2048 columns, in two bf16 numbers for dX of bf16 layers, in two float16 ones for what else there is.  Columns
// behind the vocabulary become zeros.  Blocks behind the rows' make the float16 copies of x, 2048 values each.
__global__ __launch_bounds__(256) void head_grad_kernel(HeadRowsArgs a, int segs) {
  if ((int)blockIdx.x >= a.rows * segs) {
    const int64_t i = (int64_t)(blockIdx.x - a.rows * segs) * 2048 + threadIdx.x * 8;
    const int common = common_exponent(a.range);
    if (i >= (int64_t)a.rows * a.d) return;
    const int row = (int)((uint64_t)i / (uint32_t)a.d), e = common - a.exponents[row];
    const int32_t target = a.targets[row];
    const bool there = target >= 0 && target < a.vocab;
    if (i == 0) {
      a.range->undo_dw[0] = power_of_two(-common / 2);
      a.range->undo_dw[1] = power_of_two(-common - -common / 2);
    }
    if (a.x16_lo) {
      f32x4 v[2] = {};
      if (there) {
        v[0] = *reinterpret_cast<const f32x4*>(static_cast<const float*>(a.x) + i);
        v[1] = *reinterpret_cast<const f32x4*>(static_cast<const float*>(a.x) + i + 4);
      }
      put_parts(v, e, a.x16 + i, a.x16_lo + i);
    } else {
      const bf16x8 v = *reinterpret_cast<const bf16x8*>(static_cast<const bf16_t*>(a.x) + i);
      f16x8 o;
#pragma unroll
      for (int k = 0; k < 8; ++k) o[k] = there ? (f16_t)times_2((float)v[k], e) : (f16_t)0.f;
      *reinterpret_cast<f16x8*>(a.x16 + i) = o;
    }
    return;
  }
  const int row = blockIdx.x / segs, c = (blockIdx.x - row * segs) * 2048 + threadIdx.x * 8;
  if (c >= a.ldv) return;
  const int32_t target = a.targets[row];
  const float top = a.off[2 * row], log2_sum = a.off[2 * row + 1], w = row_weight(target, a.vocab, a.d_logp + row);
  const int exponent = a.exponents[row];
  const int64_t at = (int64_t)row * a.ldv + c;
  const f32x4 v[2] = {__builtin_nontemporal_load(reinterpret_cast<const f32x4*>(a.logits + at)),  // (read once: 473 us in place of 498)
                      __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(a.logits + at + 4))};
  bf16x8 g, rest;
  f16x8 hi, lo;
  f32x4 plain[2];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float x = grad_of(v[e >> 2][e & 3], top, log2_sum, w, target, c + e, a.vocab), scaled = times_2(x, exponent);
    plain[e >> 2][e & 3] = x;
    g[e] = (bf16_t)x;
    rest[e] = (bf16_t)(x - (float)g[e]);
    hi[e] = (f16_t)scaled;
    lo[e] = (f16_t)(scaled - (float)hi[e]);
  }
  if (a.g) {
    *reinterpret_cast<bf16x8*>(a.g + at) = g;
    *reinterpret_cast<bf16x8*>(a.g_rest + at) = rest;
  }
  if (a.plain_cols && a.range->plain) {  // (for dX, in the logits' place)
    *reinterpret_cast<f32x4*>(a.logits + at) = plain[0];
    *reinterpret_cast<f32x4*>(a.logits + at + 4) = plain[1];
  }
  if (a.hi) {
    *reinterpret_cast<f16x8*>(a.hi + at) = hi;
    *reinterpret_cast<f16x8*>(a.lo + at) = lo;
  }
}

// float32 layers that take no pairs: G in the place of the logits, 2048 columns of a row a block.  The first block of a row copies x for dW.
__global__ __launch_bounds__(256) void head_grad_f32_kernel(HeadRowsArgs a, int segs) {
  const int t = blockIdx.x / segs, c0 = (blockIdx.x - t * segs) * 2048 + threadIdx.x * 4;
  const int32_t target = a.targets[t];
  const float top = a.off[2 * t], log2_sum = a.off[2 * t + 1], w = row_weight(target, a.vocab, a.d_logp + t);
  float* const row = a.logits + (int64_t)t * a.ldv;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int c = c0 + i * 1024;
    if (c >= a.ldv) break;
    f32x4 g = *reinterpret_cast<const f32x4*>(row + c);
#pragma unroll
    for (int e = 0; e < 4; ++e) g[e] = grad_of(g[e], top, log2_sum, w, target, c + e, a.vocab);
    *reinterpret_cast<f32x4*>(row + c) = g;
  }
  if (a.x32 && (int)blockIdx.x % segs == 0) {
    const float* const x = static_cast<const float*>(a.x) + (int64_t)t * a.d;
    for (int c = threadIdx.x * 4; c < a.d; c += 1024)
      *reinterpret_cast<f32x4*>(a.x32 + (int64_t)t * a.d + c) = target >= 0 && target < a.vocab ? *reinterpret_cast<const f32x4*>(x + c) : f32x4{};
  }
}

// dX of a piece: its slabs, in order.  A block takes 1024 columns of a row, or, of sixteen parts and more, 256 columns, whose parts its four
// waves share out (24 x 256, 128 parts: 4.9 us in place of 8.7; twice the parts, 64 rows: 6.9 in place of 14.6).
struct HeadJoinArgs {
  const float* slabs;
  const int32_t* exponents;  // of G's rows, and of W, by which the slabs are too large; or null
  const HeadRange* range;
  int64_t stride, rest;    // from part to part; to the rows of G's second numbers, or 0
  int32_t parts, plain_parts, d;  // plain_parts: where the product is in float32
};
template <typename T, bool SHARED>
__global__ __launch_bounds__(256) void head_join_kernel(HeadJoinArgs a, T* dX) {
  __shared__ f32x4 s_part[SHARED ? 4 : 1][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = blockIdx.x, c = SHARED ? blockIdx.y * 256 + lane * 4 : blockIdx.y * 1024 + threadIdx.x * 4;
  if (!SHARED && c >= a.d) return;
  const int64_t i = (int64_t)row * a.d + min(c, a.d - 4);
  const bool plain = a.exponents && a.range->plain;
  const int parts = plain ? a.plain_parts : a.parts;
  const int share = SHARED ? (parts + 3) / 4 : parts, first = SHARED ? wave * share : 0, end = min(first + share, parts);
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  for (int p = first; p < end; p += 8) {
    f32x4 v[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = *reinterpret_cast<const f32x4*>(a.slabs + min(p + q, end - 1) * a.stride + i);
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (p + q < end) s += v[q];
    if (a.rest) {
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] = *reinterpret_cast<const f32x4*>(a.slabs + min(p + q, end - 1) * a.stride + a.rest + i);
#pragma unroll
      for (int q = 0; q < 8; ++q)
        if (p + q < end) s += v[q];
    }
  }
  if constexpr (SHARED) {
    s_part[wave][lane] = s;
    __syncthreads();
    if (wave > 0 || c >= a.d) return;
#pragma unroll
    for (int w = 1; w < 4; ++w) s += s_part[w][lane];
  }
  if (a.exponents && !plain) {
    const int by = -a.exponents[row] - a.range->w_exponent;
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = times_2(s[e], by);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) dX[i + e] = (T)s[e];
}

template <typename T>
hipError_t run_join(const HeadJoinArgs& a, int64_t rows, T* dX, hipStream_t s) {
  if (a.parts >= 16) hipLaunchKernelGGL((head_join_kernel<T, true>), dim3((unsigned)rows, (unsigned)((a.d + 255) / 256)), dim3(256), 0, s, a, dX);
  else hipLaunchKernelGGL((head_join_kernel<T, false>), dim3((unsigned)rows, (unsigned)((a.d + 1023) / 1024)), dim3(256), 0, s, a, dX);
  return hipGetLastError();
}

// dW: the parts of its sum, in order, added to what there is or stored.
__global__ __launch_bounds__(256) void head_dw_join_kernel(const float* slabs, int parts, int64_t n, float* dW, int accumulate) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;  // (n: whole rows of 32 and more columns)
  if (i >= n) return;
  f32x4 s = accumulate ? *reinterpret_cast<const f32x4*>(dW + i) : f32x4{0.f, 0.f, 0.f, 0.f};
  for (int p = 0; p < parts; p += 8) {
    f32x4 v[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = *reinterpret_cast<const f32x4*>(slabs + min(p + q, parts - 1) * n + i);
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (p + q < parts) s += v[q];
  }
  *reinterpret_cast<f32x4*>(dW + i) = s;
}

// ---------------------------------------------------------------- few rows
// Bound by the stream of W.  A block takes 64 rows of W and up to 16 NT rows of x; its four waves share the sum over d out and go their
// own ways until the end: each moves 128 bytes of all these rows at a time straight into LDS of its own, whole lines with the
// non-temporal hint, and reads the operands of the matrix instruction from there.  What a wave waits for, the other blocks of its CU
// (four, three or two) hide: with a ring of two or three such steps, and fewer blocks, 64 rows x 32000, d = 2048, took 33 us in
// place of 30.6 and 32 x 50257, d = 256, 16.5 in place of 11.2.  (Read from memory in the order of the operands, sixteen rows of 64
// bytes a load, one row x 131072, d = 4096, took 190 us without the hint and 269 with it, as each line then came twice; this way
// 166, 6.5 TB/s.)  The waves' sums meet in LDS; what leaves the block is, for every row of x, the maximum and the sum of exponentials of
// its 64 logits.  A second launch joins them.
struct HeadStreamArgs {
  const void *x, *W;
  const int32_t* targets;
  float* pairs;      // [T][ceil(vocab / 64)] maximum and sum
  float* at_target;  // [T]
  float *logp, *log_z;
  float* logits;     // [T, ldv] or null
  float* off;        // [T][2] maximum and log2 of the sum, or null
  HeadRange* range;  // (16-bit products of gradients) or null, and what it needs
  int32_t* exponents;
  const float* d_logp;
  int32_t T, d, vocab, ldv;
};

template <typename T, int NT>
__global__ __launch_bounds__(256, 2) void head_stream_kernel(HeadStreamArgs a) {
  constexpr int ES = sizeof(T), NW = STREAM_W / 16;
  constexpr int ROWS = STREAM_W + NT * 16, UNITS = ROWS / 8, STAGE = ROWS * 128;  // unit: eight rows, one load
  typedef typename VecOf<T>::type frag_t;
  constexpr int SUMS = 4 * NW * NT * 1024;  // in the steps' place at the end: the waves' sums, then the fragments' maxima and sums
  __shared__ __attribute__((aligned(1024))) char buf[std::max(4 * STAGE, SUMS + 2 * NW * NT * 64)];
  float(*const s_m)[NT * 16] = reinterpret_cast<float(*)[NT * 16]>(buf + SUMS);
  float(*const s_s)[NT * 16] = s_m + NW;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int strips = (a.vocab + STREAM_W - 1) / STREAM_W, groups = gridDim.x / strips;
  const int strip = blockIdx.x / groups, t0 = (blockIdx.x - strip * groups) * (NT * 16), v0 = strip * STREAM_W;
  const int r = lane & 15, quad = lane >> 4;
  char* const mine = buf + wave * STAGE;
  const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_address(mine));

  // This wave's steps of 128 bytes, from a place on that differs from block to block: rows of W lie a power of two apart as a rule, and
  // blocks that all read at the same place of their rows would meet in few memory channels.
  const int bytes = a.d * ES, steps = (bytes + 127) / 128, per = (steps + 3) / 4;
  const int first = min(wave * per, steps), n = min(per, steps - first);
  const int start = n > 0 ? (strip * 5) % n : 0;
  // lane 8 i + c of a unit loads row i's chunk of sixteen bytes so that it lands at place c: chunk c ^ (row >> 1 & 7), which keeps the
  // reads of sixteen rows out of each other's banks
  const char* const w0 = static_cast<const char*>(a.W) + (int64_t)v0 * bytes;
  const char* const x0 = static_cast<const char*>(a.x) + (int64_t)t0 * bytes;
  const int row8 = lane >> 3;
  uint32_t off[UNITS];
#pragma unroll
  for (int u = 0; u < UNITS; ++u) {
    const int row = u * 8 + row8, c = (lane & 7) ^ ((row >> 1) & 7);
    off[u] = (uint32_t)(u < STREAM_W / 8 ? min(row, a.vocab - 1 - v0) : min(row - STREAM_W, a.T - 1 - t0)) * (uint32_t)bytes + c * 16;
  }
  auto issue = [&](int i) {
    const int k = i + start >= n ? i + start - n : i + start, at = (first + k) * 128;
    if (at + 128 <= bytes) {
#pragma unroll
      for (int u = 0; u < UNITS; ++u) {
        if (u < STREAM_W / 8) dma_b128_s<true>(w0 + at, off[u], lds + u * 1024);
        else dma_b128_s(x0 + at, off[u], lds + u * 1024);
      }
    } else {  // (bf16: half a step) what lies behind the rows' ends reads zeros
#pragma unroll
      for (int u = 0; u < UNITS; ++u) {
        const int c = (lane & 7) ^ (((u * 8 + row8) >> 1) & 7);
        const char* const p = (u < STREAM_W / 8 ? w0 : x0) + at + off[u];
        dma_b128(at + c * 16 < bytes ? p : reinterpret_cast<const char*>(g_zero_chunk), lds + u * 1024);
      }
    }
  };
  f32x4 acc[NW][NT];
#pragma unroll
  for (int i = 0; i < NW; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto wait = [&](bool loads) {
    __builtin_amdgcn_sched_barrier(0);
    if (loads) __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): the step has landed
    else __builtin_amdgcn_s_waitcnt(0xc07f);         // lgkmcnt(0): it has been read
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
#pragma unroll 1
  for (int i = 0; i < n; ++i) {
    issue(i);
    wait(true);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      frag_t wf[NW], xf[NT];
      auto read = [&](int row) {
        return *reinterpret_cast<const frag_t*>(mine + (row + r) * 128 + (((h * 4 + quad) ^ ((r >> 1) & 7)) << 4));
      };
#pragma unroll
      for (int q = 0; q < NW; ++q) wf[q] = read(q * 16);
#pragma unroll
      for (int j = 0; j < NT; ++j) xf[j] = read(STREAM_W + j * 16);
#pragma unroll
      for (int q = 0; q < NW; ++q)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          if constexpr (ES == 2) {
            acc[q][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[q], xf[j], acc[q][j], 0, 0, 0);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[q][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(wf[q][e], xf[j][e], acc[q][j], 0, 0, 0);
          }
        }
    }
    wait(false);
  }

  __syncthreads();  // (no step is in use any more)
  auto sum_at = [&](int w, int f) { return reinterpret_cast<f32x4*>(buf + ((w * NW * NT + f) * 64 + lane) * 16); };
#pragma unroll
  for (int i = 0; i < NW; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) *sum_at(wave, i * NT + j) = acc[i][j];
  __syncthreads();
  // wave i takes fragment i: lane holds the logits of rows 4 quad .. + 3 of the fragment and of row r of every sixteen of x
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int t = t0 + j * 16 + r, v = v0 + wave * 16 + quad * 4;
    f32x4 l = *sum_at(0, wave * NT + j);
#pragma unroll
    for (int q = 1; q < 4; ++q) l += *sum_at(q, wave * NT + j);
    if (a.logits && t < a.T && v < a.ldv) *reinterpret_cast<f32x4*>(a.logits + (int64_t)t * a.ldv + v) = l;
    const int32_t at = t < a.T ? max(a.targets[t], -1) - v : -1;
    if (at >= 0 && at < 4 && v + at < a.vocab) a.at_target[t] = at == 0 ? l[0] : at == 1 ? l[1] : at == 2 ? l[2] : l[3];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (v + e >= a.vocab) l[e] = -__builtin_inff();
    float m = fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3]));
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    m = fmaxf(m, LOWEST);
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) s += __builtin_amdgcn_exp2f((l[e] - m) * LOG2E);
    s += __shfl_xor(s, 16, 64);
    s += __shfl_xor(s, 32, 64);
    if (quad == 0) {
      s_m[wave][j * 16 + r] = m;
      s_s[wave][j * 16 + r] = s;
    }
  }
  __syncthreads();
  const int t = threadIdx.x;
  if (t >= NT * 16 || t0 + t >= a.T) return;
  float m = s_m[0][t], s = 0.f;
#pragma unroll
  for (int i = 1; i < NW; ++i) m = fmaxf(m, s_m[i][t]);
#pragma unroll
  for (int i = 0; i < NW; ++i) s += s_s[i][t] * __builtin_amdgcn_exp2f((s_m[i][t] - m) * LOG2E);
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  *reinterpret_cast<f32x2*>(a.pairs + ((int64_t)(t0 + t) * strips + strip) * 2) = f32x2{m, s};
}

// A block joins the pairs of one row.
__global__ __launch_bounds__(1024) void head_stream_join_kernel(HeadStreamArgs a, bool bf16) {
  __shared__ float s_m[16], s_s[16];
  __shared__ uint32_t s_x;
  constexpr int AHEAD = 4;
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const int t = blockIdx.x, n = (a.vocab + STREAM_W - 1) / STREAM_W, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const f32x2* const pairs = reinterpret_cast<const f32x2*>(a.pairs) + (int64_t)t * n;
  float m = LOWEST, s = 0.f;
  for (int p = threadIdx.x; p < n; p += 1024 * AHEAD) {
    f32x2 v[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) v[i] = pairs[min(p + i * 1024, n - 1)];
    float most = m;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) most = fmaxf(most, v[i][0]);
    s *= __builtin_amdgcn_exp2f((m - most) * LOG2E);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (p + i * 1024 < n) s += v[i][1] * __builtin_amdgcn_exp2f((v[i][0] - most) * LOG2E);
    m = most;
  }
  const float wm = wave_max(m);
  s = wave_sum(s * __builtin_amdgcn_exp2f((m - wm) * LOG2E));
  if (lane == 0) {
    s_m[wave] = wm;
    s_s[wave] = s;
  }
  if (a.range && wave == 15) {
    const uint32_t most = row_largest(a.x, t, a.d, bf16);
    if (lane == 0) s_x = most;
  }
  __syncthreads();
  if (threadIdx.x > 0) return;
  float top = s_m[0], sum = 0.f;
  for (int w = 1; w < 16; ++w) top = fmaxf(top, s_m[w]);
  for (int w = 0; w < 16; ++w) sum += s_s[w] * __builtin_amdgcn_exp2f((s_m[w] - top) * LOG2E);
  const float log2_sum = __builtin_amdgcn_logf(sum), log_sum = log2_sum * LN2;
  const int32_t target = a.targets[t];
  put_row(a.logp ? a.logp + t : nullptr, a.log_z ? a.log_z + t : nullptr, target, a.vocab, a.at_target[t], top, log_sum);
  if (a.off) {
    a.off[2 * t] = top;
    a.off[2 * t + 1] = log2_sum;
  }
  if (a.range) a.exponents[t] = row_exponent(a.range, t, row_weight(target, a.vocab, a.d_logp + t), probability(a.at_target[t], top, log2_sum), s_x);
}

template <typename T>
hipError_t run_stream(const HeadStreamArgs& a, hipStream_t s) {
  // A small vocabulary makes few blocks, each a chain of steps: fewer rows of x in each, while there is at most one for every CU.  64 rows with 1900 x
  // 3136, float32 72.8 -> 37.8 us, bf16 16.4 -> 18.2; 4000 x 2048 50.2 -> 28.9, 16.8 -> 15.2; 1000 x 512 18.8 -> 11.3, 9.9 -> 8.0.
  const int strips = (a.vocab + STREAM_W - 1) / STREAM_W;
  auto blocks = [&](int nt) { return (int64_t)strips * ((a.T + nt * 16 - 1) / (nt * 16)); };
  int nt = a.T <= 16 ? 1 : a.T <= 32 ? 2 : 4;
  while (nt > 1 && blocks(nt / 2) <= 256) nt /= 2;
  const dim3 grid((unsigned)blocks(nt)), block(256);
  if (nt == 1) hipLaunchKernelGGL((head_stream_kernel<T, 1>), grid, block, 0, s, a);
  else if (nt == 2) hipLaunchKernelGGL((head_stream_kernel<T, 2>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((head_stream_kernel<T, 4>), grid, block, 0, s, a);
  if (a.logp || a.log_z || a.off) hipLaunchKernelGGL(head_stream_join_kernel, dim3((unsigned)a.T), dim3(1024), 0, s, a, sizeof(T) == 2);
  return hipGetLastError();
}
size_t stream_pairs(int64_t T, int32_t vocab) { return (size_t)T * ((vocab + STREAM_W - 1) / STREAM_W) * 8; }
size_t stream_workspace(int64_t T, int32_t vocab) { return ALIGN + align_up(stream_pairs(T, vocab), ALIGN) + (size_t)T * 4; }

struct HeadLayout {
  size_t range, logits, pairs, at_target, off, exponents, g, hi, lo, x16, x16_lo, w16, w16_lo, x32, slabs, total;
};
HeadLayout layout_for(int64_t plans, int64_t rows, int64_t slab_cells, int32_t d, int32_t vocab, bool bf16,
                      bool pairs, bool grad) {
  HeadLayout w = {};
  const bool wide = bf16 || pairs;
  const size_t ldv = align_up(vocab, 64), cells = (size_t)rows * ldv;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += align_up(bytes, ALIGN);
    return here;
  };
  take(sizeof(GemmPlan) * (size_t)plans);
  // (the range ends where the targets' logits begin)
  at = align_up(at + sizeof(HeadRange), ALIGN);
  w.range = at - sizeof(HeadRange);
  w.at_target = take((size_t)rows * (pairs ? 8 : 4));
  w.logits = take(grad ? cells * 4 : 0);
  w.pairs = take(std::max(pair_cells(rows, d, vocab, bf16) * 8, stream_pairs(std::min(rows, stream_rows(vocab)), vocab)));
  w.off = take((size_t)rows * 8);
  w.exponents = take(wide && grad ? (size_t)rows * 4 : 0);
  w.g = take(bf16 && grad ? 2 * cells * 2 : 0);
  w.hi = take(wide && grad ? cells * 2 : 0);
  w.lo = take(wide && grad ? cells * 2 : 0);
  w.x16 = take(pairs || (bf16 && grad) ? (size_t)rows * d * 2 : 0);
  w.x16_lo = take(pairs ? (size_t)rows * d * 2 : 0);
  w.w16 = take(pairs ? (size_t)vocab * d * 2 : 0);
  w.w16_lo = take(pairs ? (size_t)vocab * d * 2 : 0);
  w.x32 = take(!wide && grad ? (size_t)rows * d * 4 : 0);
  w.slabs = take(grad ? (size_t)slab_cells * 4 : 0);
  w.total = at;
  return w;
}
// of all batches of at most T rows of one kind: the most tables, rows of a piece, slabs
size_t most_workspace(int64_t T, int32_t d, int32_t vocab, bool bf16, bool pairs, bool grad) {
  const bool wide = bf16 || pairs;
  const int64_t most = most_rows(vocab, bf16, pairs, grad), rows = std::min<int64_t>(padded_rows(T), most);
  HeadShape h = {};
  h.pairs = pairs;
  h.grad = grad;
  const int64_t plans = std::min<int64_t>((T + most - 1) / most, PLAN_PIECES) * head_products(h);
  const int64_t dx_rows = bf16 ? std::max(rows, std::min(2 * rows, 2 * STACK_ROWS)) : rows;
  const int64_t dw_parts = dw_most_parts(d, vocab, wide);
  const int64_t slabs = std::max(std::min(MAX_PARTS * dx_rows * d, std::max(SLAB_CELLS, dx_rows * d)), dw_parts > 1 ? dw_parts * vocab * d : 0);
  return ALIGN + layout_for(plans, rows, slabs, d, vocab, bf16, pairs, grad).total;
}
}  // namespace

size_t head_workspace(int64_t T, int32_t d, int32_t vocab, modse_dtype dt, bool grad) {
  if (T == 0) return 0;
  size_t most = 0;
  if (!grad) {
    most = stream_workspace(std::min(T, stream_rows(vocab)), vocab);
    if (T <= stream_rows(vocab)) return most;
  }
  const bool bf16 = dt == MODSE_BF16, pairs = takes_pairs(T, d, vocab, dt, grad);
  if (pairs) most = std::max(most, most_workspace(T, d, vocab, false, true, grad));
  return std::max(most, most_workspace(pairs ? std::min(T, pairs_from(d, vocab, grad) - 1) : T, d, vocab, bf16, false, grad));
}

hipError_t launch_head(modse_dtype dt, const HeadArgs& a, char* ws, hipStream_t s) {
  const bool grad = a.dX || a.dW;
  if (!grad && a.T <= stream_rows(a.vocab)) {
    float* const pairs = reinterpret_cast<float*>(align_up(reinterpret_cast<size_t>(ws), ALIGN));
    float* const at_target = pairs + align_up(stream_pairs(a.T, a.vocab), ALIGN) / 4;
    const HeadStreamArgs r = {a.x, a.W, a.targets, pairs, at_target, a.logp, a.log_z, nullptr, nullptr, nullptr, nullptr, nullptr, (int32_t)a.T, a.d, a.vocab, 0};
    return dt == MODSE_F32 ? run_stream<float>(r, s) : run_stream<bf16_t>(r, s);
  }
  const HeadShape h = head_shape(a.T, a.d, a.vocab, dt, grad);
  const HeadShape f = h.pairs ? head_shape(a.T, a.d, a.vocab, dt, grad, true) : HeadShape{};  // (pieces of the same rows)
  const int64_t plans = (int64_t)std::min(h.pieces, PLAN_PIECES) * head_products(h);
  const int64_t slabs = std::max((int64_t)std::max(h.k_parts, f.k_parts) * h.dx_rows * h.d, h.w_split > 1 ? (int64_t)h.w_split * h.vocab * h.d : 0);
  const HeadLayout w = layout_for(plans, h.rows, slabs, h.d, h.vocab, h.bf16, h.pairs, grad);
  ws = reinterpret_cast<char*>(align_up(reinterpret_cast<size_t>(ws), ALIGN));
  auto floats = [&](size_t at) { return reinterpret_cast<float*>(ws + at); };
  auto halves = [&](size_t at) { return reinterpret_cast<f16_t*>(ws + at); };
  HeadRange* const range = h.pairs || (h.bf16 && grad) ? reinterpret_cast<HeadRange*>(ws + w.range) : nullptr;
  const HeadBufs b = {reinterpret_cast<GemmPlan*>(ws), floats(w.logits), floats(w.pairs), floats(w.at_target), floats(w.off),
                      reinterpret_cast<bf16_t*>(ws + w.g), halves(w.hi), halves(w.lo), halves(w.x16), halves(w.x16_lo), reinterpret_cast<int32_t*>(ws + w.exponents),
                      halves(w.w16), halves(w.w16_lo), floats(w.x32), range, floats(w.slabs)};
  const int64_t w_cells = (int64_t)h.vocab * h.d;
  const int range_blocks = h.pairs ? (int)std::min<int64_t>((w_cells + 32767) / 32768, RANGE_BLOCKS) : 0;
  if (h.pairs) {
    hipLaunchKernelGGL(head_range_kernel, dim3(range_blocks), dim3(1024), 0, s, static_cast<const u32x4*>(a.W), w_cells / 4, range);
    hipLaunchKernelGGL(head_split_w_kernel, dim3((unsigned)std::min<int64_t>((w_cells + 2047) / 2048, 2048)), dim3(256), 0, s,
                       static_cast<const float*>(a.W), w_cells, b.w16, b.w16_lo, range, range_blocks);
  }
  const bool stream = h.T <= stream_rows(h.vocab) && h.pieces == 1;  // (only with gradients here)
  int planned = 0;  // pieces that there are tables of
  auto begin = [&](int64_t piece, int64_t t0, int64_t m) {
    const int first = (int)piece, n = piece % PLAN_PIECES ? 0 : std::min(h.pieces - first, PLAN_PIECES), tables = n * head_products(h);
    if (n) planned = n;
    int lanes = 64;
    while (lanes > 2 && lanes / 2 >= h.d / 8) lanes /= 2;
    const int64_t x_blocks = h.pairs && !stream ? (m * lanes + 255) / 256 : 0;
    const HeadPlanArgs plan = {h, b, a.x, a.W, a.targets, a.d_logp, a.dW, f, first, n, tables, (int32_t)t0, (int32_t)m, range_blocks};
    if (tables + x_blocks) hipLaunchKernelGGL(head_plan_kernel, dim3((unsigned)(tables + x_blocks)), dim3(256), 0, s, plan);
  };
  auto tiles_of = [](int64_t m, int64_t n, TileShape t) { return tiles(m, n, t.bm); };
  hipError_t e = hipGetLastError();
  // the logits of a piece, their sums and (of gradients) G
  auto table = [&](int product, int at) { return b.plans + head_table(h, product) * planned + at; };
  auto logits = [&](int at, int64_t t0, int64_t m) {
    if (stream) {
      const HeadStreamArgs r = {a.x, a.W, a.targets, b.pairs, b.at_target, a.logp, nullptr, b.logits, b.off, range, b.exponents, a.d_logp,
                                (int32_t)m, h.d, h.vocab, h.ldv};
      e = h.bf16 ? run_stream<bf16_t>(r, s) : run_stream<float>(r, s);
    } else {
      auto most_tiles = [&](const HeadShape& p) { return tiles_of(m, p.vocab, p.logits_tile) + p.w_parts * tiles_of(m, 1, p.logits_tile); };
      e = launch_grouped_gemm(dt, h.pairs ? EPI_LOGITS_PAIRS : EPI_LOGITS, h.logits_tile, table(LOGITS, at), h.w_parts, 0,
                              h.logits_tile.bm < 256 ? GEMM_SPREAD_K : GEMM_STREAM_C, most_tiles(h), s, LAYOUT_TN);
      if (e == hipSuccess && h.pairs) e = launch_rare_gemm(EPI_LOGITS, table(PLAIN_LOGITS, at), f.w_parts, most_tiles(f), s);
    }
    if (e != hipSuccess) return;
    const HeadRowsArgs r = {a.targets + t0, a.d_logp ? a.d_logp + t0 : nullptr, a.logp ? a.logp + t0 : nullptr, a.log_z ? a.log_z + t0 : nullptr,
                            b.logits, b.pairs, b.at_target, b.off, a.dX && h.bf16 ? b.g : nullptr, a.dX && h.bf16 ? b.g + (int64_t)h.rows * h.ldv : nullptr,
                            a.dW || h.pairs ? b.hi : nullptr, a.dW || h.pairs ? b.lo : nullptr, range, b.exponents,
                            static_cast<const char*>(a.x) + (size_t)t0 * h.d * (h.bf16 ? 2 : 4), b.x16, h.pairs ? b.x16_lo : nullptr,
                            a.dW && !h.wide ? b.x32 : nullptr,
                            (int32_t)m, h.vocab, h.ldv, h.rows, h.pair_cols(), h.pairs ? f.pair_cols() : 0, h.d};
    if (!stream) hipLaunchKernelGGL(head_stats_kernel, dim3((unsigned)((m + 15) / 16)), dim3(1024), 0, s, r);
    if (grad) {
      const int64_t segs = (h.ldv + 2047) / 2048, copies = a.dW && h.wide ? (m * h.d + 2047) / 2048 : 0;
      const dim3 grid((unsigned)(m * segs + copies));
      if (h.wide) hipLaunchKernelGGL(head_grad_kernel, grid, dim3(256), 0, s, r, (int)segs);
      else hipLaunchKernelGGL(head_grad_f32_kernel, grid, dim3(256), 0, s, r, (int)segs);
    }
    e = hipGetLastError();
  };
  for (int64_t piece = 0; piece < h.pieces && e == hipSuccess; ++piece) {
    const int64_t t0 = piece * h.rows, m = std::min<int64_t>(h.rows, h.T - t0);
    const int at = (int)(piece % PLAN_PIECES);
    begin(piece, t0, m);
    logits(at, t0, m);
    if (e != hipSuccess || !grad) continue;
    if (a.dW) {  // (before dX, which may lie in the buffer of x)
      const int accumulate = a.accumulate || piece > 0;
      e = launch_grouped_gemm(dt, h.pairs ? EPI_ROWS_PAIRS : EPI_ROWS_F32, h.dw_tile, table(DW, at), h.w_split, h.w_split > 1 ? 0 : accumulate, 0,
                              h.w_split * tiles_of(padded_rows(h.vocab), h.d, h.dw_tile), s, LAYOUT_AB_K);
      if (e == hipSuccess && h.w_split > 1) {
        const int64_t n = (int64_t)h.vocab * h.d;
        hipLaunchKernelGGL(head_dw_join_kernel, dim3((unsigned)((n + 1023) / 1024)), dim3(256), 0, s, b.slabs, h.w_split, n, a.dW, accumulate);
        e = hipGetLastError();
      }
      if (e != hipSuccess) break;
    }
    if (a.dX) {
      const bool stacked = h.dx_rows > h.rows;
      e = launch_grouped_gemm(dt, h.pairs ? EPI_STORE_PAIRS : h.bf16 && !stacked ? EPI_STORE_DUALK_F32 : EPI_STORE_F32, h.dx_tile,
                              table(DX, at), h.k_parts, 0, 0, h.k_parts * tiles_of(stacked ? h.dx_rows : m, h.d, h.dx_tile), s, LAYOUT_B_KN);
      if (e == hipSuccess && h.pairs)
        e = launch_rare_gemm(EPI_STORE_F32, table(PLAIN_DX, at), f.k_parts, f.k_parts * tiles_of(m, h.d, f.dx_tile), s);
      if (e != hipSuccess) break;
      const HeadJoinArgs j = {b.slabs, h.pairs ? b.exponents : nullptr, range, (int64_t)h.dx_rows * h.d, stacked ? (int64_t)h.rows * h.d : 0,
                              h.k_parts, f.k_parts, h.d};
      e = h.bf16 ? run_join(j, m, static_cast<bf16_t*>(a.dX) + t0 * h.d, s) : run_join(j, m, static_cast<float*>(a.dX) + t0 * h.d, s);
    }
  }
  return e;
}
