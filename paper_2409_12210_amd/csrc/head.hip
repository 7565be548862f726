// Log probabilities of the next tokens from the last hidden rows and the output matrix, without the logits of a whole batch, and their
// gradients.
//
//   l = x W^T,  log Z_t = log sum_v e^l_tv,  logp_t = l_t,target - log Z_t
//   G_tv = w_t (1[v = target_t] - e^(l_tv - log Z_t)),  dX = G W,  dW = G^T x
//
// The batch is taken in pieces of rows whose logits and G fit a workspace of a fixed size.  The products are those of the grouped
// GEMM kernels, whose problem tables one launch makes for all pieces.  dX is a product over the whole vocabulary with few
// columns, so its sum is cut into parts that fill the chip; the parts are float32 slabs that a last launch adds up in order.
//
// dW is float32, and a term of its sums is rounded to 2^-17: in bf16 G is kept as two numbers, hi + lo, and dW takes both.  dX
// is rounded to bf16 itself and takes hi alone.
#include "ops.h"

#include "gemm_plan.h"

namespace {
using namespace modse_gemm;

constexpr int64_t PIECE = (int64_t)1 << 28;   // logits of a piece of rows
constexpr int64_t W_PART = (int64_t)1 << 30;  // elements of W that one problem reads (kernels count them in 32 bits)
constexpr size_t ALIGN = 256;                 // of what is in the workspace, which itself may lie at any sixteen bytes
constexpr int64_t SLAB_ROWS = 8192;           // of all parts of dX together, unless one part has more

struct HeadShape {
  int64_t T;
  int32_t d, vocab, ldv;   // ldv: distance of rows of logits and G
  int32_t rows, pieces;    // rows of a piece, a multiple of 256 (of 32 where there is one piece)
  int32_t w_parts, w_rows; // problems of the logits, rows of W in each
  int32_t k_parts, k_len;  // problems of dX, columns of G in each
  int32_t bf16;
  TileShape logits_tile, dx_tile, dw_tile;
};

int32_t padded_rows(int64_t n) { return (int32_t)align_up((size_t)n, 32); }

HeadShape head_shape(int64_t T, int32_t d, int32_t vocab, modse_dtype dt) {
  HeadShape h = {};
  h.T = T;
  h.d = d;
  h.vocab = vocab;
  h.bf16 = dt == MODSE_BF16;
  h.ldv = (int32_t)align_up(vocab, 64);
  const int64_t most = head_piece_rows(vocab);
  h.pieces = (int32_t)((T + most - 1) / most);
  h.rows = h.pieces == 1 ? padded_rows(T) : (int32_t)align_up((size_t)((T + h.pieces - 1) / h.pieces), 256);
  h.pieces = (int32_t)((T + h.rows - 1) / h.rows);
  h.w_rows = (int32_t)std::min<int64_t>(vocab, W_PART / d / 256 * 256);
  h.w_parts = (vocab + h.w_rows - 1) / h.w_rows;
  auto tiles = [](int64_t m, int64_t n, int b) { return ((m + b - 1) / b) * ((n + b - 1) / b); };
  auto tile = [&](int64_t m, int64_t n) { const int b = h.bf16 ? 256 : tiles(m, n, 128) >= 512 ? 128 : 64; return TileShape{b, b}; };
  h.logits_tile = tile(h.rows, vocab);
  h.dw_tile = tile(vocab, d);
  h.dx_tile = TileShape{h.bf16 ? 256 : 128, h.bf16 ? 256 : 128};
  // Parts of dX: whole rounds of workgroups over the chip, each part with six further steps for its opening and its end, and slabs that
  // are written and read.
  const int64_t out = tiles(h.rows, d, h.dx_tile.bm), steps = (vocab + 63) / 64, slots = h.bf16 ? 256 : 512;
  const int64_t parts_most = std::min<int64_t>({32, steps, std::max<int64_t>(1, SLAB_ROWS / h.rows)});
  double best = 0;
  for (int64_t n = 1; n <= parts_most; ++n) {
    const int64_t len = (steps + n - 1) / n, parts = (steps + len - 1) / len;
    const double step_us = h.bf16 ? 1.6 : 8.0;
    const double us = (double)((out * parts + slots - 1) / slots) * (len + 6) * step_us + parts * (double)h.rows * d * 8 / 4e6;
    if (n == 1 || us < best) {
      best = us;
      h.k_parts = (int32_t)parts;
      h.k_len = (int32_t)len * 64;
    }
  }
  return h;
}

struct HeadBufs {
  GemmPlan* plans;  // [pieces][3]: logits, dX, dW
  float* logits;    // [rows, ldv]; float32 layers: then G
  bf16_t *hi, *lo;  // [rows, ldv] G
  float* slabs;     // [k_parts][rows, d]
};

struct HeadPlanArgs {
  HeadShape h;
  HeadBufs b;
  const void *x, *W;
  float* dW;
  int32_t grad;
};

// Block 3 i + g (without gradients block i): the problems of product g of piece i.
__global__ __launch_bounds__(64) void head_plan_kernel(HeadPlanArgs a) {
  __shared__ int s_tiles[MODSE_MAX_PROBLEMS];
  const HeadShape& h = a.h;
  const int lane = threadIdx.x, per = a.grad ? 3 : 1, piece = blockIdx.x / per, which = blockIdx.x % per;
  const size_t es = h.bf16 ? 2 : 4;
  const int64_t t0 = (int64_t)piece * h.rows;
  const int m = (int)min((int64_t)h.rows, h.T - t0);
  const char* const x = cadd(a.x, (size_t)t0 * h.d * es);
  GemmPlan* const plan = a.b.plans + piece * 3 + which;
  const int n = which == 0 ? h.w_parts : which == 1 ? h.k_parts : 1;
  for (int p = lane; p < n; p += 64) {
    GemmProblem P = {};
    TileShape t;
    if (which == 0) {
      const int v0 = p * h.w_rows;
      P.A = x;
      P.B = cadd(a.W, (size_t)v0 * h.d * es);
      P.C = a.b.logits + v0;
      P.M = m; P.N = min(h.w_rows, h.vocab - v0); P.K = h.d;
      P.lda = h.d; P.ldb = h.d; P.ldc = h.ldv;
      t = h.logits_tile;
    } else if (which == 1) {
      const int v0 = p * h.k_len;
      P.A = h.bf16 ? (const void*)(a.b.hi + v0) : (const void*)(a.b.logits + v0);
      P.B = cadd(a.W, (size_t)v0 * h.d * es);
      P.C = a.b.slabs + (size_t)p * h.rows * h.d;
      P.M = m; P.N = h.d; P.K = min(h.k_len, h.vocab - v0);
      P.lda = h.ldv; P.ldb = h.d; P.ldc = h.d;
      t = h.dx_tile;
    } else {
      P.A = h.bf16 ? (const void*)a.b.hi : (const void*)a.b.logits;
      P.A2 = a.b.lo;
      P.B = P.B2 = x;
      P.C = a.dW;
      P.E2 = reinterpret_cast<const void*>((intptr_t)h.vocab);
      P.M = (h.vocab + 31) / 32 * 32; P.N = h.d; P.K = m;
      P.lda = h.ldv; P.ldb = h.d; P.ldc = h.d;
      t = h.dw_tile;
    }
    s_tiles[p] = set_tiles(P, t.bm, t.bn);
    plan->prob[p] = P;
  }
  __syncthreads();
  finish_plan(plan, lane, n, s_tiles);
}

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

struct HeadRowsArgs {
  const int32_t* targets;
  const float* d_logp;
  float *logp, *log_z;
  float* logits;
  bf16_t *hi, *lo;
  int64_t t0;
  int32_t rows, vocab, ldv;
};

// A row of logits: its sums, and (GRAD) its row of G.  Columns behind the vocabulary become zeros.
template <bool GRAD, bool BF16>
__global__ __launch_bounds__(512) void head_rows_kernel(HeadRowsArgs a) {
  constexpr int W = 8;
  __shared__ float s_m[W], s_s[W];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  float* const row = a.logits + (int64_t)blockIdx.x * a.ldv;
  const int64_t t = a.t0 + blockIdx.x;
  auto load = [&](int c) {
    f32x4 v = *reinterpret_cast<const f32x4*>(row + c);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e >= a.vocab) v[e] = -__builtin_inff();
    return v;
  };
  float m = -__builtin_inff(), s = 0.f;
  for (int c = tid * 4; c < a.vocab; c += W * 256) {
    const f32x4 v = load(c);
    const float most = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
    if (most > m) {
      s *= __builtin_amdgcn_exp2f((m - most) * LOG2E);
      m = most;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) s += __builtin_amdgcn_exp2f((v[e] - m) * LOG2E);
  }
  const float wm = wave_max(m);
  s = m == wm ? s : s * __builtin_amdgcn_exp2f((m - wm) * LOG2E);
  s = wave_sum(s);
  if (lane == 0) {
    s_m[wave] = wm;
    s_s[wave] = s;
  }
  __syncthreads();
  float top = s_m[0], sum = 0.f;
#pragma unroll
  for (int w = 1; w < W; ++w) top = fmaxf(top, s_m[w]);
#pragma unroll
  for (int w = 0; w < W; ++w) sum += s_s[w] * __builtin_amdgcn_exp2f((s_m[w] - top) * LOG2E);
  const float log_sum = __builtin_amdgcn_logf(sum) * LN2;
  const int32_t target = a.targets[t];
  if (tid == 0) {
    if (a.logp) a.logp[t] = target < 0 ? 0.f : target >= a.vocab ? __builtin_nanf("") : row[target] - top - log_sum;
    if (a.log_z) a.log_z[t] = top + log_sum;
  }
  if constexpr (GRAD) {
    __syncthreads();  // (float32 layers put G where the logits are)
    const float w = target < 0 ? 0.f : target >= a.vocab ? __builtin_nanf("") : a.d_logp[t];
    const float off = top + log_sum;
    for (int c = tid * 4; c < a.ldv; c += W * 256) {
      f32x4 g = c < a.vocab ? load(c) : f32x4{};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p = __builtin_amdgcn_exp2f((g[e] - off) * LOG2E);
        g[e] = c + e >= a.vocab || target < 0 ? 0.f : c + e == target ? w * (1.f - p) : -w * p;
      }
      if constexpr (BF16) {
        bf16x4 h, l;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          h[e] = (bf16_t)g[e];
          l[e] = (bf16_t)(g[e] - (float)h[e]);
        }
        *reinterpret_cast<bf16x4*>(a.hi + (int64_t)blockIdx.x * a.ldv + c) = h;
        *reinterpret_cast<bf16x4*>(a.lo + (int64_t)blockIdx.x * a.ldv + c) = l;
      } else {
        *reinterpret_cast<f32x4*>(row + c) = g;
      }
    }
  }
}

// dX of a piece: its slabs, in order
template <typename T>
__global__ __launch_bounds__(256) void head_join_kernel(const float* slabs, int parts, int64_t stride, int64_t n, T* dX) {
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += (int64_t)gridDim.x * 1024) {  // (n: whole rows of 32 and more columns)
    f32x4 s = *reinterpret_cast<const f32x4*>(slabs + i);
    for (int p = 1; p < parts; ++p) s += *reinterpret_cast<const f32x4*>(slabs + p * stride + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) dX[i + e] = (T)s[e];
  }
}

struct HeadLayout {
  size_t plans, logits, hi, lo, slabs, total;
};
// for shapes of at most `rows` rows a piece
HeadLayout layout_for(int64_t rows, int64_t pieces, int64_t slab_rows, int32_t d, int32_t vocab, bool bf16, bool grad) {
  HeadLayout w = {};
  const size_t cells = (size_t)rows * align_up(vocab, 64);
  w.logits = align_up(sizeof(GemmPlan) * 3 * (size_t)pieces, 256);
  w.hi = w.logits + align_up(cells * 4, 256);
  w.lo = w.hi + (grad && bf16 ? align_up(cells * 2, 256) : 0);
  w.slabs = w.lo + (grad && bf16 ? align_up(cells * 2, 256) : 0);
  w.total = w.slabs + (grad ? (size_t)slab_rows * d * 4 : 0);
  return w;
}
}  // namespace

int64_t head_piece_rows(int32_t vocab) {
  return std::max<int64_t>(256, std::min<int64_t>(8192, PIECE / (int64_t)align_up(vocab, 64) / 256 * 256));
}

size_t head_workspace(int64_t T, int32_t d, int32_t vocab, modse_dtype dt, bool grad) {
  if (T == 0) return 0;
  // of all batches of at most T rows: the most rows of a piece, the most pieces, the most slabs
  const int64_t most = head_piece_rows(vocab), rows = std::min<int64_t>(padded_rows(T), most);
  const int64_t slab_rows = std::min<int64_t>(32 * rows, std::max(SLAB_ROWS, most));
  return ALIGN + layout_for(rows, (T + most - 1) / most, slab_rows, d, vocab, dt == MODSE_BF16, grad).total;
}

hipError_t launch_head(modse_dtype dt, const HeadArgs& a, char* ws, hipStream_t s) {
  const HeadShape h = head_shape(a.T, a.d, a.vocab, dt);
  const bool grad = a.dX || a.dW;
  const HeadLayout w = layout_for(h.rows, h.pieces, (int64_t)h.k_parts * h.rows, h.d, h.vocab, h.bf16, grad);
  ws = reinterpret_cast<char*>(align_up(reinterpret_cast<size_t>(ws), ALIGN));
  const HeadBufs b = {reinterpret_cast<GemmPlan*>(ws + w.plans), reinterpret_cast<float*>(ws + w.logits), reinterpret_cast<bf16_t*>(ws + w.hi),
                      reinterpret_cast<bf16_t*>(ws + w.lo), reinterpret_cast<float*>(ws + w.slabs)};
  const HeadPlanArgs plan = {h, b, a.x, a.W, a.dW, grad};
  hipLaunchKernelGGL(head_plan_kernel, dim3((unsigned)(h.pieces * (grad ? 3 : 1))), dim3(64), 0, s, plan);
  auto tiles = [](int64_t m, int64_t n, TileShape t) { return ((m + t.bm - 1) / t.bm) * ((n + t.bn - 1) / t.bn); };
  hipError_t e = hipGetLastError();
  for (int i = 0; i < h.pieces && e == hipSuccess; ++i) {
    const int64_t t0 = (int64_t)i * h.rows, m = std::min<int64_t>(h.rows, h.T - t0);
    const GemmPlan* const p = b.plans + i * 3;
    e = launch_grouped_gemm(dt, h.bf16 ? EPI_STORE_F32 : EPI_STORE, h.logits_tile, p, h.w_parts, 0, 0,
                            tiles(m, h.vocab, h.logits_tile) + h.w_parts * tiles(m, 1, h.logits_tile), s, LAYOUT_TN);
    if (e != hipSuccess) break;
    const HeadRowsArgs r = {a.targets, a.d_logp, a.logp, a.log_z, b.logits, b.hi, b.lo, t0, (int32_t)m, h.vocab, h.ldv};
    const dim3 grid((unsigned)m), block(512);
    if (!grad) hipLaunchKernelGGL((head_rows_kernel<false, false>), grid, block, 0, s, r);
    else if (h.bf16) hipLaunchKernelGGL((head_rows_kernel<true, true>), grid, block, 0, s, r);
    else hipLaunchKernelGGL((head_rows_kernel<true, false>), grid, block, 0, s, r);
    if ((e = hipGetLastError()) != hipSuccess) break;
    if (a.dW) {  // (before dX, which may lie in the buffer of x)
      e = launch_grouped_gemm(dt, EPI_ROWS_F32, h.dw_tile, p + 2, 1, a.accumulate || i > 0, 0, tiles(padded_rows(h.vocab), h.d, h.dw_tile), s, LAYOUT_AB_K);
      if (e != hipSuccess) break;
    }
    if (a.dX) {
      e = launch_grouped_gemm(dt, EPI_STORE_F32, h.dx_tile, p + 1, h.k_parts, 0, 0, h.k_parts * tiles(m, h.d, h.dx_tile), s, LAYOUT_B_KN);
      if (e != hipSuccess) break;
      const int64_t n = m * h.d, stride = (int64_t)h.rows * h.d;
      const dim3 join((unsigned)std::min<int64_t>((n + 1023) / 1024, 4096));
      if (h.bf16) hipLaunchKernelGGL((head_join_kernel<bf16_t>), join, dim3(256), 0, s, b.slabs, h.k_parts, stride, n, static_cast<bf16_t*>(a.dX) + t0 * h.d);
      else hipLaunchKernelGGL((head_join_kernel<float>), join, dim3(256), 0, s, b.slabs, h.k_parts, stride, n, static_cast<float*>(a.dX) + t0 * h.d);
      e = hipGetLastError();
    }
  }
  return e;
}
