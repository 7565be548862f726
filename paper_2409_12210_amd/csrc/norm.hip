// The norm in front of a layer: h = x + residual, y = gamma h / sqrt(mean(h^2) + eps), optionally y in 8 bits with scales, and
// its backward pass.
//
// All of it is bound by memory: a row is read once, stays in registers as it was loaded, and is written once.  A row belongs to
// one wave (W = 1: no barrier, sums by lane permutes alone), to four waves or to sixteen, each thread holds NC vectors of sixteen
// bytes of it, vector c of a row going to thread c mod 64 W, so that a wave's accesses are contiguous.  Calls of few rows cost
// their launch: one token of width 4096 is 2.6 us of kernel and 5.3 a call, and the forward is one launch for that reason.
#include "ops.h"

namespace {

// the sum / maximum over the W waves that share a row; `s`: W floats.  (Two barriers, so that `s` may be used again.)
template <int W>
__device__ __forceinline__ float row_sum(float v, float* s) {
  v = wave_sum(v);
  if constexpr (W > 1) {
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = s[0];
#pragma unroll
    for (int i = 1; i < W; ++i) v += s[i];
    __syncthreads();
  }
  return v;
}
template <int W>
__device__ __forceinline__ float row_max(float v, float* s) {
  v = wave_max(v);
  if constexpr (W > 1) {
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = s[0];
#pragma unroll
    for (int i = 1; i < W; ++i) v = fmaxf(v, s[i]);
    __syncthreads();
  }
  return v;
}

// N values (4 or 8) as e4m3, rounded to nearest even
template <int N>
__device__ __forceinline__ void store_e4m3(uint8_t* p, const float (&v)[N], int n) {
  typedef uint32_t words __attribute__((ext_vector_type(N / 4)));
  typedef words words_u __attribute__((aligned(1)));
  words w;
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const int r = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
    w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], r, true);
  }
  if (n >= N) {
    *reinterpret_cast<words_u*>(p) = w;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) p[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
  }
}
// (a smaller one has no reciprocal)
constexpr float MIN_SCALE = 1.17549435e-38f;  // 2^-126
// From v = h gamma (exact for bf16 tensors of like size) and its largest value of a group: the scale of y = v rstd is
// amax rstd / 448, and y / scale = 448 v / amax, which is rounded once before it is rounded to e4m3.  (y / scale from a rounded y
// and scale falls on the other side of a tie for one value in a few million.)
struct E4m3Scale {
  float scale, factor, below, inv;
  __device__ __forceinline__ void set(float amax, float rstd) {
    const float s = amax * rstd * (1.f / 448.f);
    scale = fmaxf(s, MIN_SCALE);  // (of NaN: the other)
    const bool usual = s > MIN_SCALE && amax > 0x1p-100f && amax < 0x1p100f;  // else 448 v or 1 / amax may leave float32
    factor = usual ? 448.f : rstd;
    below = usual ? amax : scale;
    inv = __builtin_amdgcn_rcpf(below);
  }
  __device__ __forceinline__ float operator()(float v) const {
    v *= factor;
    const float q = v * inv;
    return __builtin_amdgcn_div_fixupf(__builtin_fmaf(__builtin_fmaf(-q, below, v), inv, q), below, v);
  }
};

// Two tensors in, two out, 5 operations a value: 32768 tokens of width 2048 in bf16 take 92 us, 5.8 TB/s (a sum of two large tensors
// into a third reaches 6.2); 16384 of them with y in e4m3 and a scale per 128 columns alone 40 us, 5.9 TB/s.  gamma stays in the
// registers of a wave, which walks over rows; all of a row's loads are in flight before the first is used.
template <typename T, int W, int NC, bool STREAM>
__global__ __launch_bounds__(W == 1 ? 256 : W * 64) void norm_fwd_kernel(NormFwdArgs a) {
  constexpr int ROWS = W == 1 ? 4 : 1;  // of a block
  constexpr int N = Vec<T>::N;
  __shared__ float s_part[16];
  const int at = W == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int d = a.d;
  const T* const x = static_cast<const T*>(a.x);
  const T* const residual = static_cast<const T*>(a.residual);
  T* const y = static_cast<T*>(a.y);
  T* const h = static_cast<T*>(a.h);
  Vec<T> gamma[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int col = (i * W * 64 + at) * N;
    gamma[i].load(static_cast<const T*>(a.gamma) + col, d - col, 0.f);
  }
  for (int64_t row = (int64_t)blockIdx.x * ROWS + (W == 1 ? threadIdx.x >> 6 : 0); row < a.T; row += (int64_t)gridDim.x * ROWS) {
    const int64_t first = row * d;
    Vec<T> in[NC], res[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int col = (i * W * 64 + at) * N;
      in[i].template load<STREAM>(x + first + col, d - col, 0.f);
      if (residual) res[i].template load<STREAM>(residual + first + col, d - col, 0.f);
    }
    float v[NC][N], sum = 0.f;
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        v[i][j] = in[i][j];
        if (residual) v[i][j] += res[i][j];
        sum += v[i][j] * v[i][j];
      }
#pragma unroll
    for (int i = 0; i < NC; ++i) gamma[i].forget();
    sum = row_sum<W>(sum, s_part);
    const float rstd = 1.f / sqrtf(sum / (float)d + a.eps);
    if (a.rstd && at == 0) a.rstd[row] = rstd;
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int col = (i * W * 64 + at) * N;
      Vec<T> out;
      if (h) {
#pragma unroll
        for (int j = 0; j < N; ++j) out.set(j, v[i][j]);
        out.template store<true>(h + first + col, d - col);
      }
#pragma unroll
      for (int j = 0; j < N; ++j) {
        v[i][j] *= gamma[i][j];
        amax = fmaxf(amax, fabsf(v[i][j]));
      }
      if (y) {
#pragma unroll
        for (int j = 0; j < N; ++j) out.set(j, v[i][j] * rstd);
        out.store(y + first + col, d - col);
      }
    }
    if (a.q) {
      const int lanes = a.group / N;
      E4m3Scale to;
      if (lanes == 0) {
        to.set(row_max<W>(amax, s_part), rstd);
        if (at == 0) a.scale[row] = to.scale;
      }
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int c = i * W * 64 + at, col = c * N;
        if (lanes) {
          amax = 0.f;
#pragma unroll
          for (int j = 0; j < N; ++j) amax = fmaxf(amax, fabsf(v[i][j]));
          to.set(group_max(amax, lanes), rstd);
          if (col < d && (c & (lanes - 1)) == 0) a.scale[row * ((d + a.group - 1) / a.group) + c / lanes] = to.scale;
        }
        float out[N];
#pragma unroll
        for (int j = 0; j < N; ++j) out[j] = to(v[i][j]);
        store_e4m3(a.q + first + col, out, d - col);
      }
    }
  }
}

// dgamma of LANES vectors' worth of columns, over all tokens: LANES threads a row, as many rows at a time as the block has threads
// for, four of them of a thread in flight.  The result depends on T and d alone.
template <typename T, int THREADS, int LANES>
__device__ __forceinline__ void norm_bwd_columns(const NormBwdArgs& a, int block) {
  constexpr int N = Vec<T>::N, ROWS = THREADS / LANES, AT_ONCE = 4;
  __shared__ float s_sum[THREADS / 64][LANES * N];
  const int lane = threadIdx.x % LANES, row0 = threadIdx.x / LANES, col = (block * LANES + lane) * N, d = a.d;
  const T* const h = static_cast<const T*>(a.h);
  const T* const dY = static_cast<const T*>(a.dY);
  float sum[N];
#pragma unroll
  for (int j = 0; j < N; ++j) sum[j] = 0.f;
  for (int64_t first = row0; first < a.T; first += ROWS * AT_ONCE) {
    Vec<T> hv[AT_ONCE], dy[AT_ONCE];
    float rstd[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int64_t row = first + i * ROWS;
      const int n = row < a.T ? d - col : 0;
      hv[i].load(h + row * d + col, n, 0.f);
      dy[i].load(dY + row * d + col, n, 0.f);
      rstd[i] = row < a.T ? a.rstd[row] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) sum[j] += dy[i][j] * (hv[i][j] * rstd[i]);
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
#pragma unroll
    for (int k = LANES; k < 64; k *= 2) sum[j] += __shfl_xor(sum[j], k, 64);
    if ((threadIdx.x & 63) < LANES) s_sum[threadIdx.x >> 6][lane * N + j] = sum[j];
  }
  __syncthreads();
  const int c = block * LANES * N + threadIdx.x;
  if (threadIdx.x < LANES * N && c < d) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) v += s_sum[w][threadIdx.x];
    a.dgamma[c] = a.accumulate ? a.dgamma[c] + v : v;
  }
}

constexpr int column_lanes(int w) { return w == 16 ? 8 : 4; }  // of W waves a row

// dX = rstd (g - hat mean(g hat)) + dH with g = dY gamma, hat = h rstd; dgamma = sum of dY hat over the tokens.  A block walks
// over rows, its waves keep their share of dgamma in registers, and the blocks' shares are added up by a second launch in block
// order: the result depends on T and d alone.  Three tensors in, one out: 32768 tokens of width 2048 in bf16 take 95 us, 5.7 TB/s, and
// the second launch 5.  With FEW rows the first `columns` blocks read h and dY once more, for dgamma alone, and there is no second launch:
// 128 tokens of width 4096 4.0 us instead of 8.3, and a launch less of the host's time.
template <typename T, int W, int NC, bool STREAM, bool FEW>
__global__ __launch_bounds__(W == 1 ? 256 : W * 64) void norm_bwd_kernel(NormBwdArgs a, int columns) {
  constexpr int ROWS = W == 1 ? 4 : 1;
  constexpr int N = Vec<T>::N, WIDTH = NC * N * 64;  // columns of a wave
  __shared__ float s_part[16];
  __shared__ float s_gamma[W == 1 && !FEW ? 4 : 1][W == 1 && !FEW ? WIDTH : 1];
  if constexpr (FEW) {
    if ((int)blockIdx.x < columns) {
      norm_bwd_columns<T, W == 1 ? 256 : W * 64, column_lanes(W)>(a, blockIdx.x);
      return;
    }
  }
  const int block = FEW ? blockIdx.x - columns : blockIdx.x, blocks = FEW ? gridDim.x - columns : gridDim.x;
  const int at = W == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int d = a.d;
  const T* const h = static_cast<const T*>(a.h);
  const T* const dY = static_cast<const T*>(a.dY);
  const T* const dH = static_cast<const T*>(a.dH);
  T* const dX = static_cast<T*>(a.dX);
  Vec<T> gamma[NC];
  float share[NC][N];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int col = (i * W * 64 + at) * N;
    gamma[i].load(static_cast<const T*>(a.gamma) + col, d - col, 0.f);
#pragma unroll
    for (int j = 0; j < N; ++j) share[i][j] = 0.f;
  }
  for (int64_t row = (int64_t)block * ROWS + (W == 1 ? threadIdx.x >> 6 : 0); row < a.T; row += (int64_t)blocks * ROWS) {
    const int64_t first = row * d;
    Vec<T> hv[NC], dy[NC], dh[NC];
    const float rstd = a.rstd[row];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int col = (i * W * 64 + at) * N;
      hv[i].template load<STREAM>(h + first + col, d - col, 0.f);
      dy[i].template load<STREAM>(dY + first + col, d - col, 0.f);
      if (dH && W < 16) dh[i].template load<STREAM>(dH + first + col, d - col, 0.f);
    }
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float t = dy[i][j] * (hv[i][j] * rstd);
        if constexpr (!FEW) share[i][j] += t;
        dot += t * gamma[i][j];
      }
    }
    // (the row waits in the form it was loaded in: bf16 as float32 takes 201 registers at NC = 4 where 156 do, and fewer waves fit)
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      hv[i].forget();
      dy[i].forget();
      gamma[i].forget();
    }
    dot = row_sum<W>(dot, s_part) / (float)d;
    const float k = rstd * rstd * dot;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int col = (i * W * 64 + at) * N;
      if (dH && W == 16) dh[i].template load<STREAM>(dH + first + col, d - col, 0.f);  // (128 registers do not hold it with the rest)
      Vec<T> out;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        float v = (rstd * gamma[i][j]) * dy[i][j] - hv[i][j] * k;
        if (dH) v += dh[i][j];
        out.set(j, v);
      }
      out.store(dX + first + col, d - col);
    }
  }
  if constexpr (FEW) return;
  float* const part = a.part + (int64_t)blockIdx.x * d;
  if constexpr (W == 1 && !FEW) {
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) s_gamma[threadIdx.x >> 6][(i * N + j) * 64 + at] = share[i][j];
    __syncthreads();
    for (int c = threadIdx.x; c < d; c += 256) {
      const int k = (c / (64 * N) * N + c % N) * 64 + c / N % 64;
      part[c] = (s_gamma[0][k] + s_gamma[1][k]) + (s_gamma[2][k] + s_gamma[3][k]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int col = (i * W * 64 + at) * N;
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (col + j < d) part[col + j] = share[i][j];
    }
  }
}

// dgamma = the sum of the blocks' shares (4 MB of them at most at width 2048: they are in the caches, and the launch counts, 5 us).
// Sixteen columns per block: 64 rows of threads share the blocks' shares, and their sums are added up in two steps
__global__ __launch_bounds__(1024) void norm_dgamma_kernel(const float* __restrict__ part, int blocks, int d, int accumulate, float* __restrict__ dgamma) {
  __shared__ float s[64][17];
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4;
  const int col = blockIdx.x * 16 + c;
  float v = 0.f;
  if (col < d) {
#pragma unroll 4
    for (int b = r; b < blocks; b += 64) v += part[(int64_t)b * d + col];
  }
  s[r][c] = v;
  __syncthreads();
  if (r < 4) {
    v = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) v += s[r * 16 + i][c];
    v += __shfl_xor(v, 16, 64);
    v += __shfl_xor(v, 32, 64);
    if (r == 0 && col < d) dgamma[col] = accumulate ? dgamma[col] + v : v;
  }
}

// Tensors of 64 MB and more are read with the non-temporal hint: neither this nor another operator's caches will hold them.  us
// without / with it, d = 2048, bf16: 32768 tokens forward 91.7 / 90.6, into e4m3 81.7 / 74.3, backward 100 / 97; 16384 tokens (64
// MB) 48.9 / 45.0, 43.4 / 40.6; 8192 tokens 25.3 / 26.0, 20.1 / 23.4; 4096 tokens, whose inputs are in the caches, 11.1 / 15.1.  h is stored
// with the hint at every size (nothing reads it before the next norm or the backward pass: 8192 tokens into e4m3 25.0 / 20.1, forward
// and the router behind it 53.1 / 51.2), y without (the router reads it next: 4096 tokens, both 41.1 / 47.1).
constexpr int64_t STREAM_BYTES = (int64_t)64 << 20;

// Blocks of the forward pass, at most.  us of the GPU with 2048 / 8192 / as many as the rows are worth: bf16 32768 x 2048 80 / 79 / 79, 131072 x
// 2048 394 / 391 / 363, 32768 x 8192 399 / 393 / 363, 16384 x 16384 410 / 387 / 390; float32 131072 x 2048 821 / 805 / 800.  (A launch has
// fewer than 2^32 threads.)
constexpr int64_t FWD_BLOCKS = 1 << 16;
template <typename T, int W, int NC>
hipError_t norm_fwd(const NormFwdArgs& a, hipStream_t s) {
  const int64_t blocks = W == 1 ? (a.T + 3) / 4 : a.T;
  const dim3 grid((unsigned)(blocks < FWD_BLOCKS ? blocks : FWD_BLOCKS)), block(W == 1 ? 256 : W * 64);
  if (a.T * a.d * (int64_t)sizeof(T) >= STREAM_BYTES) hipLaunchKernelGGL((norm_fwd_kernel<T, W, NC, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((norm_fwd_kernel<T, W, NC, false>), grid, block, 0, s, a);
  return hipGetLastError();
}
// Rows of 1025 to 2048 values belong to four waves where there are few of them.  us of the GPU, four waves / one, by rows: bf16, 2048 wide, 64 2.6 /
// 3.9, 1023 4.0 / 4.8, 1536 4.8 / 5.4, 2048 5.5 / 6.1, 4096 10.9 / 10.5, 32768 80 / 79; 1100 wide, 64 3.0 / 4.9, 1536 5.3 / 6.1, 2048 6.1 / 6.3,
// 4096 9.6 / 8.8, 32768 80 / 67; float32, 2048 wide, 64 2.8 / 4.6, 1536 6.9 / 8.4, 2048 10.9 / 10.4, 4096 20.3 / 21.4, 32768 155 / 161.
// (vectors of a thread: float32 has twice as many of them in a row)
template <typename T>
hipError_t norm_fwd_any(const NormFwdArgs& a, hipStream_t s) {
  constexpr int X = 8 / Vec<T>::N;
  const int chunks = (a.d + 7) / 8;
  const bool few = a.T < 2048;
  if (chunks <= 64) return norm_fwd<T, 1, X>(a, s);
  if (chunks <= 128) return norm_fwd<T, 1, 2 * X>(a, s);
  if (!few && chunks <= 256) return norm_fwd<T, 1, 4 * X>(a, s);
  if (chunks <= 256) return norm_fwd<T, 4, X>(a, s);
  if (chunks <= 512) return norm_fwd<T, 4, 2 * X>(a, s);
  if (chunks <= 1024) return norm_fwd<T, 4, 4 * X>(a, s);
  return norm_fwd<T, 16, 2 * X>(a, s);
}

// us of the GPU with a second launch / without, by tokens: width 512 bf16 1: 4.2 / 4.1, 512: 4.9 / 4.0, 1021: 5.0 / 5.9; 1535 float32 128:
// 7.3 / 4.4, 512: 8.8 / 6.6, 1021: 11.1 / 10.6 (but with the forward pass in front of it 15.9 / 16.6); 4096 bf16 128: 8.3 / 4.0, 512: 13.6 /
// 8.1, 2048: 21.1 / 22.6; 16384 bf16 1: 13.7 / 6.5, 512: 28 / 18, 2048: 62 / 74.  (The launch costs the host another 4 to 5.)  Eight lanes a
// row of columns where rows have sixteen waves: 512 tokens of width 16384 26 -> 18; four elsewhere: 1021 of 2048 12.1 -> 10.5.
constexpr int64_t FEW_ROWS = 512;
template <typename T, int W, int NC>
hipError_t norm_bwd(const NormBwdArgs& a, hipStream_t s) {
  const dim3 block(W == 1 ? 256 : W * 64);
  if (a.T <= FEW_ROWS) {
    const int rows = (int)(W == 1 ? (a.T + 3) / 4 : a.T), of_block = column_lanes(W) * Vec<T>::N, columns = (a.d + of_block - 1) / of_block;
    const size_t bytes = (size_t)a.T * a.d * sizeof(T);
    auto over = [&](const void* p) {
      const uintptr_t x = (uintptr_t)p, y = (uintptr_t)a.dX;
      return x < y + bytes && y < x + bytes;
    };
    if (!over(a.h) && !over(a.dY)) {
      hipLaunchKernelGGL((norm_bwd_kernel<T, W, NC, false, true>), dim3(columns + rows), block, 0, s, a, columns);
      return hipGetLastError();
    }
    // dX takes the place of what dgamma is made of: one behind the other
    hipLaunchKernelGGL((norm_bwd_kernel<T, W, NC, false, true>), dim3(columns), block, 0, s, a, columns);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((norm_bwd_kernel<T, W, NC, false, true>), dim3(rows), block, 0, s, a, 0);
    return hipGetLastError();
  }
  const int blocks = norm_bwd_blocks(a.T, a.d);
  if (a.T * a.d * (int64_t)sizeof(T) >= STREAM_BYTES) hipLaunchKernelGGL((norm_bwd_kernel<T, W, NC, true, false>), dim3(blocks), block, 0, s, a, 0);
  else hipLaunchKernelGGL((norm_bwd_kernel<T, W, NC, false, false>), dim3(blocks), block, 0, s, a, 0);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(norm_dgamma_kernel, dim3((a.d + 15) / 16), dim3(1024), 0, s, a.part, blocks, a.d, a.accumulate, a.dgamma);
  return hipGetLastError();
}
constexpr int BWD_ONE_WAVE_CHUNKS = 256;  // rows of at most so many eights belong to one wave
template <typename T>
hipError_t norm_bwd_any(const NormBwdArgs& a, hipStream_t s) {
  constexpr int X = 8 / Vec<T>::N;
  const int chunks = (a.d + 7) / 8;
  if (chunks <= 64) return norm_bwd<T, 1, X>(a, s);
  if (chunks <= 128) return norm_bwd<T, 1, 2 * X>(a, s);
  if (chunks <= BWD_ONE_WAVE_CHUNKS) return norm_bwd<T, 1, 4 * X>(a, s);
  if (chunks <= 512) return norm_bwd<T, 4, 2 * X>(a, s);
  if (chunks <= 1024) return norm_bwd<T, 4, 4 * X>(a, s);
  return norm_bwd<T, 16, 2 * X>(a, s);
}
}  // namespace

// Each block writes a share of dgamma that the second launch reads, and more blocks than the row loop needs leave the last of them
// alone with the memory.  us a call with 256 / 512 / 768 blocks, bf16: one wave a row 32768 x 2048 112 / 97 / 101, 4096 x 2048 18.5 / 17.1 / -,
// 2048 x 2048 13.2 / 14.0 / 14.0; four waves a row 16384 x 4096 123 / 100 / 111, 8192 x 8192 113 / 104 / 114, 512 x 4096 12.9 / 16.8 / 16.8; sixteen
// waves, one block a compute unit, 4096 x 16384 110 / 121 / -.
int norm_bwd_blocks(int64_t T, int32_t d) {
  const int chunks = (d + 7) / 8, rows = chunks <= BWD_ONE_WAVE_CHUNKS ? 4 : 1;  // of a block at a time
  const int64_t most = chunks <= 1024 ? 512 : 256, some = T / 8;
  const int64_t blocks = (T + rows - 1) / rows, wanted = some < 256 ? 256 : some < most ? some : most;
  return (int)(blocks < wanted ? blocks : wanted);
}
hipError_t launch_norm_fwd(modse_dtype dt, const NormFwdArgs& a, hipStream_t s) {
  return dt == MODSE_F32 ? norm_fwd_any<float>(a, s) : norm_fwd_any<bf16_t>(a, s);
}
hipError_t launch_norm_bwd(modse_dtype dt, const NormBwdArgs& a, hipStream_t s) {
  return dt == MODSE_F32 ? norm_bwd_any<float>(a, s) : norm_bwd_any<bf16_t>(a, s);
}
