// The norm in front of a layer: h = x + residual, y = gamma h / sqrt(mean(h^2) + eps), optionally y in 8 bits with scales, and
// its backward pass.
//
// All of it is bound by memory: a row is read once, stays in registers as it was loaded, and is written once.  A row belongs to
// one wave (W = 1: no barrier, sums by lane permutes alone), to four waves or to sixteen, each thread holds NC chunks of eight
// elements of it, chunk c of a row going to thread c mod 64 W, so that a wave's accesses are contiguous.
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

typedef uint32_t u32x2_u __attribute__((ext_vector_type(2), aligned(1)));
// eight values as e4m3, rounded to nearest even
__device__ __forceinline__ void store_e4m3(uint8_t* p, const float v[8], int n) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
    w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], r, true);
  }
  if (n >= 8) {
    u32x2_u o = {w[0], w[1]};
    *reinterpret_cast<u32x2_u*>(p) = o;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
  }
}
// (a smaller one has no reciprocal)
constexpr float MIN_SCALE = 1.17549435e-38f;  // 2^-126
__device__ __forceinline__ float scale_of(float amax) { return fmaxf(amax * (1.f / 448.f), MIN_SCALE); }

template <typename T, int W, int NC>
__global__ __launch_bounds__(W == 1 ? 256 : W * 64) void norm_fwd_kernel(NormFwdArgs a) {
  constexpr int ROWS = W == 1 ? 4 : 1;  // of a block
  __shared__ float s_part[16];
  const int at = W == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int d = a.d;
  const T* const x = static_cast<const T*>(a.x);
  const T* const residual = static_cast<const T*>(a.residual);
  T* const y = static_cast<T*>(a.y);
  T* const h = static_cast<T*>(a.h);
  Raw8<T> gamma[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int col = (i * W * 64 + at) * 8;
    load_some(gamma[i], static_cast<const T*>(a.gamma) + col, d - col, 0.f);
  }
  for (int64_t row = (int64_t)blockIdx.x * ROWS + (W == 1 ? threadIdx.x >> 6 : 0); row < a.T; row += (int64_t)gridDim.x * ROWS) {
    const int64_t first = row * d;
    Raw8<T> in[NC], res[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int col = (i * W * 64 + at) * 8;
      load_some(in[i], x + first + col, d - col, 0.f);
      if (residual) load_some(res[i], residual + first + col, d - col, 0.f);
    }
    float v[NC][8], sum = 0.f;
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[i][j] = in[i][j];
        if (residual) v[i][j] += res[i][j];
        sum += v[i][j] * v[i][j];
      }
    sum = row_sum<W>(sum, s_part);
    const float rstd = 1.f / sqrtf(sum / (float)d + a.eps);
    if (a.rstd && at == 0) a.rstd[row] = rstd;
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int col = (i * W * 64 + at) * 8;
      Raw8<T> out;
      if (h) {
#pragma unroll
        for (int j = 0; j < 8; ++j) out.set(j, v[i][j]);
        store_some(out, h + first + col, d - col);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[i][j] *= rstd * gamma[i][j];
        amax = fmaxf(amax, fabsf(v[i][j]));
      }
      if (y) {
#pragma unroll
        for (int j = 0; j < 8; ++j) out.set(j, v[i][j]);
        store_some(out, y + first + col, d - col);
      }
    }
    if (a.q) {
      const int lanes = a.group >> 3;
      float scale = 0.f;
      if (lanes == 0) {
        scale = scale_of(row_max<W>(amax, s_part));
        if (at == 0) a.scale[row] = scale;
      }
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int c = i * W * 64 + at, col = c * 8;
        if (lanes) {
          amax = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf(v[i][j]));
          scale = scale_of(group_max(amax, lanes));
          if (col < d && (c & (lanes - 1)) == 0) a.scale[row * ((d + a.group - 1) / a.group) + c / lanes] = scale;
        }
        const float inv = 1.f / scale;
        float out[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) out[j] = v[i][j] * inv;
        store_e4m3(a.q + first + col, out, d - col);
      }
    }
  }
}

// dX = rstd (g - hat mean(g hat)) + dH with g = dY gamma, hat = h rstd; dgamma = sum of dY hat over the tokens.  A block walks
// over rows, its waves keep their share of dgamma in registers, and the blocks' shares are added up by a second launch in block
// order: the result depends on T and d alone.
template <typename T, int W, int NC>
__global__ __launch_bounds__(W == 1 ? 256 : W * 64) void norm_bwd_kernel(NormBwdArgs a) {
  constexpr int ROWS = W == 1 ? 4 : 1;
  __shared__ float s_part[16];
  __shared__ float s_gamma[W == 1 ? NC * 512 : 1];
  const int at = W == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int d = a.d;
  const T* const h = static_cast<const T*>(a.h);
  const T* const dY = static_cast<const T*>(a.dY);
  const T* const dH = static_cast<const T*>(a.dH);
  T* const dX = static_cast<T*>(a.dX);
  Raw8<T> gamma[NC];
  float share[NC][8];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int col = (i * W * 64 + at) * 8;
    load_some(gamma[i], static_cast<const T*>(a.gamma) + col, d - col, 0.f);
#pragma unroll
    for (int j = 0; j < 8; ++j) share[i][j] = 0.f;
  }
  for (int64_t row = (int64_t)blockIdx.x * ROWS + (W == 1 ? threadIdx.x >> 6 : 0); row < a.T; row += (int64_t)gridDim.x * ROWS) {
    const int64_t first = row * d;
    Raw8<T> hv[NC], dy[NC], dh[NC];
    const float rstd = a.rstd[row];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int col = (i * W * 64 + at) * 8;
      load_some(hv[i], h + first + col, d - col, 0.f);
      load_some(dy[i], dY + first + col, d - col, 0.f);
      if (dH) load_some(dh[i], dH + first + col, d - col, 0.f);
    }
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float t = dy[i][j] * (hv[i][j] * rstd);
        share[i][j] += t;
        dot += t * gamma[i][j];
      }
    dot = row_sum<W>(dot, s_part) / (float)d;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int col = (i * W * 64 + at) * 8;
      Raw8<T> out;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float v = rstd * (dy[i][j] * gamma[i][j] - hv[i][j] * rstd * dot);
        if (dH) v += dh[i][j];
        out.set(j, v);
      }
      store_some(out, dX + first + col, d - col);
    }
  }
  float* const part = a.part + (int64_t)blockIdx.x * d;
  if constexpr (W == 1) {
    const int wave = threadIdx.x >> 6;
#pragma unroll 1
    for (int w = 0; w < 4; ++w) {
      if (wave == w) {
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float* const p = s_gamma + (i * 8 + j) * 64 + at;
            *p = w == 0 ? share[i][j] : *p + share[i][j];
          }
      }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < d; c += 256) part[c] = s_gamma[((c >> 9) * 8 + (c & 7)) * 64 + ((c >> 3) & 63)];
  } else {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int col = (i * W * 64 + at) * 8;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (col + j < d) part[col + j] = share[i][j];
    }
  }
}

// 64 columns per block; sixteen rows of threads share the blocks' shares, then one adds up their sums
__global__ __launch_bounds__(1024) void norm_dgamma_kernel(const float* __restrict__ part, int blocks, int d, int accumulate, float* __restrict__ dgamma) {
  __shared__ float s[16][64];
  const int lane = threadIdx.x & 63, r = threadIdx.x >> 6;
  const int col = blockIdx.x * 64 + lane;
  float v = 0.f;
  if (col < d)
    for (int b = r; b < blocks; b += 16) v += part[(int64_t)b * d + col];
  s[r][lane] = v;
  __syncthreads();
  if (r == 0 && col < d) {
#pragma unroll
    for (int i = 1; i < 16; ++i) v += s[i][lane];
    dgamma[col] = accumulate ? dgamma[col] + v : v;
  }
}

template <typename T, int W, int NC>
hipError_t norm_fwd(const NormFwdArgs& a, hipStream_t s) {
  const int64_t blocks = W == 1 ? (a.T + 3) / 4 : a.T;
  hipLaunchKernelGGL((norm_fwd_kernel<T, W, NC>), dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(W == 1 ? 256 : W * 64), 0, s, a);
  return hipGetLastError();
}
template <typename T>
hipError_t norm_fwd_any(const NormFwdArgs& a, hipStream_t s) {
  const int chunks = (a.d + 7) / 8;
  const bool few = a.T < 1024;
  if (chunks <= 64) return norm_fwd<T, 1, 1>(a, s);
  if (chunks <= 128) return norm_fwd<T, 1, 2>(a, s);
  if (!few && chunks <= 256) return norm_fwd<T, 1, 4>(a, s);
  if (chunks <= 256) return norm_fwd<T, 4, 1>(a, s);
  if (chunks <= 512) return norm_fwd<T, 4, 2>(a, s);
  if (chunks <= 1024) return norm_fwd<T, 4, 4>(a, s);
  return norm_fwd<T, 16, 2>(a, s);
}

template <typename T, int W, int NC>
hipError_t norm_bwd(const NormBwdArgs& a, hipStream_t s) {
  const int blocks = norm_bwd_blocks(a.T, a.d);
  hipLaunchKernelGGL((norm_bwd_kernel<T, W, NC>), dim3(blocks), dim3(W == 1 ? 256 : W * 64), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(norm_dgamma_kernel, dim3((a.d + 63) / 64), dim3(1024), 0, s, a.part, blocks, a.d, a.accumulate, a.dgamma);
  return hipGetLastError();
}
constexpr int BWD_ONE_WAVE_CHUNKS = 256;  // rows of at most so many chunks belong to one wave
template <typename T>
hipError_t norm_bwd_any(const NormBwdArgs& a, hipStream_t s) {
  const int chunks = (a.d + 7) / 8;
  if (chunks <= 64) return norm_bwd<T, 1, 1>(a, s);
  if (chunks <= 128) return norm_bwd<T, 1, 2>(a, s);
  if (chunks <= BWD_ONE_WAVE_CHUNKS) return norm_bwd<T, 1, 4>(a, s);
  if (chunks <= 512) return norm_bwd<T, 4, 2>(a, s);
  if (chunks <= 1024) return norm_bwd<T, 4, 4>(a, s);
  return norm_bwd<T, 16, 2>(a, s);
}
}  // namespace

int norm_bwd_blocks(int64_t T, int32_t d) {
  const int64_t rows = (d + 7) / 8 <= BWD_ONE_WAVE_CHUNKS ? 4 : 1, most = rows == 4 ? 512 : 768;
  const int64_t blocks = (T + rows - 1) / rows;
  return (int)(blocks < most ? blocks : most);
}
hipError_t launch_norm_fwd(modse_dtype dt, const NormFwdArgs& a, hipStream_t s) {
  return dt == MODSE_F32 ? norm_fwd_any<float>(a, s) : norm_fwd_any<bf16_t>(a, s);
}
hipError_t launch_norm_bwd(modse_dtype dt, const NormBwdArgs& a, hipStream_t s) {
  return dt == MODSE_F32 ? norm_bwd_any<float>(a, s) : norm_bwd_any<bf16_t>(a, s);
}
