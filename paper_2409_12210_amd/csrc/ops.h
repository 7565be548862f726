// Internal declarations of the operators around the layer: norm and log probabilities (gfx950 only).
#pragma once
#include "common.h"

#define MODSE_NORM_MAX_D 16384

// norm.hip
struct NormFwdArgs {
  const void *x, *residual, *gamma;
  void *y, *h;
  float* rstd;
  uint8_t* q;
  float* scale;
  int64_t T;
  int32_t d, group;
  float eps;
};
hipError_t launch_norm_fwd(modse_dtype dt, const NormFwdArgs& a, hipStream_t s);

struct NormBwdArgs {
  const void *h, *gamma;
  const float* rstd;
  const void *dY, *dH;
  void* dX;
  float* dgamma;
  float* part;  // [norm_bwd_blocks, d] shares of dgamma
  int64_t T;
  int32_t d, accumulate;
};
int norm_bwd_blocks(int64_t T, int32_t d);
hipError_t launch_norm_bwd(modse_dtype dt, const NormBwdArgs& a, hipStream_t s);

// logprobs.hip
struct LogprobsFwdArgs {
  const void* logits;
  int64_t ld;
  const int32_t* targets;
  float *logp, *stats, *entropy;
  int32_t* top_idx;
  float* top_logp;
  f32x4* part;       // [T, splits] maximum, sum, weighted sum of a row's segments
  uint64_t* keys;    // [T, splits, top] their most probable entries
  int64_t T;
  int32_t vocab, top;
};
struct LogprobsSplit {
  int32_t splits, segment;  // blocks of a row, entries of each but the last
};
LogprobsSplit logprobs_split(int64_t T, int32_t vocab, int32_t top);
hipError_t launch_logprobs_fwd(modse_dtype dt, const LogprobsFwdArgs& a, LogprobsSplit split, hipStream_t s);

struct LogprobsBwdArgs {
  const void* logits;
  int64_t ld;
  const int32_t* targets;
  const float *stats, *entropy, *d_logp, *d_entropy;
  void* d_logits;
  int64_t ldd;
  int64_t T;
  int32_t vocab;
};
hipError_t launch_logprobs_bwd(modse_dtype dt, const LogprobsBwdArgs& a, hipStream_t s);

// ---------------------------------------------------------------- rows of any alignment
// Eight elements of a row that starts anywhere: gfx950 takes 16-byte accesses at the alignment of the element, so a row of
// odd length needs no path of its own.  `n`: elements that there are (the rest reads 0).
typedef f32x4 f32x4_u __attribute__((aligned(4)));
typedef bf16x8 bf16x8_u __attribute__((aligned(2)));
template <typename T> struct Raw8;
template <> struct Raw8<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const f32x4_u*>(p);
    b = *reinterpret_cast<const f32x4_u*>(p + 4);
  }
  __device__ __forceinline__ float operator[](int i) const { return i < 4 ? a[i] : b[i - 4]; }
  __device__ __forceinline__ void set(int i, float v) { if (i < 4) a[i] = v; else b[i - 4] = v; }
  __device__ __forceinline__ void store(float* p) const {
    *reinterpret_cast<f32x4_u*>(p) = a;
    *reinterpret_cast<f32x4_u*>(p + 4) = b;
  }
};
template <> struct Raw8<bf16_t> {
  bf16x8 a;
  __device__ __forceinline__ void load(const bf16_t* p) { a = *reinterpret_cast<const bf16x8_u*>(p); }
  __device__ __forceinline__ float operator[](int i) const { return (float)a[i]; }
  __device__ __forceinline__ void set(int i, float v) { a[i] = (bf16_t)v; }
  __device__ __forceinline__ void store(bf16_t* p) const { *reinterpret_cast<bf16x8_u*>(p) = a; }
};
template <typename T>
__device__ __forceinline__ void load_some(Raw8<T>& r, const T* p, int n, float rest) {
  if (n >= 8) {
    r.load(p);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.set(i, i < n ? (float)p[i] : rest);
  }
}
template <typename T>
__device__ __forceinline__ void store_some(const Raw8<T>& r, T* p, int n) {
  if (n >= 8) {
    r.store(p);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (T)r[i];
  }
}

// ---------------------------------------------------------------- reductions over a wave by lane permutes of the vector unit
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float dpp_f32(float old, float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, old), __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float lane_f32(float v, int lane) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}
// (lanes to the right within a row of sixteen, then row 0 to 1 and 2 to 3, then the lower half to the upper: lane 63 has it all)
__device__ __forceinline__ float wave_sum(float v) {
  v += dpp_f32<0x111>(0.f, v);
  v += dpp_f32<0x112>(0.f, v);
  v += dpp_f32<0x114>(0.f, v);
  v += dpp_f32<0x118>(0.f, v);
  v += dpp_f32<0x142, 0xa>(0.f, v);
  v += dpp_f32<0x143, 0xc>(0.f, v);
  return lane_f32(v, 63);
}
__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, dpp_f32<0x111>(v, v));
  v = fmaxf(v, dpp_f32<0x112>(v, v));
  v = fmaxf(v, dpp_f32<0x114>(v, v));
  v = fmaxf(v, dpp_f32<0x118>(v, v));
  v = fmaxf(v, dpp_f32<0x142, 0xa>(v, v));
  v = fmaxf(v, dpp_f32<0x143, 0xc>(v, v));
  return lane_f32(v, 63);
}
// the maximum of every aligned group of 4, 8 or 16 lanes, in all of them
__device__ __forceinline__ float group_max(float v, int lanes) {
  v = fmaxf(v, dpp_f32<0xb1>(v, v));    // lane ^ 1
  v = fmaxf(v, dpp_f32<0x4e>(v, v));    // lane ^ 2
  if (lanes >= 8) v = fmaxf(v, dpp_f32<0x141>(v, v));   // 7 - lane: the other half of eight
  if (lanes >= 16) v = fmaxf(v, dpp_f32<0x140>(v, v));  // 15 - lane
  return v;
}
