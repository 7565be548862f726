// Internal declarations of the operators around the layer (gfx950 only).
#pragma once
#include <algorithm>

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

// dropout.hip
struct DropoutArgs {
  const void *x, *residual;
  void* y;
  const uint64_t* rng;  // seed, offset
  int64_t n;            // elements
  uint32_t call, limit; // kept: 16 random bits of at least `limit`
  float scale;
};
hipError_t launch_dropout(modse_dtype dt, const DropoutArgs& a, hipStream_t s);

// embed.hip
#define MODSE_MAX_VOCAB (1 << 20)
constexpr int EMBED_MAX_ROWS = 512;  // of the vocabulary that one block sorts
struct EmbedFwdArgs {
  const int32_t* tokens;
  const void* E;
  void* x;
  int64_t T;
  int32_t d, vocab;
  float scale;
};
hipError_t launch_embed_fwd(modse_dtype dt, const EmbedFwdArgs& a, hipStream_t s);

struct EmbedBwdArgs {
  const int32_t* tokens;
  const void* dX;
  float* dE;
  int32_t* n_sorted;  // [1] tokens of the vocabulary
  int32_t* order;     // [T] their places in the batch, by token and then by place
  int32_t* keys;      // [T] the tokens themselves in that order
  float* part;        // [2 ceil(T / chunk), part_ld] partial sums of runs that cross chunks
  int64_t T;
  int32_t d, vocab, chunk, part_ld, accumulate;
  float scale;
};
// Places of the sorted list that are summed together, 64 at the most.
inline int embed_chunk(int64_t T) { return T <= 8192 ? 8 : T <= 32768 ? 32 : 64; }
inline int64_t embed_chunks(int64_t T) { return (T + embed_chunk(T) - 1) / embed_chunk(T); }
// the most chunks of all batches of at most T tokens
inline int64_t embed_most_chunks(int64_t T) {
  return std::max(embed_chunks(T), std::max(embed_chunks(std::min<int64_t>(T, 8192)), embed_chunks(std::min<int64_t>(T, 32768))));
}
hipError_t launch_embed_bwd(modse_dtype dt, const EmbedBwdArgs& a, hipStream_t s);

// head.hip
struct HeadArgs {
  const void *x, *W;
  const int32_t* targets;
  const float* d_logp;
  float *logp, *log_z;
  void* dX;   // with dX or dW: gradients
  float* dW;
  int64_t T;
  int32_t d, vocab, accumulate;
};
size_t head_workspace(int64_t T, int32_t d, int32_t vocab, modse_dtype dt, bool grad);
hipError_t launch_head(modse_dtype dt, const HeadArgs& a, char* ws, hipStream_t s);

// ---------------------------------------------------------------- rows of any alignment
// Sixteen bytes of a row that starts anywhere: gfx950 takes such accesses at the alignment of the element, so a row of odd length
// needs no path of its own.  Neighbouring lanes take neighbouring vectors.  (Eight float32 per lane, in two loads half of whose
// bytes lie between the other's, read 4096 x 4096 with the non-temporal hint at 4.7 TB/s; this way 5.4.)
template <typename T> struct VecOf;
template <> struct VecOf<float> { typedef f32x4 type; };
template <> struct VecOf<bf16_t> { typedef bf16x8 type; };
template <typename T>
struct Vec {
  static constexpr int N = 16 / sizeof(T);
  typedef typename VecOf<T>::type V;
  typedef V V_u __attribute__((aligned(sizeof(T))));
  V v;
  __device__ __forceinline__ float operator[](int i) const { return (float)v[i]; }
  __device__ __forceinline__ void set(int i, float x) { v[i] = (T)x; }
  // what was computed from it is not kept in registers
  __device__ __forceinline__ void forget() {
    u32x4 t = __builtin_bit_cast(u32x4, v);
    asm volatile("" : "+v"(t));
    v = __builtin_bit_cast(V, t);
  }
  // the first n elements that there are from p on; the others become `rest`.  STREAM: with the non-temporal hint
  template <bool STREAM = false>
  __device__ __forceinline__ void load(const T* p, int n, float rest) {
    if (n >= N) {
      if constexpr (STREAM) v = __builtin_nontemporal_load(reinterpret_cast<const V_u*>(p));
      else v = *reinterpret_cast<const V_u*>(p);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = i < n ? p[i] : (T)rest;
    }
  }
  template <bool STREAM = false>
  __device__ __forceinline__ void store(T* p, int n) const {
    if (n >= N) {
      if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<V_u*>(p));
      else *reinterpret_cast<V_u*>(p) = v;
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i < n) p[i] = v[i];
    }
  }
};

// ---------------------------------------------------------------- reductions over a wave by lane permutes of the vector unit
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float dpp_f32(float old, float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, old), __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float lane_f32(float v, int lane) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}
__device__ __forceinline__ void wave_lds_order() {  // LDS writes of this wave's lanes are there for its other lanes
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
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
// the maximum of every aligned group of 4, 8, 16 or 32 lanes, in all of them
__device__ __forceinline__ float group_max(float v, int lanes) {
  v = fmaxf(v, dpp_f32<0xb1>(v, v));    // lane ^ 1
  v = fmaxf(v, dpp_f32<0x4e>(v, v));    // lane ^ 2
  if (lanes >= 8) v = fmaxf(v, dpp_f32<0x141>(v, v));   // 7 - lane: the other half of eight
  if (lanes >= 16) v = fmaxf(v, dpp_f32<0x140>(v, v));  // 15 - lane
  if (lanes >= 32) v = fmaxf(v, __shfl_xor(v, 16, 64));
  return v;
}
