// Dropout from a counter-based generator: y = residual + keep x / (1 - p), and its backward pass dX = keep dY / (1 - p).  The mask is
// never stored: both directions make it from the same counters.
//
// The generator is Philox-4x32 with seven rounds (J. Salmon, M. Moraes, R. Dror, D. Shaw: Parallel random numbers: as easy as 1, 2, 3,
// 2011; seven are the fewest that pass all of their tests): key = seed, counter = (index / 8, call, offset), and its four words are
// the 16 random bits of each of eight consecutive elements, the low half of word w that of element 2 w.  With 16 bits an element p is
// a multiple of 2^-16, and the kept ones are scaled by 1 / (1 - p) of that p.
//
// A thread takes the eight elements of one counter.  Large calls are bound by memory: 32768 rows of 2048, bf16, with a residual 61 us (6.6
// TB/s), backwards 38 (7.0, partly from the caches).  The generator is some 14 products of 32 bits and as many words of xor for 48 bytes
// read and written, and hides behind them.  Small calls are one launch, 2.5 us of the GPU.
#include "ops.h"

namespace {

__device__ __forceinline__ u32x4 philox7(u32x4 c, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 7; ++r) {
    const uint64_t p0 = (uint64_t)0xD2511F53u * c[0], p1 = (uint64_t)0xCD9E8D57u * c[2];
    c = u32x4{(uint32_t)(p1 >> 32) ^ c[1] ^ k0, (uint32_t)p1, (uint32_t)(p0 >> 32) ^ c[3] ^ k1, (uint32_t)p0};
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return c;
}

// Reads with the non-temporal hint from a size on that the caches do not hold (the last level has 256 MiB).  Without / with it, us,
// with the norm that reads y behind it: 16384 rows of 2048, bf16 (192 MiB read and written) 52 / 57, 32768 (384 MiB) 115 / 103,
// 32768 of 4096 240 / 220; backwards alone 32768 of 2048 (256 MiB) 38 / 44, of 4096 89 / 85.  (Hinted stores of y: 57 in place of 52, 125
// in place of 115.)
constexpr int64_t STREAM_BYTES = (int64_t)320 << 20;

template <typename T, bool RESIDUAL, bool STREAM>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a) {
  constexpr int N = Vec<T>::N, NV = 8 / N;
  const T* const x = static_cast<const T*>(a.x);
  const T* const res = static_cast<const T*>(a.residual);
  T* const y = static_cast<T*>(a.y);
  const uint64_t seed = a.rng[0], offset = a.rng[1];
  const int64_t blocks = (a.n + 7) >> 3;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < blocks; i += (int64_t)gridDim.x * 256) {
    const int64_t at = i * 8;
    const int64_t left = a.n - at;
    Vec<T> v[NV], r[NV];
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int n = (int)(left - q * N < N ? left - q * N : N);
      v[q].template load<STREAM>(x + at + q * N, n, 0.f);
      if constexpr (RESIDUAL) r[q].template load<STREAM>(res + at + q * N, n, 0.f);
    }
    const u32x4 w = philox7(u32x4{(uint32_t)i, a.call, (uint32_t)offset, (uint32_t)(offset >> 32)}, (uint32_t)seed, (uint32_t)(seed >> 32));
#pragma unroll
    for (int q = 0; q < NV; ++q) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int k = q * N + e;
        const uint32_t bits = k & 1 ? w[k >> 1] >> 16 : w[k >> 1] & 0xffffu;
        // (chosen, not multiplied: what is dropped may be an infinity)
        float o = bits >= a.limit ? v[q][e] * a.scale : 0.f;
        if constexpr (RESIDUAL) o += r[q][e];
        v[q].set(e, o);
      }
      const int n = (int)(left - q * N < N ? left - q * N : N);
      v[q].store(y + at + q * N, n);
    }
  }
}

template <typename T>
hipError_t run(const DropoutArgs& a, hipStream_t s) {
  const int64_t blocks = (a.n + 2047) / 2048;
  const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : 1 << 20));
  const bool stream = a.n * (int64_t)sizeof(T) * (a.residual ? 3 : 2) >= STREAM_BYTES;
  if (a.residual && stream) hipLaunchKernelGGL((dropout_kernel<T, true, true>), grid, dim3(256), 0, s, a);
  else if (a.residual) hipLaunchKernelGGL((dropout_kernel<T, true, false>), grid, dim3(256), 0, s, a);
  else if (stream) hipLaunchKernelGGL((dropout_kernel<T, false, true>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((dropout_kernel<T, false, false>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_dropout(modse_dtype dt, const DropoutArgs& a, hipStream_t s) {
  return dt == MODSE_F32 ? run<float>(a, s) : run<bf16_t>(a, s);
}
