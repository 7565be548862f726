// Log probabilities of given tokens, entropy and the most probable entries of softmax over rows of logits, and the gradient of
// the logits.
//
// Forward: one pass over a row.  Every thread keeps the maximum m of the entries it has seen, S = sum e^(x - m) and W = sum
// e^(x - m) (x - m); pairs (m, S, W) are joined by rescaling to the larger maximum, over the wave, the block and, where there
// are few rows and each is shared by several blocks, by a second launch.  Then log Z = log S (relative to m), log p = x - m -
// log Z and the entropy is log Z - W / S.
//
// Top entries: the order is by falling value, then by rising index, which is the order of the 64-bit keys (ordered bits of the
// value, ~index).  A wave keeps a list of candidates in LDS and a bound below which an entry cannot be among the n largest any
// more, because n larger ones have been seen.  Entries are compared with it 32 of a lane at a time through their maximum, which
// the softmax needs anyway, so that a row costs little more than its sums.  The bound comes from the lanes' maxima at first (the n
// largest of 64 are n entries), and from the list whenever that fills up.
//
// Large calls are bound by memory: both kernels read the logits once, in vectors of sixteen bytes, 128 bytes of a thread in flight.
// Small ones are bound by the launches.  us of the GPU and a call: one row or 256 of 32000 without top entries, one launch, 4.0 to 4.7 and 5.5; one
// row of 131072 with the 5 most probable, two launches, 8.6 and 9.1; 64 of 32000 with 20, two launches, 13 one by one and 12.3 where the
// second runs into the next call's first.
#include "ops.h"

namespace {

constexpr int MAX_TOP = MODSE_LOGPROBS_MAX_TOP;
constexpr int LIST = 192;       // candidates of a wave: LIST_FULL, and 64 more that one step can add
constexpr int LIST_FULL = 128;  // at which the list is cut back to the n largest
constexpr int LOOK = 32;        // entries of a thread that are loaded, and looked through, together, in vectors of sixteen bytes
constexpr int GROUP = LOOK * 256;  // entries that a block takes at a time
constexpr float LOG2E = 1.44269504088896340736f;
constexpr float LOWEST = -3.402823466e38f;
constexpr float FAR = -1e30f;   // differences of logits below it are held at it: e^FAR is 0, and 0 * FAR is no NaN
constexpr float NIL = -200.f;   // where they are multiplied by a gradient first: e^NIL is 0, and NIL times any loss scale is finite

// keys of the order above; none is 0
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.f);  // (the two zeros are one value)
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o) {
  return __builtin_bit_cast(float, o ^ ((uint32_t)(~(int32_t)o >> 31) | 0x80000000u));
}
__device__ __forceinline__ uint64_t key_of(float v, uint32_t index) { return (uint64_t)ordered(v) << 32 | (uint32_t)~index; }
__device__ __forceinline__ float key_value(uint64_t k) { return unordered((uint32_t)(k >> 32)); }
__device__ __forceinline__ int key_index(uint64_t k) { return (int)~(uint32_t)k; }

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#define STEP(CTRL, ROWS) { const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, ROWS, 0xf, false); v = max(v, o); }
  STEP(0x111, 0xf) STEP(0x112, 0xf) STEP(0x114, 0xf) STEP(0x118, 0xf) STEP(0x142, 0xa) STEP(0x143, 0xc)
#undef STEP
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// A bound K so that n to n + slack of the wave's keys are K or more (R per lane, distinct but for 0 = none, more than n in all):
// bisection between the smallest and the largest, first over the values, and where several entries have the n-th value over
// their indices.  Distinct values come apart in 6 to 8 of its steps.
template <int R>
__device__ __forceinline__ uint64_t nth_key(const uint64_t (&key)[R], int n, int slack) {
  uint32_t top = 0, least = 0;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const uint32_t h = (uint32_t)(key[r] >> 32);
    top = max(top, h);
    least = max(least, h ? ~h : 0);
  }
  uint32_t hi = wave_max_u32(top), lo = ~wave_max_u32(least);  // at least n keys are lo or more
#pragma unroll 1
  while (lo < hi) {
    const uint32_t t = lo + (hi - lo + 1) / 2;
    int m = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) m += __popcll(__ballot((uint32_t)(key[r] >> 32) >= t));
    if (m >= n) {
      lo = t;
      if (m <= n + slack) return (uint64_t)t << 32;
    } else {
      hi = t - 1;
    }
  }
  int above = 0, with = 0;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    above += __popcll(__ballot((uint32_t)(key[r] >> 32) > lo));
    with += __popcll(__ballot((uint32_t)(key[r] >> 32) >= lo));
  }
  if (with <= n + slack) return (uint64_t)lo << 32;
  uint32_t last = 0, first = 0;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool tied = (uint32_t)(key[r] >> 32) == lo;
    last = max(last, tied ? (uint32_t)key[r] : 0);
    first = max(first, tied ? ~(uint32_t)key[r] : 0);
  }
  uint32_t q_hi = wave_max_u32(last), q = ~wave_max_u32(first);
#pragma unroll 1
  while (q < q_hi) {
    const uint32_t t = q + (q_hi - q + 1) / 2;
    int m = above;
#pragma unroll
    for (int r = 0; r < R; ++r) m += __popcll(__ballot((uint32_t)(key[r] >> 32) == lo && (uint32_t)key[r] >= t));
    if (m >= n) {
      q = t;
      if (m <= n + slack) break;
    } else {
      q_hi = t - 1;
    }
  }
  return (uint64_t)lo << 32 | q;
}

// The candidates of one wave.  All members are the same in every lane.
struct Candidates {
  uint64_t* list;
  int n, count;
  uint64_t bound;  // n entries above this key have been seen, and an entry that is not above it is out
  float bound_value;
  __device__ __forceinline__ void start(uint64_t* at, int top) {
    list = at;
    n = top;
    count = 0;
    bound = (uint64_t)ordered(-__builtin_inff()) << 32 | 0xffffffffu;  // masked entries are never in
    bound_value = -__builtin_inff();
  }
  __device__ __forceinline__ void raise(uint64_t least) {  // n entries of at least this key have been seen
    bound = least - 1;
    bound_value = key_value(bound);
  }
  __device__ __forceinline__ void add(uint64_t k, bool mine, uint64_t in) {
    if (mine) list[count + __builtin_amdgcn_mbcnt_hi((uint32_t)(in >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)in, 0))] = k;
    count += __popcll(in);
  }
  __device__ __forceinline__ void cut() {  // to the n largest, or a few more, 64 at most (count > 64)
    constexpr int R = LIST / 64;
    const int lane = threadIdx.x & 63;
    wave_lds_order();
    uint64_t k[R];
#pragma unroll
    for (int r = 0; r < R; ++r) k[r] = r * 64 + lane < count ? list[r * 64 + lane] : 0;
    const uint64_t least = nth_key(k, n, 64 - n);
    wave_lds_order();
    count = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) add(k[r], k[r] >= least, __ballot(k[r] >= least));
    raise(least);
  }
  // LOOK entries of this lane in vectors of N, their maximum, the index of the first; the vectors are 256 N apart
  template <int N>
  __device__ __forceinline__ void take(const float (&v)[LOOK], float most, uint32_t at) {
    const uint64_t lanes = __ballot(most > bound_value);  // (entries that come later lose ties)
    if (lanes == 0) return;
    if (__popcll(lanes) > n) {
      // more lanes than entries that are wanted: the n largest of their maxima bound the rest.  (A maximum can be at the last of
      // a lane's places.)
      const uint64_t k[1] = {most > bound_value ? key_of(most, at + (LOOK / N - 1) * 256 * N + N - 1) : 0};
      const uint64_t least = nth_key(k, n, n / 2 + 2);
      if (least - 1 > bound) raise(least);
    }
    uint32_t left = 0;  // which of this lane's are not below the bound
#pragma unroll
    for (int i = 0; i < LOOK; ++i) left |= v[i] >= bound_value ? 1u << i : 0;
    // (a loop that picks the value, not a body for each of the 32: as code it would be larger than what it runs on)
#pragma unroll 1
    while (__ballot(left != 0)) {
      const int i = __builtin_ffs((int)left) - 1;
      float x[LOOK];
#pragma unroll
      for (int k = 0; k < LOOK; ++k) x[k] = v[k];
#pragma unroll
      for (int b = 0; b < 5; ++b)
#pragma unroll
        for (int k = 0; k < LOOK >> (b + 1); ++k) x[k] = i >> b & 1 ? x[2 * k + 1] : x[2 * k];
      const uint64_t k = key_of(x[0], at + i / N * (256 * N) + i % N);
      const bool mine = left != 0 && k > bound;
      left &= left - 1;
      add(k, mine, __ballot(mine));
      if (count > LIST_FULL) cut();
    }
  }
  // the n largest among at most 64, and zeros behind them
  __device__ __forceinline__ void finish() {
    if (count > 64) cut();
    const int lane = threadIdx.x & 63;
    if (lane >= count) list[lane] = 0;
  }
};

struct Sums {
  float m, S, W;
};
// to a maximum that is not below m
__device__ __forceinline__ Sums rescaled(Sums a, float m) {
  const float z = fmaxf(a.m - m, FAR);
  const float f = __builtin_amdgcn_exp2f(z * LOG2E);
  return {m, a.S * f, f * (a.W + a.S * z)};
}

// the sums of a wave, in all of its lanes
__device__ __forceinline__ Sums wave_joined(Sums t) {
  t = rescaled(t, wave_max(t.m));
  t.S = wave_sum(t.S);
  t.W = wave_sum(t.W);
  return t;
}
// those of a block's four waves
__device__ __forceinline__ Sums waves_joined(const float (&s)[4][3]) {
  float m = LOWEST;
#pragma unroll
  for (int w = 0; w < 4; ++w) m = fmaxf(m, s[w][0]);
  Sums all = {m, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const Sums o = rescaled({s[w][0], s[w][1], s[w][2]}, m);
    all.S += o.S;
    all.W += o.W;
  }
  return all;
}

// what a row's sums say of it; returns log Z (an entry's log probability is x - m - log Z)
__device__ __forceinline__ float row_outputs(const LogprobsFwdArgs& a, int64_t row, Sums t, float target_logit, int target, bool write) {
  const float none = -__builtin_inff();
  const bool empty = t.S == 0.f;
  const float log_z = empty ? __builtin_inff() : logf(t.S), m = empty ? 0.f : t.m;
  if (write) {
    if (a.logp) {
      float v = target < 0 ? 0.f : empty ? none : (target_logit - m) - log_z;
      a.logp[row] = target >= a.vocab ? __builtin_nanf("") : v;
    }
    if (a.entropy) a.entropy[row] = empty ? 0.f : log_z - t.W / t.S;
    if (a.stats) {
      a.stats[2 * row] = m;
      a.stats[2 * row + 1] = log_z;  // (+inf: no distribution)
    }
  }
  return log_z;
}

// 16384 rows of 32000 in bf16 take 157 us, 6.7 TB/s of reads; 2047 of 50257 in float32 with the 5 most probable 73, 5.6 TB/s; one row
// of 131072 with them 5.5, and 64 of 32000 with the 20 most probable 8.8.
//
// APART: a row of at most FEW_GROUPS groups in one block, four waves a group, that joins their sums as logprobs_join_kernel does: the same
// bits as with the top entries, for which such a row is shared.  us from the host / of the GPU alone, one row of 32000 and 256: 5.5 / 4.0 and 5.4 / 4.7;
// four waves that take one group after the other 5.7 / 5.6 and 6.1 / 6.1, and in one sum, with other bits, 5.4 / 4.7 and 5.4 / 5.3; two
// launches 7.5 / 4.3 and 7.3 / 6.2.
constexpr int FEW_GROUPS = 4;
template <typename T, bool TOP, bool ENTROPY, bool SPLIT, bool STREAM, bool APART = false>
__global__ __launch_bounds__(APART ? 256 * FEW_GROUPS : 256) void logprobs_fwd_kernel(LogprobsFwdArgs a, int splits, int segment) {
  static_assert(!APART || (!TOP && !SPLIT));
  __shared__ uint64_t s_list[TOP ? 4 * LIST : 1];
  __shared__ float s_sums[APART ? FEW_GROUPS : 1][4][3];
  __shared__ int s_count[4];
  const int thread = APART ? threadIdx.x & 255 : threadIdx.x, lane = thread & 63, wave = thread >> 6;
  const int64_t row = SPLIT ? blockIdx.x / splits : blockIdx.x;
  const int split = SPLIT ? blockIdx.x % splits : APART ? threadIdx.x >> 8 : 0;
  const int begin = split * segment, end = SPLIT || APART ? min(a.vocab, begin + segment) : a.vocab;
  const T* const x = static_cast<const T*>(a.logits) + row * a.ld;
  int target = -1;
  float target_logit = 0.f;
  if (a.targets) {
    target = a.targets[row];
    if (target >= (APART ? 0 : begin) && target < (APART ? a.vocab : end)) target_logit = (float)x[target];
  }
  Candidates top;
  if constexpr (TOP) top.start(s_list + wave * LIST, a.top);
  Sums t = {LOWEST, 0.f, 0.f};
  constexpr int N = Vec<T>::N;
  const int mine = thread * N;
#pragma unroll 1
  for (int base = begin; base < end; base += GROUP) {
    Vec<T> raw[LOOK / N];
#pragma unroll
    for (int u = 0; u < LOOK / N; ++u) {
      const int col = base + u * 256 * N + mine;
      raw[u].template load<STREAM>(x + col, end - col, -__builtin_inff());
    }
    float v[LOOK], most = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < LOOK; ++i) {
      v[i] = raw[i / N][i % N];
      most = fmaxf(most, v[i]);
    }
    t = rescaled(t, fmaxf(t.m, most));
#pragma unroll
    for (int u = 0; u < LOOK / N; ++u) {
      if (base + u * 256 * N < end) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float z = v[u * N + j] - t.m;  // (NaN and +inf go on into S)
          const float e = __builtin_amdgcn_exp2f(z * LOG2E);
          t.S += e;
          if constexpr (ENTROPY) t.W += e * fmaxf(z, FAR);
        }
      }
    }
    if constexpr (TOP) top.template take<N>(v, most, base + mine);
  }
  t = wave_joined(t);
  if (lane == 0) {
    float* const to = s_sums[APART ? split : 0][wave];
    to[0] = t.m;
    to[1] = t.S;
    to[2] = t.W;
  }
  if constexpr (TOP) {
    top.finish();
    if (lane == 0) s_count[wave] = top.count;
  }
  __syncthreads();
  Sums all;
  if constexpr (APART) {
    all = {LOWEST, 0.f, 0.f};
    if (lane * segment < a.vocab) all = waves_joined(s_sums[lane]);
    all = wave_joined(all);
  } else {
    all = waves_joined(s_sums[0]);
  }
  float log_z = 0.f;
  if constexpr (SPLIT) {
    if (threadIdx.x == 0) a.part[blockIdx.x] = f32x4{all.m, all.S, all.W, target_logit};
  } else {
    log_z = row_outputs(a, row, all, target_logit, target, threadIdx.x == 0);
  }
  if constexpr (TOP) {
    // a candidate's rank is the number of larger ones
    int total = 0, most = 0, before = 0;  // before: threads without a candidate in front of this wave
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int c = s_count[w];
      total += c;
      most = max(most, c);
      before += w < wave ? 64 - c : 0;
    }
    const uint64_t k = s_list[wave * LIST + lane];
    int rank = 0;
#pragma unroll 2
    for (int i = 0; i < most; ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) rank += s_list[w * LIST + i] > k;
    if (k == 0) rank = total + before + lane - s_count[wave];  // the places that stay empty
    if (rank < a.top) {
      if constexpr (SPLIT) {
        a.keys[(int64_t)blockIdx.x * a.top + rank] = k;
      } else {
        a.top_idx[row * a.top + rank] = k ? key_index(k) : -1;
        a.top_logp[row * a.top + rank] = k ? (key_value(k) - all.m) - log_z : -__builtin_inff();
      }
    }
  }
}

// Joins the segments of a row: one wave per row, one lane per segment for the sums; the segments' entries are ranked as above.
// 3.2 us for one row of 16 segments, 4.2 for 64 rows of 4: a launch and three rounds to memory, nothing of which grows with a row.
constexpr int JOIN_KEYS = 8;  // per lane
__global__ __launch_bounds__(64) void logprobs_join_kernel(LogprobsFwdArgs a, int splits, int segment) {
  __shared__ uint64_t s_list[64];
  const int lane = threadIdx.x;
  const int64_t row = blockIdx.x;
  const int n = splits * a.top;
  uint64_t key[JOIN_KEYS];
#pragma unroll
  for (int r = 0; r < JOIN_KEYS; ++r) key[r] = r * 64 + lane < n ? a.keys[row * n + r * 64 + lane] : 0;
  const int target = a.targets ? a.targets[row] : -1;
  float target_logit = 0.f;
  Sums t = {LOWEST, 0.f, 0.f};
  if (lane < splits) {
    const f32x4 p = a.part[row * splits + lane];
    t = {p[0], p[1], p[2]};
    target_logit = p[3];
  }
  target_logit = lane_f32(target_logit, target >= 0 && target < a.vocab ? target / segment : 0);
  t = wave_joined(t);
  const float log_z = row_outputs(a, row, t, target_logit, target, lane == 0);
  if (a.top == 0) return;
  int count = 0;
#pragma unroll
  for (int r = 0; r < JOIN_KEYS; ++r) count += __popcll(__ballot(key[r] != 0));
  const uint64_t least = count > 64 ? nth_key(key, a.top, 64 - a.top) : 1;
  Candidates all;
  all.start(s_list, a.top);
#pragma unroll
  for (int r = 0; r < JOIN_KEYS; ++r) all.add(key[r], key[r] >= least, __ballot(key[r] >= least));
  wave_lds_order();
  const uint64_t k = lane < all.count ? s_list[lane] : 0;
  int rank = 0;
#pragma unroll 4
  for (int i = 0; i < all.count; ++i) rank += s_list[i] > k;
  if (k == 0) rank = lane;
  if (rank < a.top) {
    a.top_idx[row * a.top + rank] = k ? key_index(k) : -1;
    a.top_logp[row * a.top + rank] = k ? (key_value(k) - t.m) - log_z : -__builtin_inff();
  }
}

// d_logits = w (1[target] - p) - dE p (log p + H), from the row's m and log Z: a read and a write of the matrix.  16384 rows of 32000 in
// bf16 take 356 us, 5.9 TB/s of the 6.2 that a sum of two large tensors into a third reaches.  A row without a target and without a
// gradient of its entropy is not read.
template <typename T, bool ENTROPY, bool STREAM>
__global__ __launch_bounds__(256) void logprobs_bwd_kernel(LogprobsBwdArgs a, int segments) {
  const int64_t row = blockIdx.x / segments;
  constexpr int N = Vec<T>::N;
  const int col0 = blockIdx.x % segments * GROUP + threadIdx.x * N;
  const T* const x = static_cast<const T*>(a.logits) + row * a.ld;
  T* const dx = static_cast<T*>(a.d_logits) + row * a.ldd;
  const int target = a.targets ? a.targets[row] : -1;
  const float m = a.stats[2 * row], log_z = a.stats[2 * row + 1];
  const bool empty = log_z == __builtin_inff();
  const float w = target < 0 || empty ? 0.f : target >= a.vocab ? __builtin_nanf("") : a.d_logp[row];
  const float dE = ENTROPY && !empty ? a.d_entropy[row] : 0.f, H = ENTROPY ? a.entropy[row] : 0.f;
  const bool zero = w == 0.f && dE == 0.f;
  Vec<T> raw[LOOK / N];
  if (!zero) {
#pragma unroll
    for (int u = 0; u < LOOK / N; ++u) {
      const int col = col0 + u * 256 * N;
      raw[u].template load<STREAM>(x + col, a.vocab - col, 0.f);
    }
  }
#pragma unroll
  for (int u = 0; u < LOOK / N; ++u) {
    const int col = col0 + u * 256 * N;
    Vec<T> out;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      float g = 0.f;
      if (!zero) {
        const float z = (raw[u][j] - m) - log_z;
        const float p = __builtin_amdgcn_exp2f(z * LOG2E);
        g = -w;
        if constexpr (ENTROPY) g -= dE * (fmaxf(z, NIL) + H);
        g *= p;
        if (col + j == target) g += w;
      }
      out.set(j, g);
    }
    out.template store<STREAM>(dx + col, a.vocab - col);
  }
}

// Logits that the caches do not hold are read, and their gradient stored, with the non-temporal hint.  us without / with it, forward and
// backward: 16384 x 32000 bf16 (1.05 GB) 176 + 384 / 157 + 358, one behind the other 582 / 515; 2047 x 50257 float32 (411 MB) 241 / 222; 4096
// x 32000 (262 MB), where the backward pass finds part of the logits in the cache, 156 / 132 but 127 with hinted stores alone; 1024 x 32000
// 40.1 / 38.4, and a product that reads the gradient next loses what the stores gain: 305.0 / 307.0.
constexpr int64_t STREAM_BYTES = (int64_t)384 << 20;

template <typename T, bool TOP, bool ENTROPY>
hipError_t fwd(const LogprobsFwdArgs& a, LogprobsSplit split, hipStream_t s) {
  const auto [splits, segment] = split;
  if (splits == 1) {
    const dim3 grid((unsigned)a.T);
    const bool apart = !TOP && logprobs_split(a.T, a.vocab, 1).splits > 1;
    if (apart)
      hipLaunchKernelGGL((logprobs_fwd_kernel<T, false, ENTROPY, false, false, true>), grid, dim3((a.vocab + GROUP - 1) / GROUP * 256), 0, s, a, 1, GROUP);
    else if (a.T * a.vocab * (int64_t)sizeof(T) >= STREAM_BYTES)
      hipLaunchKernelGGL((logprobs_fwd_kernel<T, TOP, ENTROPY, false, true>), grid, dim3(256), 0, s, a, 1, 0);
    else
      hipLaunchKernelGGL((logprobs_fwd_kernel<T, TOP, ENTROPY, false, false>), grid, dim3(256), 0, s, a, 1, 0);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((logprobs_fwd_kernel<T, TOP, ENTROPY, true, false>), dim3((unsigned)(a.T * splits)), dim3(256), 0, s, a, splits, segment);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(logprobs_join_kernel, dim3((unsigned)a.T), dim3(64), 0, s, a, splits, segment);
  return hipGetLastError();
}
template <typename T>
hipError_t fwd_any(const LogprobsFwdArgs& a, LogprobsSplit split, hipStream_t s) {
  if (a.top) return a.entropy ? fwd<T, true, true>(a, split, s) : fwd<T, true, false>(a, split, s);
  return a.entropy ? fwd<T, false, true>(a, split, s) : fwd<T, false, false>(a, split, s);
}
template <typename T, bool ENTROPY>
hipError_t bwd(const LogprobsBwdArgs& a, hipStream_t s) {
  const int segments = (a.vocab + GROUP - 1) / GROUP;
  const dim3 grid((unsigned)(a.T * segments));
  if (a.T * a.vocab * (int64_t)sizeof(T) >= STREAM_BYTES) hipLaunchKernelGGL((logprobs_bwd_kernel<T, ENTROPY, true>), grid, dim3(256), 0, s, a, segments);
  else hipLaunchKernelGGL((logprobs_bwd_kernel<T, ENTROPY, false>), grid, dim3(256), 0, s, a, segments);
  return hipGetLastError();
}
template <typename T>
hipError_t bwd_any(const LogprobsBwdArgs& a, hipStream_t s) {
  return a.d_entropy ? bwd<T, true>(a, s) : bwd<T, false>(a, s);
}
}  // namespace

// A row is shared by several blocks where there are few rows, each taking a whole number of the groups of tiles that are loaded
// together, and no more entries being left to join than a wave holds.  us a call, one block a row / one for every 8192 entries
// (bf16): 1 x 131072, top 5 28.6 / 7.9, without top 14.7 / 4.7; 64 x 32000, top 5 11.8 / 8.3; 256 x 32000 12.8 / 11.2, without top
// 5.7 / 6.9; 256 x 131072 34.9 / 24.9; 512 x 32000 15.5 / 16.2; 512 x 131072, without top 24.3 / 23.7; 700 x 131072 31.8 / 30.5, top 5
// 50.0 / 52.3.  Few groups are not worth the second launch (from the host / of the GPU alone): two with top 5, 1 x 16384 6.6 / 6.4 and 8.9 / 6.8,
// 256 x 16384 8.8 / 8.7 and 9.7 / 9.3; four without, see APART.  Finer cuts than a group: 64 x 32000 in 16 11.4, 1 x 131072 in 64 8.6.
LogprobsSplit logprobs_split(int64_t T, int32_t vocab, int32_t top) {
  const int groups = (vocab + GROUP - 1) / GROUP, most = top > 8 ? JOIN_KEYS * 64 / top : 64;
  if (T > 512 || (T > 256 && groups < 8) || groups <= (top ? 2 : FEW_GROUPS)) return {1, vocab};
  const int each = (groups + most - 1) / most;
  return {(groups + each - 1) / each, each * GROUP};
}
hipError_t launch_logprobs_fwd(modse_dtype dt, const LogprobsFwdArgs& a, LogprobsSplit split, hipStream_t s) {
  return dt == MODSE_F32 ? fwd_any<float>(a, split, s) : fwd_any<bf16_t>(a, split, s);
}
hipError_t launch_logprobs_bwd(modse_dtype dt, const LogprobsBwdArgs& a, hipStream_t s) {
  return dt == MODSE_F32 ? bwd_any<float>(a, s) : bwd_any<bf16_t>(a, s);
}
