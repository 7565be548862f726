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
// more, because n larger ones have been seen.  Entries are compared with it eight at a time through their maximum, which the
// softmax needs anyway, so that a row costs little more than its sums.  The bound comes from the eights' maxima at first (the n
// largest of 64 are n entries), and from the list whenever that fills up.
#include "ops.h"

namespace {

constexpr int MAX_TOP = MODSE_LOGPROBS_MAX_TOP;
constexpr int LIST = 192;       // candidates of a wave: LIST_FULL, and 64 more that one step can add
constexpr int LIST_FULL = 128;  // at which the list is cut back to the n largest
constexpr int TILE = 2048;      // entries that a block takes in one step: eight per thread
constexpr int AHEAD = 4;        // tiles that are loaded together
constexpr float LOG2E = 1.44269504088896340736f;
constexpr float LOWEST = -3.402823466e38f;
constexpr float FAR = -1e30f;   // differences of logits below it are held at it: e^FAR is 0, and 0 * FAR is no NaN

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

__device__ __forceinline__ void wave_lds_order() {  // LDS writes of this wave's lanes are there for its other lanes
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A bound K so that exactly n of the wave's keys (R per lane, distinct but for 0 = none, more than n in all) are K or more: its
// bits are set from the highest as long as n keys stay.
template <int R>
__device__ __forceinline__ uint64_t nth_key(const uint64_t (&key)[R], int n) {
  uint32_t p = 0;
  int c = 0;
#pragma unroll 1
  for (uint32_t bit = 0x80000000u; bit; bit >>= 1) {
    const uint32_t t = p | bit;
    int m = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) m += __popcll(__ballot((uint32_t)(key[r] >> 32) >= t));
    if (m >= n) {
      p = t;
      c = m;
      if (m == n) break;
    }
  }
  if (c == n) return (uint64_t)p << 32;
  // several entries of the n-th value: those of the lowest indices
  int above = 0;
#pragma unroll
  for (int r = 0; r < R; ++r) above += __popcll(__ballot((uint32_t)(key[r] >> 32) > p));
  uint32_t q = 0;
#pragma unroll 1
  for (uint32_t bit = 0x80000000u; bit; bit >>= 1) {
    const uint32_t t = q | bit;
    int m = above;
#pragma unroll
    for (int r = 0; r < R; ++r) m += __popcll(__ballot((uint32_t)(key[r] >> 32) == p && (uint32_t)key[r] >= t));
    if (m >= n) q = t;
  }
  return (uint64_t)p << 32 | q;
}

// The candidates of one wave.  All members are the same in every lane.
struct Candidates {
  uint64_t* list;
  int n, count;
  uint64_t bound;  // n entries of at least this key have been seen, and an entry that is not above it is out
  float bound_value;
  __device__ __forceinline__ void start(uint64_t* at, int top) {
    list = at;
    n = top;
    count = 0;
    bound = (uint64_t)ordered(-__builtin_inff()) << 32 | 0xffffffffu;  // masked entries are never in
    bound_value = -__builtin_inff();
  }
  __device__ __forceinline__ void raise(uint64_t k) {
    bound = k;
    bound_value = key_value(k);
  }
  __device__ __forceinline__ void cut() {  // to the n largest (count > n)
    constexpr int R = LIST / 64;
    const int lane = threadIdx.x & 63;
    wave_lds_order();
    uint64_t k[R];
#pragma unroll
    for (int r = 0; r < R; ++r) k[r] = r * 64 + lane < count ? list[r * 64 + lane] : 0;
    const uint64_t least = nth_key(k, n);
    wave_lds_order();
    count = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const uint64_t in = __ballot(k[r] >= least);
      if (k[r] >= least) list[count + __builtin_amdgcn_mbcnt_hi((uint32_t)(in >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)in, 0))] = k[r];
      count += __popcll(in);
    }
    raise(least);
  }
  // eight entries of this lane from index `at` on, their maximum
  __device__ __forceinline__ void take(const float (&v)[8], float most, uint32_t at) {
    const uint64_t lanes = __ballot(most > bound_value);
    if (lanes == 0) return;
    if (__popcll(lanes) > n) {
      // more lanes than entries that are wanted: the n largest of their maxima bound the rest
      // (the maximum is at one of eight places, and a bound has to be at the last of them)
      const uint64_t k[1] = {most > bound_value ? key_of(most, at + 7) : 0};
      const uint64_t least = nth_key(k, n);
      // (what is as large as the bound is to stay in)
      if (least - 1 > bound) raise(least - 1);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint64_t k = key_of(v[j], at + j);
      const bool mine = v[j] == v[j] && k > bound;
      const uint64_t in = __ballot(mine);
      if (in) {
        if (mine) list[count + __builtin_amdgcn_mbcnt_hi((uint32_t)(in >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)in, 0))] = k;
        count += __popcll(in);
        if (count > LIST_FULL) cut();
      }
    }
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

template <typename T, bool TOP, bool ENTROPY, bool SPLIT>
__global__ __launch_bounds__(256) void logprobs_fwd_kernel(LogprobsFwdArgs a, int splits, int segment) {
  __shared__ uint64_t s_list[TOP ? 4 * LIST : 1];
  __shared__ float s_sums[4][3];
  __shared__ int s_count[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = SPLIT ? blockIdx.x / splits : blockIdx.x;
  const int split = SPLIT ? blockIdx.x % splits : 0;
  const int begin = split * segment, end = SPLIT ? min(a.vocab, begin + segment) : a.vocab;
  const T* const x = static_cast<const T*>(a.logits) + row * a.ld;
  int target = -1;
  float target_logit = 0.f;
  if (!SPLIT && a.targets) {
    target = a.targets[row];
    if (target >= 0 && target < a.vocab) target_logit = (float)x[target];
  }
  Candidates top;
  if constexpr (TOP) top.start(s_list + wave * LIST, a.top);
  Sums t = {LOWEST, 0.f, 0.f};
  const int mine = threadIdx.x * 8;
#pragma unroll 1
  for (int base = begin; base < end; base += AHEAD * TILE) {
    Raw8<T> raw[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int col = base + u * TILE + mine;
      load_some(raw[u], x + col, end - col, -__builtin_inff());
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      float v[8], most = -__builtin_inff();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[j] = raw[u][j];
        most = fmaxf(most, v[j]);
      }
      t = rescaled(t, fmaxf(t.m, most));
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float z = v[j] - t.m;  // (NaN and +inf go on into S)
        const float e = __builtin_amdgcn_exp2f(z * LOG2E);
        t.S += e;
        if constexpr (ENTROPY) t.W += e * fmaxf(z, FAR);
      }
      if constexpr (TOP) top.take(v, most, base + u * TILE + mine);
    }
  }
  t = rescaled(t, wave_max(t.m));
  t.S = wave_sum(t.S);
  t.W = wave_sum(t.W);
  if (lane == 0) {
    s_sums[wave][0] = t.m;
    s_sums[wave][1] = t.S;
    s_sums[wave][2] = t.W;
  }
  if constexpr (TOP) {
    if (top.count > a.top) top.cut();
    if (lane == 0) s_count[wave] = top.count;
  }
  __syncthreads();
  float m = LOWEST;
#pragma unroll
  for (int w = 0; w < 4; ++w) m = fmaxf(m, s_sums[w][0]);
  Sums all = {m, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const Sums o = rescaled({s_sums[w][0], s_sums[w][1], s_sums[w][2]}, m);
    all.S += o.S;
    all.W += o.W;
  }
  float log_z = 0.f;
  if constexpr (SPLIT) {
    if (threadIdx.x == 0) a.part[blockIdx.x] = f32x4{all.m, all.S, all.W, 0.f};
  } else {
    log_z = row_outputs(a, row, all, target_logit, target, threadIdx.x == 0);
  }
  if constexpr (TOP) {
    // a candidate's rank is the number of larger ones
    const int total = s_count[0] + s_count[1] + s_count[2] + s_count[3];
    int rank = threadIdx.x;  // (of a thread without a candidate: the first place that stays empty, and on)
    uint64_t k = 0;
    if (lane < s_count[wave]) {
      k = s_list[wave * LIST + lane];
      rank = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w)
        for (int i = 0; i < s_count[w]; ++i) rank += s_list[w * LIST + i] > k;
    } else {
      int before = 0;  // threads without a candidate in front of this one
#pragma unroll
      for (int w = 0; w < 4; ++w)
        if (w < wave) before += 64 - s_count[w];
      rank = total + before + lane - s_count[wave];
    }
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

// Joins the segments of a row: one wave per row, one lane per segment.  The segments' lists are sorted, so the largest key left
// is one of their heads; of equal values the lowest segment has the lower index.
__global__ __launch_bounds__(64) void logprobs_join_kernel(LogprobsFwdArgs a, int splits, int bf16) {
  extern __shared__ uint64_t s_keys[];
  const int lane = threadIdx.x;
  const int64_t row = blockIdx.x;
  int target = -1;
  float target_logit = 0.f;
  if (a.targets) {
    target = a.targets[row];
    if (target >= 0 && target < a.vocab) {
      const int64_t i = row * a.ld + target;
      target_logit = bf16 ? (float)static_cast<const bf16_t*>(a.logits)[i] : static_cast<const float*>(a.logits)[i];
    }
  }
  const int n = splits * a.top;
  for (int i = lane; i < n; i += 64) s_keys[i] = a.keys[row * n + i];
  Sums t = {LOWEST, 0.f, 0.f};
  if (lane < splits) {
    const f32x4 p = a.part[row * splits + lane];
    t = {p[0], p[1], p[2]};
  }
  t = rescaled(t, wave_max(t.m));
  t.S = wave_sum(t.S);
  t.W = wave_sum(t.W);
  const float log_z = row_outputs(a, row, t, target_logit, target, lane == 0);
  if (a.top == 0) return;
  __syncthreads();
  int next = 0;
  uint64_t head = lane < splits ? s_keys[lane * a.top] : 0;
  uint64_t won = 0;  // of place `lane`
#pragma unroll 1
  for (int i = 0; i < a.top; ++i) {
    const uint32_t o = (uint32_t)(head >> 32);
    const float v = head ? unordered(o) : -__builtin_inff();
    const float best = wave_max(v);
    const uint64_t at = __ballot(head != 0 && v == best);
    if (at == 0) break;
    const int from = __builtin_ctzll(at);
    const uint64_t k = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)o, from) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)head, from);
    if (lane == i) won = k;
    if (lane == from) {
      ++next;
      head = next < a.top ? s_keys[lane * a.top + next] : 0;
    }
  }
  if (lane < a.top) {
    a.top_idx[row * a.top + lane] = won ? key_index(won) : -1;
    a.top_logp[row * a.top + lane] = won ? (key_value(won) - t.m) - log_z : -__builtin_inff();
  }
}

// d_logits = w (1[target] - p) - dE p (log p + H)
template <typename T, bool ENTROPY>
__global__ __launch_bounds__(256) void logprobs_bwd_kernel(LogprobsBwdArgs a, int segments) {
  const int64_t row = blockIdx.x / segments;
  const int col0 = blockIdx.x % segments * (TILE * AHEAD) + threadIdx.x * 8;
  const T* const x = static_cast<const T*>(a.logits) + row * a.ld;
  T* const dx = static_cast<T*>(a.d_logits) + row * a.ldd;
  const int target = a.targets ? a.targets[row] : -1;
  const float m = a.stats[2 * row], log_z = a.stats[2 * row + 1];
  const bool empty = log_z == __builtin_inff();
  const float w = target < 0 || empty ? 0.f : target >= a.vocab ? __builtin_nanf("") : a.d_logp[row];
  const float dE = ENTROPY && !empty ? a.d_entropy[row] : 0.f, H = ENTROPY ? a.entropy[row] : 0.f;
  const bool zero = w == 0.f && dE == 0.f;
  Raw8<T> raw[AHEAD];
  if (!zero) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int col = col0 + u * TILE;
      load_some(raw[u], x + col, a.vocab - col, 0.f);
    }
  }
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) {
    const int col = col0 + u * TILE;
    Raw8<T> out;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float g = 0.f;
      if (!zero) {
        const float z = (raw[u][j] - m) - log_z;
        const float p = __builtin_amdgcn_exp2f(z * LOG2E);
        g = -w;
        if constexpr (ENTROPY) g -= dE * (fmaxf(z, FAR) + H);
        g *= p;
        if (col + j == target) g += w;
      }
      out.set(j, g);
    }
    store_some(out, dx + col, a.vocab - col);
  }
}

template <typename T, bool TOP, bool ENTROPY>
hipError_t fwd(const LogprobsFwdArgs& a, int splits, hipStream_t s) {
  if (splits == 1) {
    hipLaunchKernelGGL((logprobs_fwd_kernel<T, TOP, ENTROPY, false>), dim3((unsigned)a.T), dim3(256), 0, s, a, 1, 0);
    return hipGetLastError();
  }
  const int segment = ((a.vocab + splits - 1) / splits + 7) / 8 * 8;
  hipLaunchKernelGGL((logprobs_fwd_kernel<T, TOP, ENTROPY, true>), dim3((unsigned)(a.T * splits)), dim3(256), 0, s, a, splits, segment);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(logprobs_join_kernel, dim3((unsigned)a.T), dim3(64), (size_t)splits * a.top * 8, s, a, splits, sizeof(T) == 2);
  return hipGetLastError();
}
template <typename T>
hipError_t fwd_any(const LogprobsFwdArgs& a, int splits, hipStream_t s) {
  if (a.top) return a.entropy ? fwd<T, true, true>(a, splits, s) : fwd<T, true, false>(a, splits, s);
  return a.entropy ? fwd<T, false, true>(a, splits, s) : fwd<T, false, false>(a, splits, s);
}
template <typename T>
hipError_t bwd(const LogprobsBwdArgs& a, hipStream_t s) {
  const int segments = (a.vocab + TILE * AHEAD - 1) / (TILE * AHEAD);
  const dim3 grid((unsigned)(a.T * segments));
  if (a.d_entropy) hipLaunchKernelGGL((logprobs_bwd_kernel<T, true>), grid, dim3(256), 0, s, a, segments);
  else hipLaunchKernelGGL((logprobs_bwd_kernel<T, false>), grid, dim3(256), 0, s, a, segments);
  return hipGetLastError();
}
}  // namespace

// Blocks that share a row: enough for four on every CU, each with a tile at least.
int logprobs_splits(int64_t T, int32_t vocab) {
  const int64_t want = 1024 / (T > 0 ? T : 1), most = (vocab + TILE - 1) / TILE;
  const int64_t n = want < most ? want : most;
  return (int)(n < 1 ? 1 : n > 64 ? 64 : n);
}
hipError_t launch_logprobs_fwd(modse_dtype dt, const LogprobsFwdArgs& a, int splits, hipStream_t s) {
  return dt == MODSE_F32 ? fwd_any<float>(a, splits, s) : fwd_any<bf16_t>(a, splits, s);
}
hipError_t launch_logprobs_bwd(modse_dtype dt, const LogprobsBwdArgs& a, hipStream_t s) {
  return dt == MODSE_F32 ? bwd<float>(a, s) : bwd<bf16_t>(a, s);
}
