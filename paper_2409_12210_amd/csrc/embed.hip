// Embedding lookup x_t = scale E[token_t], and its gradient dE_v = scale sum of dX_t over the tokens t that are v, in float32.
//
// Lookup: a wave takes up to 2048 (bf16) or 1024 (float32) columns of one row.  Bound by memory (32768 rows of 2048, bf16: 37 us, 7.2
// TB/s), or by the launch.  (Hinted stores take 15.6 us where 17.3 are for 16384 rows, but with the norm that reads them behind it 44
// in place of 40.)
//
// Gradient, three launches, every sum in an order that the tokens alone fix:
//   embed_sort_kernel  a block owns a range of the vocabulary and sorts the tokens of its range, stably: it reads all tokens (they
//                      are in the caches), counts those below its range, which is where its part of the sorted list begins, and
//                      those of each of its rows by wave, and in a second pass every wave puts its tokens where its counts say.
//                      No block waits for another.  Rows that do not occur become zeros here.
//   embed_sum_kernel   a block takes `chunk` consecutive places of the sorted list, whatever rows they belong to, so that frequent
//                      tokens do not hold up a launch.  Runs of one token that lie inside are done; the others leave partial sums.
//   embed_join_kernel  adds up the partial sums of runs that cross chunks, in order.
#include "ops.h"

namespace {

constexpr int LOOKUP_VECS = 4;  // vectors of sixteen bytes that a lane takes

template <typename T>
__global__ __launch_bounds__(256) void embed_lookup_kernel(EmbedFwdArgs a) {
  constexpr int N = Vec<T>::N, SEG = 64 * LOOKUP_VECS * N;
  const int lane = threadIdx.x & 63;
  const int segs = (a.d + SEG - 1) / SEG;
  const int64_t units = a.T * segs;
  for (int64_t u = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); u < units; u += (int64_t)gridDim.x * 4) {
    const int64_t t = u / segs;
    const int c0 = (int)(u - t * segs) * SEG + lane * N;
    const int32_t token = a.tokens[t];
    T* const out = static_cast<T*>(a.x) + t * a.d;
    Vec<T> v[LOOKUP_VECS];
    if (token >= 0 && token < a.vocab) {
      const T* const row = static_cast<const T*>(a.E) + (int64_t)token * a.d;
#pragma unroll
      for (int i = 0; i < LOOKUP_VECS; ++i)
        if (c0 + i * 64 * N < a.d) v[i].load(row + c0 + i * 64 * N, a.d - c0 - i * 64 * N, 0.f);
#pragma unroll
      for (int i = 0; i < LOOKUP_VECS; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) v[i].set(e, v[i][e] * a.scale);
    } else {
      const float fill = token < 0 ? 0.f : __builtin_nanf("");
#pragma unroll
      for (int i = 0; i < LOOKUP_VECS; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) v[i].set(e, fill);
    }
#pragma unroll
    for (int i = 0; i < LOOKUP_VECS; ++i)
      if (c0 + i * 64 * N < a.d) v[i].store(out + c0 + i * 64 * N, a.d - c0 - i * 64 * N);
  }
}

constexpr int SORT_WAVES = 16;

__global__ __launch_bounds__(SORT_WAVES * 64) void embed_sort_kernel(EmbedBwdArgs a, int rows_per_block) {
  __shared__ int32_t hist[SORT_WAVES][EMBED_MAX_ROWS];  // of a wave's tokens, by row; then where they go
  __shared__ int32_t total[EMBED_MAX_ROWS], below[SORT_WAVES], scan[SORT_WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t lo = blockIdx.x * rows_per_block, rows = min(rows_per_block, a.vocab - lo);
  for (int i = lane; i < rows; i += 64) hist[wave][i] = 0;
  wave_lds_order();

  // this wave's tokens: a stretch of whole groups of 64
  const int64_t groups = (a.T + 63) / 64, per = (groups + SORT_WAVES - 1) / SORT_WAVES;
  const int64_t g0 = wave * per, g1 = g0 + per < groups ? g0 + per : groups;
  auto token = [&](int64_t g) -> int32_t {
    const int64_t t = g * 64 + lane;
    return g < g1 && t < a.T ? a.tokens[t] : -1;
  };
  constexpr int AHEAD = 8;  // groups that are loaded together
  int32_t before = 0;
  for (int64_t g = g0; g < g1; g += AHEAD) {
    int32_t k[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) k[i] = token(g + i);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      before += k[i] >= 0 && k[i] < lo;
      if (k[i] >= lo && k[i] < lo + rows) atomicAdd(&hist[wave][k[i] - lo], 1);  // (a count: the order does not matter)
    }
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) before += __shfl_xor(before, o, 64);
  if (lane == 0) below[wave] = before;
  __syncthreads();

  // where each wave's tokens of each row begin
  const int r = tid;  // (as many threads as rows at the most)
  int32_t n = 0;
  if (r < rows)
    for (int w = 0; w < SORT_WAVES; ++w) n += hist[w][r];
  int32_t incl = n;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int32_t up = __shfl_up(incl, o, 64);
    if (lane >= o) incl += up;
  }
  if (lane == 63) scan[wave] = incl;
  __syncthreads();
  int32_t at = incl - n;
  for (int w = 0; w < SORT_WAVES; ++w) {
    at += below[w];
    if (w < wave) at += scan[w];
  }
  if (r < rows) {
    total[r] = n;
    if (lo + r == a.vocab - 1) *a.n_sorted = at + n;
    for (int w = 0; w < SORT_WAVES; ++w) {
      const int32_t m = hist[w][r];
      hist[w][r] = at;
      at += m;
    }
  }
  __syncthreads();

  for (int64_t g = g0; g < g1; g += AHEAD) {
    int32_t k[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) k[i] = token(g + i);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      uint64_t left = __ballot(k[i] >= lo && k[i] < lo + rows);
      while (left) {  // one token of the range after the other, all of its lanes at once
        const int first = __builtin_ctzll(left);
        const int32_t id = __builtin_amdgcn_readlane(k[i], first);
        const uint64_t same = __ballot(k[i] == id);
        const int32_t base = hist[wave][id - lo];
        if (k[i] == id) {
          const int32_t pos = base + __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0));
          a.order[pos] = (int32_t)((g + i) * 64 + lane);
          a.keys[pos] = id;
        }
        wave_lds_order();
        if (lane == first) hist[wave][id - lo] = base + __popcll(same);
        wave_lds_order();
        left &= ~same;
      }
    }
  }

  if (a.accumulate) return;
  for (int q = wave; q < rows; q += SORT_WAVES) {
    if (total[q]) continue;
    float* const row = a.dE + (int64_t)(lo + q) * a.d;
    Vec<float> zero;
    zero.v = f32x4{0.f, 0.f, 0.f, 0.f};
    int c = lane * 4;
    for (; c + 772 <= a.d; c += 1024)
#pragma unroll
      for (int i = 0; i < 4; ++i) zero.store(row + c + i * 256, 4);
    for (; c < a.d; c += 256) zero.store(row + c, a.d - c);
  }
}

// Four columns of a row from p on, `n` of them there: scaled sums that are added to what there is (accumulate) or stored.
__device__ __forceinline__ void put_row(const EmbedBwdArgs& a, int32_t key, int c, f32x4 s) {
  float* const p = a.dE + (int64_t)key * a.d + c;
  const int n = a.d - c;
  Vec<float> v;
  if (a.accumulate) {
    v.load(p, n, 0.f);
    v.v += s * a.scale;
  } else {
    v.v = s * a.scale;
  }
  v.store(p, n);
}
// (rows of the workspace are padded to whole vectors)
__device__ __forceinline__ void put_part(const EmbedBwdArgs& a, int64_t slot, int c, f32x4 s) {
  *reinterpret_cast<f32x4*>(a.part + slot * a.part_ld + c) = s;
}
// Four elements of a row that starts anywhere.
template <typename T> struct Quad;
template <> struct Quad<float> { typedef f32x4 type; };
template <> struct Quad<bf16_t> { typedef bf16x4 type; };

// Partial sums: slot 2 i is the beginning of chunk i, which belongs to a run that begins before it, slot 2 i + 1 its end, of a run that
// begins in it and goes on behind it.
//
// A wave takes 512 columns of a chunk's rows, a lane four of either half, so that its stores, like its loads, go to whole lines.  (Eight
// neighbouring columns a lane, whose float32 results are stored half a line at a time: 71 us for 32768 tokens of width 2048.)  The
// rows are loaded a batch at a time, without a branch between the loads, which would make them wait for each other: a lane at or behind the
// row's end loads the row's last four columns.  (EDGE: the row's length is no multiple of four, and a lane at its end needs some of
// them; the columns of rows of less than four are loaded one by one.)
template <typename T, bool EDGE, bool NARROW = false>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedBwdArgs a) {
  typedef typename Quad<T>::type quad_t;
  typedef quad_t quad_u __attribute__((aligned(sizeof(T))));
  constexpr int SEG = 512, AHEAD = 8;
  const int lane = threadIdx.x & 63;
  const int segs = (a.d + SEG - 1) / SEG;
  const int64_t u = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t i = u / segs;
  const int n_sorted = *a.n_sorted;
  const int64_t first = i * a.chunk;
  if (first >= n_sorted) return;
  const int n = (int)min((int64_t)a.chunk, n_sorted - first);
  const int c = (int)(u - i * segs) * SEG + lane * 4;
  // lane q holds place first + q of the list (a.chunk <= 64), and the keys around the chunk
  const int32_t order = a.order[first + min(lane, n - 1)];
  const int32_t key = lane < n ? a.keys[first + lane] : -1;
  const int32_t key_before = __builtin_amdgcn_readfirstlane(first > 0 ? a.keys[first - 1] : -1);
  const int32_t key_after = __builtin_amdgcn_readfirstlane(first + n < n_sorted ? a.keys[first + n] : -1);
  // places where a run ends
  const int32_t key_right = __shfl_down(key, 1, 64);
  const uint64_t ends = __ballot(lane < n && (lane == n - 1 || key != key_right));
  const T* const base = static_cast<const T*>(a.dX);
  auto load = [&](const T* row, int col) {
    if constexpr (NARROW) {
      quad_t v = {};
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (col + e < a.d) v[e] = row[col + e];
      return v;
    }
    // (read once, whole lines: with the hint 46 us where 68 were.  A wave's columns of an EDGE row begin and end inside a line, which
    // would come twice then)
    if constexpr (EDGE) return (quad_t)*reinterpret_cast<const quad_u*>(row + min(col, a.d - 4));
    else return (quad_t)__builtin_nontemporal_load(reinterpret_cast<const quad_u*>(row + min(col, a.d - 4)));
  };
  // what was loaded for columns c + 256 h on, of which the row's last vector may hold the first ones further on
  auto value = [&](quad_t v, int h, int e) {
    if constexpr (!EDGE || NARROW) return (float)v[e];
    const int by = max(c + h * 256 - (a.d - 4), 0);
    float x = (float)v[e];
#pragma unroll
    for (int k = 1; k + e < 4; ++k) x = by == k ? (float)v[e + k] : x;
    return x;
  };
  f32x4 s[2] = {};
  bool from_before = __builtin_amdgcn_readlane(key, 0) == key_before;
  for (int q0 = 0; q0 < n; q0 += AHEAD) {
    quad_t v[AHEAD][2];
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      const T* const row = base + (int64_t)__builtin_amdgcn_readlane(order, min(q0 + q, n - 1)) * a.d;
#pragma unroll
      for (int h = 0; h < 2; ++h) v[q][h] = load(row, c + h * 256);
    }
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      if (q0 + q < n) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[h][e] += value(v[q][h], h, e);
        if (ends >> (q0 + q) & 1) {
          const bool last = q0 + q == n - 1;
          const int32_t k = __builtin_amdgcn_readlane(key, q0 + q);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (c + h * 256 < a.d) {
              if (from_before) put_part(a, 2 * i, c + h * 256, s[h]);
              else if (last && k == key_after) put_part(a, 2 * i + 1, c + h * 256, s[h]);
              else put_row(a, k, c + h * 256, s[h]);
            }
            s[h] = f32x4{0.f, 0.f, 0.f, 0.f};
          }
          from_before = false;
        }
      }
    }
  }
}

// A block for each chunk and 256 columns: if a run begins in the chunk and goes on behind it, its partial sums are added up.
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedBwdArgs a) {
  __shared__ f32x4 sums[3][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int segs = (a.d + 255) / 256;
  const int64_t i = blockIdx.x / segs;
  const int n_sorted = *a.n_sorted;
  const int64_t behind = (i + 1) * a.chunk;
  if (behind >= n_sorted) return;
  const int32_t key = a.keys[behind - 1];
  if (key != a.keys[behind]) return;
  const int64_t first = i * a.chunk;
  if (first > 0 && a.keys[first] == key && a.keys[first - 1] == key) return;  // it begins before
  // chunks that the run reaches into, 64 looked at together: slots 2 (i + 1), ..., 2 (i + more)
  int64_t more = 1;
  for (;;) {
    const int64_t at = behind + (more + lane) * a.chunk;
    const uint64_t other = __ballot(at >= n_sorted || a.keys[min(at, (int64_t)n_sorted - 1)] != key);
    if (other) {
      more += __builtin_ctzll(other);
      break;
    }
    more += 64;
  }
  const int c = (int)(blockIdx.x % segs) * 256 + lane * 4;
  const int64_t per = (more + 3) / 4, j0 = wave * per, j1 = j0 + per < more ? j0 + per : more;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (c < a.d) {
    if (wave == 0) s = *reinterpret_cast<const f32x4*>(a.part + (2 * i + 1) * a.part_ld + c);
    constexpr int AHEAD = 8;
    for (int64_t j = j0; j < j1; j += AHEAD) {
      f32x4 v[AHEAD];
#pragma unroll
      for (int q = 0; q < AHEAD; ++q)
        if (j + q < j1) v[q] = *reinterpret_cast<const f32x4*>(a.part + 2 * (i + 1 + j + q) * a.part_ld + c);
#pragma unroll
      for (int q = 0; q < AHEAD; ++q)
        if (j + q < j1) s += v[q];
    }
  }
  if (wave > 0) sums[wave - 1][lane] = s;
  __syncthreads();
  if (wave > 0 || c >= a.d) return;
  for (int w = 0; w < 3; ++w) s += sums[w][lane];
  put_row(a, key, c, s);
}

template <typename T>
hipError_t run_fwd(const EmbedFwdArgs& a, hipStream_t s) {
  constexpr int SEG = 64 * LOOKUP_VECS * Vec<T>::N;
  const int64_t blocks = (a.T * ((a.d + SEG - 1) / SEG) + 3) / 4;
  hipLaunchKernelGGL((embed_lookup_kernel<T>), dim3((unsigned)(blocks < (1 << 20) ? blocks : 1 << 20)), dim3(256), 0, s, a);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_embed_fwd(modse_dtype dt, const EmbedFwdArgs& a, hipStream_t s) {
  return dt == MODSE_F32 ? run_fwd<float>(a, s) : run_fwd<bf16_t>(a, s);
}

hipError_t launch_embed_bwd(modse_dtype dt, const EmbedBwdArgs& a, hipStream_t s) {
  // Two blocks for every CU, as each reads all tokens.  (One: 88 us for 1021 tokens of width 1535, float32, vocabulary 50257, in place of 84,
  // and the same for 32768 tokens.)
  const int rows = std::min(EMBED_MAX_ROWS, (a.vocab + 511) / 512);
  hipLaunchKernelGGL(embed_sort_kernel, dim3((unsigned)((a.vocab + rows - 1) / rows)), dim3(SORT_WAVES * 64), 0, s, a, rows);
  const int64_t chunks = embed_chunks(a.T);
  const dim3 sums((unsigned)((chunks * ((a.d + 511) / 512) + 3) / 4)), joins((unsigned)(chunks * ((a.d + 255) / 256)));
  auto run = [&](auto t) {
    typedef decltype(t) T;
    if (a.d % 4 == 0) hipLaunchKernelGGL((embed_sum_kernel<T, false>), sums, dim3(256), 0, s, a);
    else if (a.d > 4) hipLaunchKernelGGL((embed_sum_kernel<T, true>), sums, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((embed_sum_kernel<T, true, true>), sums, dim3(256), 0, s, a);
  };
  if (dt == MODSE_F32) run(float{});
  else run(bf16_t{});
  if (chunks > 1) hipLaunchKernelGGL(embed_join_kernel, joins, dim3(256), 0, s, a);
  return hipGetLastError();
}
