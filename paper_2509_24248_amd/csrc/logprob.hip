// Log probabilities of given tokens, entropy and best alternatives of rows of logits.
//
// With l' = l / T, M = max l, y = (l - M) / T, n = how many tokens equal M, S = sum over the others of e^y, U = sum of y e^y:
//   ln p_i = y_i - ln n - ln(1 + S / n),   H = ln n + ln(1 + S / n) - U / (n + S)
// The best tokens' weight is counted, not summed: a row whose best token has nearly everything keeps the digits of what is left.
//
// Two launches.  k_logprob_chunk reads the logits once: a workgroup holds a chunk of a row in registers, 8 or 32 values a thread, takes its maximum, its sums and its
// n_top best.  k_logprob_row, a workgroup per row, adds the chunks' sums, in their order, and selects among their best.
//
// The best of a chunk without sorting it: the n-th largest of the maxima of 32 groups of threads is a bound that at least n values meet, and about n (1 + n / 64) of 8192
// do; those go to a list in LDS, where every one counts how many are before it.  Where more than the list holds do (many equal values, or a chunk sorted so that a
// few groups have them all), the chunk is searched n times for the best that is left.
#include "common.hpp"
#include "kernels.hpp"

#include <float.h>
#include <limits.h>
#include <algorithm>
#include <type_traits>

namespace sx {

namespace {

constexpr int kThreads = 256;
constexpr int kGroups = 32;            // of eight threads
constexpr int kList = 512;             // candidates of a chunk
constexpr int kNarrow = 8, kWide = 32; // values of a thread
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;

typedef unsigned long long u64;

// Keys in the order (logit descending, index ascending); none is 0.  (Adding zero makes one zero of two.)
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float of_ordered(uint32_t k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xFFFFFFFFu)); }
__device__ __forceinline__ u64 key_of(float x, int i) { return static_cast<u64>(ordered(x + 0.f)) << 32 | (0xFFFFFFFFu - static_cast<uint32_t>(i)); }
__device__ __forceinline__ int index_of(u64 key) { return static_cast<int>(0xFFFFFFFFu - static_cast<uint32_t>(key)); }

// units of the exponent per logit: log2(e) / T
__device__ __forceinline__ float row_heat(const LogprobArgs& a, int r) {
  return a.temperature ? fminf(fmaxf(a.temperature[r / a.rows_per_seq], 0x1p-10f), 0x1p96f) : 1.f;
}
__device__ __forceinline__ u64 wave_max_u64(u64 v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const u64 w = __shfl_xor(v, o, 64);
    v = w > v ? w : v;
  }
  return v;
}
// The n-th largest of the values that lanes 0 .. M - 1 hold (equal ones count apart), by counting.
template <int M>
__device__ __forceinline__ float nth_largest(float v, int n) {
  const int lane = threadIdx.x & 63;
  int before = 0;
#pragma unroll
  for (int j = 0; j < M; ++j) {
    const float x = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), j));
    before += x > v || (x == v && j < lane);
  }
  const uint64_t it = __builtin_amdgcn_ballot_w64(lane < M && before == n - 1);
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), static_cast<int>(__builtin_ctzll(it))));
}
// The n-th largest of m <= 128 distinct keys of LDS, in every wave.
__device__ __forceinline__ u64 nth_largest(const u64* v, int m, int n) {
  const int lane = threadIdx.x & 63;
  u64 mine[2], found = 0;
  int before[2] = {0, 0};
#pragma unroll
  for (int u = 0; u < 2; ++u) mine[u] = lane + 64 * u < m ? v[lane + 64 * u] : 0;
#pragma unroll 4
  for (int j = 0; j < m; ++j) {
    const u64 x = v[j];
#pragma unroll
    for (int u = 0; u < 2; ++u) before[u] += x > mine[u] || (x == mine[u] && j < lane + 64 * u);
  }
#pragma unroll
  for (int u = 0; u < 2; ++u)
    if (lane + 64 * u < m && before[u] == n - 1) found = mine[u];
  return wave_max_u64(found);
}
// Places in a list of LDS for the lanes that want one: one atomic operation a wave.
__device__ __forceinline__ int list_place(int* listed, bool wanted) {
  const uint64_t who = __builtin_amdgcn_ballot_w64(wanted);
  if (!who) return 0;
  const int lane = threadIdx.x & 63;
  int first = 0;
  if (lane == 0) first = atomicAdd(listed, static_cast<int>(__popcll(who)));
  first = __builtin_amdgcn_readfirstlane(first);
  return first + static_cast<int>(__popcll(who & ((1ull << lane) - 1)));
}
// Every one of `count` distinct keys counts how many are above it; the n best go to out in their order, the rest of out is 0.
__device__ __forceinline__ void rank_keys(const u64* list, int count, int n, u64* out) {
  for (int i = threadIdx.x; i < count; i += kThreads) {
    const u64 mine = list[i];
    int before = 0;
#pragma unroll 4
    for (int j = 0; j < count; ++j) before += list[j] > mine;
    if (before < n) out[before] = mine;
  }
  for (int i = count + threadIdx.x; i < n; i += kThreads) out[i] = 0;
}

// The sums of a thread's values from the best one of the chunk: p = 2^((x - ref) unit), sum of p and of p (x - ref).  What is ruled out, infinitely far below, weighs nothing; with a
// reference beyond 2^102 a distance can leave the range (FAR).
template <int EPT, bool FAR>
__device__ __forceinline__ void chunk_sums(const float (&x)[EPT], float ref, float unit, float& s, float& w) {
#pragma unroll
  for (int e = 0; e < EPT; ++e) {
    float d = fmaxf(x[e], -FLT_MAX) - ref;
    if (FAR) d = fmaxf(d, -FLT_MAX);
    const float p = __builtin_amdgcn_exp2f(d * unit);
    s += p;
    w = fmaf(p, d, w);
  }
}

// What a value costs here: 1 instruction for the maximum, 5 and an exponential for the sums, 2 for the candidates; what the best one's exclusion costs falls to the threads that hold one.
template <typename T, int EPT>
__global__ __launch_bounds__(kThreads) void k_logprob_chunk(const LogprobArgs a) {
  constexpr int N = 16 / sizeof(T), U = EPT / N;
  __shared__ float group_max[kGroups];
  __shared__ float sums[kThreads / 64][3];
  __shared__ u64 list[kList], best_of[kThreads / 64];
  __shared__ int listed;
  const int c = blockIdx.x, r = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const T* row = static_cast<const T*>(a.logits) + static_cast<int64_t>(r) * a.ld;
  // chunks begin at multiples of 16 bytes: `skew` values in front of the row
  const int skew = static_cast<int>(reinterpret_cast<uintptr_t>(row) & 15) / static_cast<int>(sizeof(T));
  const int base = c * (kThreads * EPT) - skew;
  float x[EPT];
  if (base >= 0 && base + kThreads * EPT <= a.V) {
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = *reinterpret_cast<const uint4*>(row + base + (u * kThreads + tid) * N);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if constexpr (sizeof(T) == 2) {
        float f[8];
        unpack16(v[u], f);
#pragma unroll
        for (int e = 0; e < N; ++e) x[u * N + e] = f[e];
      } else {
        x[u * N] = __uint_as_float(v[u].x); x[u * N + 1] = __uint_as_float(v[u].y);
        x[u * N + 2] = __uint_as_float(v[u].z); x[u * N + 3] = __uint_as_float(v[u].w);
      }
    }
  } else {                                                // a row's first or last chunk
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = base + (u * kThreads + tid) * N;
#pragma unroll
      for (int e = 0; e < N; ++e) x[u * N + e] = i + e >= 0 && i + e < a.V ? Elem<T>::load(row + i + e) : -INFINITY;
    }
  }
  if (tid == 0) listed = 0;
  float mine = -INFINITY;
#pragma unroll
  for (int e = 0; e < EPT; ++e) mine = fmaxf(mine, x[e]);         // (a NaN is passed over)
  // maxima of eight lanes
  float g = mine;
  g = fmaxf(g, row_lane<0xB1>(g));
  g = fmaxf(g, row_lane<0x4E>(g));
  g = fmaxf(g, row_lane<0x141>(g));
  if ((lane & 7) == 0) group_max[tid >> 3] = g;
  __syncthreads();
  const float groups = group_max[lane & (kGroups - 1)];
  const float top = wave_max_dpp(groups);
  const float heat = row_heat(a, r), unit = kLog2e / heat;
  const float ref = top == -INFINITY ? 0.f : top;
  float s = 0.f, w = 0.f, n = 0.f;
  if (fabsf(ref) < 0x1p102f) chunk_sums<EPT, false>(x, ref, unit, s, w);
  else chunk_sums<EPT, true>(x, ref, unit, s, w);
  if (mine == top) {                                      // the thread that holds the best value, or several: that one is counted
    s = w = 0.f;
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
      const bool is_top = x[e] == top;
      const float d = fmaxf(fmaxf(x[e], -FLT_MAX) - ref, -FLT_MAX), p = __builtin_amdgcn_exp2f(d * unit);
      n += is_top ? 1.f : 0.f;
      s += is_top ? 0.f : p;
      w += is_top ? 0.f : p * d;
    }
    if (top == -INFINITY) n = 0.f;
  }
  s = wave_sum_dpp(s);
  w = wave_sum_dpp(w);
  n = wave_sum_dpp(n);
  if (lane == 0) { sums[tid >> 6][0] = n; sums[tid >> 6][1] = s; sums[tid >> 6][2] = w * unit; }
  const bool select = a.n_top > 0;
  if (select) {
    const float bound = a.n_top == 1 ? top : nth_largest<kGroups>(groups, a.n_top);
    uint32_t meets = 0;
    if (mine >= bound) {
#pragma unroll
      for (int e = 0; e < EPT; ++e) meets |= (x[e] >= bound ? 1u : 0u) << e;
    }
    if (bound == -INFINITY) {                             // (what is ruled out meets it as well)
#pragma unroll
      for (int e = 0; e < EPT; ++e) meets &= ~((x[e] == -INFINITY ? 1u : 0u) << e);
    }
    while (__builtin_amdgcn_ballot_w64(meets != 0) != 0ull) {
      const bool has = meets != 0;
      const int at = list_place(&listed, has);
      if (has) {
        const int e = __builtin_ctz(meets), i = base + (e / N * kThreads + tid) * N + e % N;
        meets &= meets - 1;
        if (at < kList) list[at] = key_of(Elem<T>::load(row + i), i);          // (read again: registers have no index)
      }
    }
  }
  __syncthreads();
  const int64_t slot = static_cast<int64_t>(r) * a.chunks + c;
  if (tid == 0) {
    float4 t = make_float4(top, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kThreads / 64; ++k) { t.y += sums[k][0]; t.z += sums[k][1]; t.w += sums[k][2]; }
    a.stats[slot] = t;
  }
  if (!select) return;
  u64* out = a.best + slot * a.n_top;
  if (listed <= kList) {
    rank_keys(list, listed, a.n_top, out);
    return;
  }
  u64 last = ~0ull;
  for (int k = 0; k < a.n_top; ++k) {
    u64 key = 0;
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
      const u64 ke = key_of(x[e], base + (e / N * kThreads + tid) * N + e % N);
      if (x[e] > -INFINITY && ke < last && ke > key) key = ke;
    }
    key = wave_max_u64(key);
    __syncthreads();
    if (lane == 0) best_of[tid >> 6] = key;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kThreads / 64; ++j) key = best_of[j] > key ? best_of[j] : key;
    if (tid == 0) out[k] = key;
    last = key;
  }
}

constexpr int kMostChunks = 128;

template <typename T>
__global__ __launch_bounds__(kThreads) void k_logprob_row(const LogprobArgs a) {
  __shared__ u64 heads[kMostChunks], list[kLogprobMaxTop * kLogprobMaxTop], ranked[kLogprobMaxTop];
  __shared__ int listed;
  arguments_at_once<sizeof(LogprobArgs)>();
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const float4* stats = a.stats + static_cast<int64_t>(r) * a.chunks;
  const u64* best = a.best + static_cast<int64_t>(r) * a.chunks * a.n_top;
  // everything is asked for at once: the chunks' sums, their t-th best, the tokens' logits
  constexpr int kPer = kMostChunks / 64;
  float4 st[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) st[k] = lane + 64 * k < a.chunks ? stats[lane + 64 * k] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
  // ceil(n / t) chunks whose t-th best meet a bound hold n values that do; the least t that as many chunks as there are suffice for
  const int t = a.n_top ? (a.n_top + a.chunks - 1) / a.chunks : 1;
  if (a.n_top && tid < a.chunks) heads[tid] = best[static_cast<int64_t>(tid) * a.n_top + t - 1];
  float mine = 0.f;
  bool known = false;
  if (tid < a.n_tok) {
    const int token = a.token[static_cast<int64_t>(r) * a.n_tok + tid];
    known = token >= 0 && token < a.V;
    if (!known && token != -1) report_status(a.status, kStatusBadToken);
    if (known) mine = Elem<T>::load(static_cast<const T*>(a.logits) + static_cast<int64_t>(r) * a.ld + token);
  }
  if (tid == 0) listed = 0;
  const float heat = row_heat(a, r), unit = kLog2e / heat;
  float top = -INFINITY;
#pragma unroll
  for (int k = 0; k < kPer; ++k) top = fmaxf(top, st[k].x);
  top = wave_max_dpp(top);
  float n = 0.f, s = 0.f, w = 0.f;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (st[k].x == -INFINITY) continue;
    if (st[k].x == top) {
      n += st[k].y; s += st[k].z; w += st[k].w;
    } else {
      const float y = fmaxf((st[k].x - top) * unit, -1000.f), f = __builtin_amdgcn_exp2f(y);
      s += f * (st[k].y + st[k].z);
      w += f * (st[k].w + y * (st[k].y + st[k].z));
    }
  }
  n = wave_sum_dpp(n);
  s = wave_sum_dpp(s);
  w = wave_sum_dpp(w);
  const float norm = logf(n) + log1pf(s / n);             // ln of the sum of the weights
  auto logprob = [&](float x) {
    if (x != x || x == -INFINITY || top == -INFINITY) return -INFINITY;
    return (x == top ? 0.f : 2.f * ((0.5f * x - 0.5f * top) / heat)) - norm;       // (halves: their difference stays in range)
  };
  if (tid < a.n_tok) a.logprob[static_cast<int64_t>(r) * a.n_tok + tid] = known ? logprob(mine) : __uint_as_float(0x7FC00000u);
  if (tid == 0 && a.entropy) a.entropy[r] = top == -INFINITY ? 0.f : norm - kLn2 * w / (n + s);
  if (a.n_top == 0) return;
  __syncthreads();
  u64 bound = nth_largest(heads, a.chunks, (a.n_top + t - 1) / t);
  if (bound == 0) bound = 1;
  for (int i0 = 0; i0 < a.chunks * a.n_top; i0 += kThreads) {
    const u64 key = i0 + tid < a.chunks * a.n_top ? best[i0 + tid] : 0;
    const int at = list_place(&listed, key >= bound);
    if (key >= bound) list[at] = key;
  }
  __syncthreads();
  rank_keys(list, listed, a.n_top, ranked);
  __syncthreads();
  if (tid < a.n_top) {
    const u64 key = ranked[tid];
    a.top_token[static_cast<int64_t>(r) * a.n_top + tid] = key ? index_of(key) : -1;
    if (a.top_logprob) a.top_logprob[static_cast<int64_t>(r) * a.n_top + tid] = key ? logprob(of_ordered(static_cast<uint32_t>(key >> 32))) : -INFINITY;
  }
}

// chunks of a row, its alignment not known
int chunks_of(int V, int per_thread) { return (V + 7 + kThreads * per_thread - 1) / (kThreads * per_thread); }

template <typename T>
void launch_as(const LogprobArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(a.chunks), static_cast<unsigned>(a.M));
  if (a.wide) hipLaunchKernelGGL((k_logprob_chunk<T, kWide>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((k_logprob_chunk<T, kNarrow>), grid, dim3(kThreads), 0, s, a);
  hipLaunchKernelGGL(k_logprob_row<T>, dim3(static_cast<unsigned>(a.M)), dim3(kThreads), 0, s, a);
}

}  // namespace

// Few rows are cut finer, so that they fill the chip too.
constexpr int64_t kFewChunks = 512;
void logprob_plan(LogprobArgs& a) {
  a.wide = static_cast<int64_t>(a.M) * chunks_of(a.V, kWide) >= kFewChunks || chunks_of(a.V, kNarrow) > kMostChunks;
  a.chunks = chunks_of(a.V, a.wide ? kWide : kNarrow);
}

size_t logprob_carve(LogprobArgs& a, void* base) {
  // never less for more rows or a larger V: narrow chunks count four times those of kFewChunks at most
  const int64_t wide = static_cast<int64_t>(a.M) * chunks_of(a.V, kWide), narrow = static_cast<int64_t>(a.M) * chunks_of(a.V, kNarrow);
  const size_t chunks = static_cast<size_t>(std::max(wide, std::min(narrow, 4 * kFewChunks)));
  char* p = static_cast<char*>(base);
  a.stats = reinterpret_cast<float4*>(p);
  const size_t stats = (chunks * sizeof(float4) + 255) & ~static_cast<size_t>(255);
  a.best = reinterpret_cast<unsigned long long*>(p + stats);
  return stats + ((chunks * a.n_top * sizeof(unsigned long long) + 255) & ~static_cast<size_t>(255));
}

hipError_t launch_logprob(const LogprobArgs& a, hipStream_t s) {
  if (a.f32) launch_as<float>(a, s);
  else launch_as<bf16_t>(a, s);
  return hipGetLastError();
}

}  // namespace sx
