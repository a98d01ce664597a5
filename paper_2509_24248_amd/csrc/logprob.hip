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

// Keys in the order (logit descending, index ascending); none is 0.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float of_ordered(uint32_t k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xFFFFFFFFu)); }
__device__ __forceinline__ u64 key_of(float x, int i) { return static_cast<u64>(ordered(x)) << 32 | (0xFFFFFFFFu - static_cast<uint32_t>(i)); }
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
// The n-th largest of m values of LDS (duplicates count), m <= 128, by counting; the same in every wave.
__device__ __forceinline__ u64 nth_largest(const u64* v, int m, int n) {
  const int lane = threadIdx.x & 63;
  u64 mine[2], found = 0;
  int before[2] = {0, 0};
#pragma unroll
  for (int u = 0; u < 2; ++u) mine[u] = lane + 64 * u < m ? v[lane + 64 * u] : 0;
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
// Every one of `count` distinct keys counts how many are above it; the n best go to out in their order, the rest of out is 0.
__device__ __forceinline__ void rank_keys(const u64* list, int count, int n, u64* out) {
  for (int i = threadIdx.x; i < count; i += kThreads) {
    const u64 mine = list[i];
    int before = 0;
    for (int j = 0; j < count; ++j) before += list[j] > mine;
    if (before < n) out[before] = mine;
  }
  for (int i = count + threadIdx.x; i < n; i += kThreads) out[i] = 0;
}

template <typename T, int EPT>
__global__ __launch_bounds__(kThreads) void k_logprob_chunk(const LogprobArgs a) {
  constexpr int N = 16 / sizeof(T), U = EPT / N;
  __shared__ float group_max[kGroups];
  __shared__ u64 group_key[kGroups];
  __shared__ float sums[kThreads / 64][3];
  __shared__ u64 list[kList], best_of[kThreads / 64];
  __shared__ int listed;
  const int c = blockIdx.x, r = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const T* row = static_cast<const T*>(a.logits) + static_cast<int64_t>(r) * a.ld;
  // chunks begin at multiples of 16 bytes: `skew` values in front of the row
  const int skew = static_cast<int>(reinterpret_cast<uintptr_t>(row) & 15) / static_cast<int>(sizeof(T));
  const int base = c * (kThreads * EPT) - skew;
  float x[EPT];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = base + (u * kThreads + tid) * N;
    if (i >= 0 && i + N <= a.V) {
      const uint4 v = *reinterpret_cast<const uint4*>(row + i);
      if constexpr (sizeof(T) == 2) {
        float f[8];
        unpack16(v, f);
#pragma unroll
        for (int e = 0; e < N; ++e) x[u * N + e] = f[e];
      } else {
        x[u * N] = __uint_as_float(v.x); x[u * N + 1] = __uint_as_float(v.y);
        x[u * N + 2] = __uint_as_float(v.z); x[u * N + 3] = __uint_as_float(v.w);
      }
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) x[u * N + e] = i + e >= 0 && i + e < a.V ? Elem<T>::load(row + i + e) : -INFINITY;
    }
  }
  if (tid == 0) listed = 0;
  float mine = -INFINITY;
#pragma unroll
  for (int e = 0; e < EPT; ++e) {
    x[e] = (x[e] != x[e] ? -INFINITY : x[e]) + 0.f;       // NaN counts as ruled out, the zeros as one
    mine = fmaxf(mine, x[e]);
  }
  // maxima of eight lanes
  float g = mine;
  g = fmaxf(g, row_lane<0xB1>(g));
  g = fmaxf(g, row_lane<0x4E>(g));
  g = fmaxf(g, row_lane<0x141>(g));
  if ((lane & 7) == 0) group_max[tid >> 3] = g;
  __syncthreads();
  float top = group_max[lane & (kGroups - 1)];
  top = wave_max_dpp(top);
  const float heat = row_heat(a, r), unit = kLog2e / heat;
  const float ref = top == -INFINITY ? 0.f : top;
  float s = 0.f, w = 0.f;
  int n = 0;
#pragma unroll
  for (int e = 0; e < EPT; ++e) {
    const bool is_top = x[e] == top;
    const float y = fmaxf((x[e] - ref) * unit, -1000.f);  // (2^-1000 is 0; of the best ones, where both are infinite, not used)
    const float p = __builtin_amdgcn_exp2f(y);
    n += is_top;
    s += is_top ? 0.f : p;
    w += is_top ? 0.f : p * y;
  }
  float nf = top == -INFINITY ? 0.f : static_cast<float>(n);
  s = wave_sum_dpp(s);
  w = wave_sum_dpp(w);
  nf = wave_sum_dpp(nf);
  if (lane == 0) { sums[tid >> 6][0] = nf; sums[tid >> 6][1] = s; sums[tid >> 6][2] = w; }
  const bool select = a.n_top > 0;
  float bound = INFINITY;
  if (select) {
    if (tid < kGroups) group_key[tid] = ordered(group_max[tid]);
    __syncthreads();
    bound = of_ordered(static_cast<uint32_t>(nth_largest(group_key, kGroups, a.n_top)));
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
      if (x[e] >= bound && x[e] > -INFINITY) {
        const int at = atomicAdd(&listed, 1);
        if (at < kList) list[at] = key_of(x[e], base + (e / N * kThreads + tid) * N + e % N);
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

template <typename T>
__global__ __launch_bounds__(kThreads) void k_logprob_row(const LogprobArgs a) {
  __shared__ u64 heads[128], list[kLogprobMaxTop * kLogprobMaxTop], ranked[kLogprobMaxTop];
  __shared__ int listed;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const float4* stats = a.stats + static_cast<int64_t>(r) * a.chunks;
  // the token's logits are wanted last and asked for first
  float mine = 0.f;
  bool known = false;
  if (tid < a.n_tok) {
    const int token = a.token[static_cast<int64_t>(r) * a.n_tok + tid];
    known = token >= 0 && token < a.V;
    if (!known && token != -1) report_status(a.status, kStatusBadToken);
    if (known) mine = Elem<T>::load(static_cast<const T*>(a.logits) + static_cast<int64_t>(r) * a.ld + token);
  }
  const float heat = row_heat(a, r), unit = kLog2e / heat;
  float top = -INFINITY;
  for (int c = lane; c < a.chunks; c += 64) top = fmaxf(top, stats[c].x);
  top = wave_max_dpp(top);
  float n = 0.f, s = 0.f, w = 0.f;
  for (int c = lane; c < a.chunks; c += 64) {
    const float4 t = stats[c];
    if (t.x == -INFINITY) continue;
    if (t.x == top) {
      n += t.y; s += t.z; w += t.w;
    } else {
      const float y = fmaxf((t.x - top) * unit, -1000.f), f = __builtin_amdgcn_exp2f(y);
      s += f * (t.y + t.z);
      w += f * (t.w + y * (t.y + t.z));
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
  // the n-th largest of the chunks' best bounds the row's n-th: at most n chunks meet it, with n values each
  const u64* best = a.best + static_cast<int64_t>(r) * a.chunks * a.n_top;
  if (tid == 0) listed = 0;
  for (int c = tid; c < a.chunks; c += kThreads) heads[c] = best[static_cast<int64_t>(c) * a.n_top];
  __syncthreads();
  u64 bound = a.chunks < a.n_top ? 0 : nth_largest(heads, a.chunks, a.n_top);
  if (bound == 0) bound = 1;
  for (int i = tid; i < a.chunks * a.n_top; i += kThreads) {
    const u64 key = best[i];
    if (key >= bound) list[atomicAdd(&listed, 1)] = key;
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
  a.wide = static_cast<int64_t>(a.M) * chunks_of(a.V, kWide) >= kFewChunks || chunks_of(a.V, kNarrow) > 128;
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
