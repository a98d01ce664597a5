// Log probabilities of given tokens, entropy and best alternatives of rows of logits.
//
// With l' = l / T, M = max l, y = (l - M) / T, n = how many tokens equal M, S = sum over the others of e^y, U = sum of y e^y:
//   ln p_i = y_i - ln n - ln(1 + S / n),   H = ln n + ln(1 + S / n) - U / (n + S)
// The best tokens' weight is counted, not summed: a row whose best token has nearly everything keeps the digits of what is left.
//
// Two launches.  k_logprob_part reads the logits once: a wave holds 16 or 32 values a lane and takes its maximum, its sums and the maxima of its eight groups of eight lanes; no
// barrier, no LDS.  k_logprob_row, a workgroup per row, adds the parts' sums, in their order, and finds the row's n_top best: the n-th largest of the maxima of
// 64 sets of groups is a bound that at least n values meet and, in any order of the logits that does not conspire, few more; the groups that reach it (n and some) are read again, a
// load instruction each, and what meets the bound goes to a list in LDS, where every one counts how many are before it.
// A list that runs over (many equal values, or a few groups that hold all the best) is cut to its n best, whose last becomes the bound, and the groups go on.
#include "common.hpp"
#include "kernels.hpp"

#include <float.h>
#include <limits.h>
#include <algorithm>
#include <type_traits>

namespace sx {

namespace {

constexpr int kThreads = 256;
constexpr int kNarrow = 16, kWide = 32;                    // values of a lane
constexpr int kMostParts = 272;                            // parts of a row at most: 2^18 logits, 1024 a part
constexpr int kList = 1536;                                // candidates
constexpr float kLog2e = 1.44269504088896340736f, kLog2eRest = 1.9259630e-8f, kLn2 = 0.693147180559945309417f;

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
// The n-th largest of a wave's values, equal ones counting apart: the least that fewer than n are above.
__device__ __forceinline__ float nth_largest(float v, int n) {
  int above = 0;
#pragma unroll
  for (int j = 0; j < 64; ++j) above += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), j)) > v;
  return -wave_max_dpp(above < n ? -v : -INFINITY);
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

// Maxima that hand a NaN on: the instruction takes three values and needs no quieting of its inputs, of which there would be one each.
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// A lane's 16 bytes of a row from value i on, ruled out where they are not of the row.
template <typename T>
__device__ __forceinline__ void load_piece(const T* row, int i, int V, float (&f)[16 / sizeof(T)]) {
  constexpr int N = 16 / sizeof(T);
  if (i >= 0 && i + N <= V) {
    const uint4 v = *reinterpret_cast<const uint4*>(row + i);
    if constexpr (sizeof(T) == 2) {
      unpack16(v, f);
    } else {
      f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = i + e >= 0 && i + e < V ? Elem<T>::load(row + i + e) : -INFINITY;
  }
}
// Parts begin at multiples of 16 bytes: values in front of the row.
template <typename T> __device__ __forceinline__ int row_skew(const T* row) {
  return static_cast<int>(reinterpret_cast<uintptr_t>(row) & 15) / static_cast<int>(sizeof(T));
}

// Bound by vector instructions before memory: 8.5 and an exponential a value (half a maximum, 2 that take the best one out, 6 for the sums).
template <typename T, int EPT>
__global__ __launch_bounds__(kThreads) void k_logprob_part(const LogprobArgs a) {
  constexpr int N = 16 / sizeof(T), U = EPT / N;
  const int lane = threadIdx.x & 63, r = blockIdx.y;
  const int part = blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (part >= a.parts) return;
  const T* row = static_cast<const T*>(a.logits) + static_cast<int64_t>(r) * a.ld;
  const int base = part * (64 * EPT) - row_skew(row);
  float x[EPT];
  if (base >= 0 && base + 64 * EPT <= a.V) {
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = *reinterpret_cast<const uint4*>(row + base + (u * 64 + lane) * N);
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
  } else {                                                // a row's first or last part
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[N];
      load_piece(row, base + (u * 64 + lane) * N, a.V, f);
#pragma unroll
      for (int e = 0; e < N; ++e) x[u * N + e] = f[e];
    }
  }
  float mine = x[0];
#pragma unroll
  for (int e = 1; e < EPT; ++e) mine = max_nan(mine, x[e]);
  if (__builtin_amdgcn_ballot_w64(mine != mine) != 0ull) {        // (uniform, rare) NaN counts as ruled out
    mine = -INFINITY;
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
      x[e] = x[e] != x[e] ? -INFINITY : x[e];
      mine = max_nan(mine, x[e]);
    }
  }
  float g = mine;                                         // of eight lanes
  g = fmaxf(g, row_lane<0xB1>(g));
  g = fmaxf(g, row_lane<0x4E>(g));
  g = fmaxf(g, row_lane<0x141>(g));
  const int64_t slot = static_cast<int64_t>(r) * a.parts + part;
  if (a.n_top && (lane & 7) == 0) a.groups[slot * 8 + (lane >> 3)] = g;
  const float top = quad_row_max(fmaxf(g, row_lane<0x128>(g)));
  const float unit = kLog2e / row_heat(a, r);
  const float ref = top == -INFINITY ? 0.f : top;
  // what equals the best one is counted and taken out; the sums are of p = 2^(d unit) and p d, d = x - ref, from -FLT_MAX on (what is ruled out weighs nothing)
  float s = 0.f, w = 0.f;
  int n = 0;
#pragma unroll
  for (int e = 0; e < EPT; ++e) {
    const bool is_top = x[e] == top;
    n += static_cast<int>(__popcll(__builtin_amdgcn_ballot_w64(is_top)));
    const float d = max_nan((is_top ? -INFINITY : x[e]) - ref, -FLT_MAX), p = __builtin_amdgcn_exp2f(d * unit);
    s += p;
    w = fmaf(p, d, w);
  }
  s = wave_sum_dpp(s);
  w = wave_sum_dpp(w);
  if (lane == 0) a.stats[slot] = make_float4(top, top == -INFINITY ? 0.f : static_cast<float>(n), s, w * unit);
}

template <typename T, int EPT>
__global__ __launch_bounds__(kThreads) void k_logprob_row(const LogprobArgs a) {
  constexpr int N = 16 / sizeof(T), U = EPT / N, kLanes = 8 * U;         // lanes that read a group again
  constexpr int kPer = (kMostParts + 63) / 64, kGroupsPer = kMostParts * 8 / kThreads + 1;
  static_assert(kLanes <= 64, "");
  __shared__ float waves_max[kThreads / 64][64];
  __shared__ uint16_t met[kMostParts * 8];
  __shared__ u64 list[kList], ranked[kLogprobMaxTop];
  __shared__ int listed, groups_met;
  arguments_at_once<sizeof(LogprobArgs)>();
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const T* row = static_cast<const T*>(a.logits) + static_cast<int64_t>(r) * a.ld;
  const int64_t first = static_cast<int64_t>(r) * a.parts;
  // everything is asked for at once: the parts' sums, the groups' maxima, the tokens' logits
  float4 st[kPer];
  float gm[kGroupsPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) st[k] = lane + 64 * k < a.parts ? a.stats[first + lane + 64 * k] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
  if (a.n_top) {
#pragma unroll
    for (int k = 0; k < kGroupsPer; ++k) gm[k] = tid + kThreads * k < a.parts * 8 ? a.groups[first * 8 + tid + kThreads * k] : -INFINITY;
  }
  float mine = 0.f;
  bool known = false;
  if (tid < a.n_tok) {
    const int token = a.token[static_cast<int64_t>(r) * a.n_tok + tid];
    known = token >= 0 && token < a.V;
    if (!known && token != -1) report_status(a.status, kStatusBadToken);
    if (known) mine = Elem<T>::load(row + token);
  }
  if (tid == 0) listed = groups_met = 0;
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
  // The exponents' unit was rounded, log2(e) (1 - off) / T in its place: to first order the sum is off by off times its weights' logarithms, which w has.  (bf16 logits with
  // temperatures: the best alternatives' log probabilities 7.7e-8 of their norm away from 64 bits without, 3.7e-8 with it.  The entropy is left as that of the rounded unit, off times the
  // logarithms' variance away.)
  const float off = (fmaf(-unit, heat, kLog2e) + kLog2eRest) * kLn2;
  const float norm = logf(n) + log1pf(fmaxf(fmaf(off * kLn2, w, s), 0.f) / n);             // ln of the sum of the weights
  auto logprob = [&](float x) {
    if (x != x || x == -INFINITY || top == -INFINITY) return -INFINITY;
    return (x == top ? 0.f : 2.f * ((0.5f * x - 0.5f * top) / heat)) - norm;       // (halves: their difference stays in range)
  };
  if (tid < a.n_tok) a.logprob[static_cast<int64_t>(r) * a.n_tok + tid] = known ? logprob(mine) : __uint_as_float(0x7FC00000u);
  if (tid == 0 && a.entropy) a.entropy[r] = top == -INFINITY ? 0.f : logf(n) + log1pf(s / n) - kLn2 * w / (n + s);
  if (a.n_top == 0) return;
  // ---- the bound, and the groups that meet it
  float best = -INFINITY;
#pragma unroll
  for (int k = 0; k < kGroupsPer; ++k) best = fmaxf(best, gm[k]);
  waves_max[wv][lane] = best;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kThreads / 64; ++k) best = fmaxf(best, waves_max[k][lane]);
  const float bound = a.n_top == 1 ? wave_max_dpp(best) : nth_largest(best, a.n_top);
#pragma unroll
  for (int k = 0; k < kGroupsPer; ++k) {
    const bool meets = gm[k] >= bound && gm[k] > -INFINITY;
    const int at = list_place(&groups_met, meets);
    if (meets) met[at] = static_cast<uint16_t>(tid + kThreads * k);
  }
  __syncthreads();
  const int count = groups_met, skew = row_skew(row);
  u64 least = 0;                                          // of the list's best, once it was cut
  // group i of those: eight lanes of a part, U pieces of each
  auto place_of = [&](int i) {
    const int id = met[i];
    return (id >> 3) * (64 * EPT) - skew + ((lane >> 3) * 64 + (id & 7) * 8 + (lane & 7)) * N;
  };
  auto keep = [&](const float (&f)[N], int at, bool mine) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const u64 key = key_of(f[e], at + e);
      const bool in = mine && f[e] >= bound && f[e] > -INFINITY && key > least;
      const int place = list_place(&listed, in);
      if (in && place < kList) list[place] = key;
    }
  };
  constexpr int kWaves = kThreads / 64;
  constexpr int kTogether = 8;                            // groups of a wave that are asked for together
#pragma unroll 1
  for (int i0 = wv; i0 < count; i0 += kWaves * kTogether) {
    float f[kTogether][N];
#pragma unroll
    for (int k = 0; k < kTogether; ++k) {
      const int i = i0 + k * kWaves;
      if (i < count && lane < kLanes) load_piece(row, place_of(i), a.V, f[k]);
    }
#pragma unroll
    for (int k = 0; k < kTogether; ++k) {
      const int i = i0 + k * kWaves;
      if (i < count) keep(f[k], place_of(i), lane < kLanes);
    }
  }
  __syncthreads();
  if (listed > kList) {                                   // (uniform) again, a group a wave at a time
    __syncthreads();
    if (tid == 0) listed = 0;
    __syncthreads();
#pragma unroll 1
    for (int i = 0; i < count; i += kWaves) {
      if (i + wv < count) {
        float f[N];
        if (lane < kLanes) load_piece(row, place_of(i + wv), a.V, f);
        keep(f, place_of(i + wv), lane < kLanes);
      }
      __syncthreads();
      const int have = listed;                            // (read by all in front of the next barrier: a wave that goes on adds to it)
      __syncthreads();
      if (have > kList - kWaves * 64 * N || i + kWaves >= count) {
        rank_keys(list, have, a.n_top, ranked);
        __syncthreads();
        if (tid < a.n_top) list[tid] = ranked[tid];
        if (tid == 0) listed = min(have, a.n_top);
        if (have >= a.n_top) least = ranked[a.n_top - 1];
        __syncthreads();
      }
    }
  }
  rank_keys(list, listed, a.n_top, ranked);
  __syncthreads();
  if (tid < a.n_top) {
    const u64 key = ranked[tid];
    a.top_token[static_cast<int64_t>(r) * a.n_top + tid] = key ? index_of(key) : -1;
    if (a.top_logprob) a.top_logprob[static_cast<int64_t>(r) * a.n_top + tid] = key ? logprob(of_ordered(static_cast<uint32_t>(key >> 32))) : -INFINITY;
  }
}

// parts of a row, its alignment not known
int parts_of(int V, int per_lane) { return (V + 7 + 64 * per_lane - 1) / (64 * per_lane); }

template <typename T, int EPT>
void launch_ept(const LogprobArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((k_logprob_part<T, EPT>), dim3(static_cast<unsigned>((a.parts + 3) / 4), static_cast<unsigned>(a.M)), dim3(kThreads), 0, s, a);
  hipLaunchKernelGGL((k_logprob_row<T, EPT>), dim3(static_cast<unsigned>(a.M)), dim3(kThreads), 0, s, a);
}

template <typename T>
void launch_as(const LogprobArgs& a, hipStream_t s) {
  if (a.wide) launch_ept<T, kWide>(a, s);
  else launch_ept<T, kNarrow>(a, s);
}

}  // namespace

// Few rows are cut finer, so that they fill the chip too.
constexpr int64_t kFewParts = 2048;
void logprob_plan(LogprobArgs& a) {
  a.wide = static_cast<int64_t>(a.M) * parts_of(a.V, kWide) >= kFewParts;
  a.parts = parts_of(a.V, a.wide ? kWide : kNarrow);
}

size_t logprob_carve(LogprobArgs& a, void* base) {
  // never less for more rows or a larger V: narrow parts count twice those of kFewParts at most
  const int64_t wide = static_cast<int64_t>(a.M) * parts_of(a.V, kWide), narrow = static_cast<int64_t>(a.M) * parts_of(a.V, kNarrow);
  const size_t parts = static_cast<size_t>(std::max(wide, std::min(narrow, 2 * kFewParts)));
  char* p = static_cast<char*>(base);
  a.stats = reinterpret_cast<float4*>(p);
  const size_t stats = (parts * sizeof(float4) + 255) & ~static_cast<size_t>(255);
  a.groups = reinterpret_cast<float*>(p + stats);
  return stats + (a.n_top ? (parts * 8 * sizeof(float) + 255) & ~static_cast<size_t>(255) : 0);
}

hipError_t launch_logprob(const LogprobArgs& a, hipStream_t s) {
  if (a.f32) launch_as<float>(a, s);
  else launch_as<bf16_t>(a, s);
  return hipGetLastError();
}

}  // namespace sx
