// A token per row of logits from a given uniform number: temperature, top-k, top-p, min-p, then the inverse of the kept weights'
// cumulative sum in index order.
//
// Weights are w = 2^((l - l_max) log2(e) / T), in 64-bit arithmetic (a polynomial: see weight()) and added up as 45-bit fixed-point
// numbers, so that a sum is the same whatever its order.  A weight is half a step off at most, 2^-46 of the best one's, and a border of V tokens' sums V
// times that: 2.2e-9 at V = 151936, a twenty-seventh of a step of u near 1.  Tokens below 2^-40 of the best one's weight count as none.
//
// What a filter keeps is a prefix of the tokens in the order (logit descending, index ascending).  Three launches find it without
// sorting a row; a row is cut into chunks, so that few rows fill the chip too:
//   1 k_sample_bins  one pass over the logits: a histogram of every chunk over bins of 1/16 nat of l / T (counts for top-k, else
//                    masses for top-p, else none; counted from the chunk's best, and halved as often as the span of its logits allows).
//   2 k_sample_mass  adds the row's histograms (the grids of two chunks differ by powers of two), takes the bins that the borders of top-k and top-p lie in, finds the least logits of
//                    those (a search over the keys of all floats: what follows compares logits, not weights or bins), reads the logits
//                    again: masses of what is kept for certain per segment of 512 tokens, and a list of the tokens in doubt.
//   3 k_sample_pick  a workgroup per row finds the border in the list (at most 4096), the draw's segment and in it the token.
// Rows without any difference need no border but a number.
// The slow way.  A list holds 4096 tokens, 2048 of a chunk.  What is in doubt is every token of the bins of a row's borders, and those are 1/16 nat wide as soon
// as one of the row's chunks has a token more than 8 nats (and less than 4096) below its best one; only where all chunks span less are they halved,
// up to twelve times.  The border of top-p is known to 2e-5 of the sum, so from top-p 0.99998 on everything below it is in doubt.  Rows with more tokens in
// doubt than that, and logits beyond 2^20 temperatures, are selected from whole by the third kernel, with equal results: 0.42 to 0.49 ms for 151936
// fp32 logits, 0.71 to 0.82 for 262144, whether of one row or 144.  That happens in earnest (top-p alone, microseconds of 1 row and of 144, not 25 to 75):
//   151936 logits, a head's rows, top-p 0.9999: 30 and 488; from 0.99997 on 430 and 488    a flat body (deviation 0.3 or 0.5) and one token 10 above: 430, 480
//   262144 logits of deviation 1 and more, top-p 0.9: 710, 800 (deviation 0.9: 42, and 777 where one of the 144 rows is taken so); 144 rows of 151936 of deviation 1.4, top-p 0.95: 460
// What bounds it: 144 rows of 151936 fp32 logits (87.5 MB, 16.6 us at a copy's rate) take 21 us in the first kernel (4.2 TB/s), 34 in the
// second (vector instructions, 86 % of its time: fifteen in 64 bits and as many others for a token's weight) and 12 in the third; 7 rows with
// top-k 4.5, 8 and 6.4 us: chains of dependent loads, five in the last.  One pass that kept every weight would write as much as it reads.
#include "common.hpp"
#include "kernels.hpp"

#include <limits.h>
#include <algorithm>
#include <type_traits>

namespace sx {

namespace {

constexpr int kT = 512;                 // threads of a workgroup
constexpr int kWaves = kT / 64;
constexpr int kSeg = 512;               // tokens of a segment (a wave's step; a workgroup's in the last kernel)
constexpr int kBins = 512;              // bins of a histogram: 32 nats
constexpr float kPerNat = 16.f;
static_assert(kBins == kT, "a thread per bin");
constexpr int kFinest = 12;             // bins are 1/16 nat to 2^-16 nat
constexpr float kWide = 128.f;          // a row whose logits span that many bins has no finer ones
constexpr int kChunkSegs = 64;          // segments of a chunk, at most
constexpr int kList = 4096, kListPart = 2048;      // tokens in doubt of a row, and of one of its chunks
constexpr int kFar = 1 << 24;           // bins are forced into -kFar .. kFar: a product within them is off by half a bin at most
constexpr double kFix = 35184372088832.0;          // 2^45
constexpr double kFloor = 9.094947017729282e-13;   // 2^-40

enum { kModeEmpty = 0, kModeAll = 1, kModeTopK = 2, kModeTopP = 3, kModeScan = 4, kModeEqual = 5 };

// A row's settings, forced into range.
struct Setting {
  int k;             // 0: off
  float s;           // bins per logit
  double c;          // log2(e) / T
  double p, m;       // top-p (1: off), min-p
};
__device__ __forceinline__ Setting setting_of(const SampleArgs& a, int row) {
  const int i = row / a.rows_per_seq;
  float T = a.temperature ? a.temperature[i] : 1.f;
  const float p = a.top_p ? a.top_p[i] : 1.f, m = a.min_p ? a.min_p[i] : 0.f;
  int k = a.top_k ? a.top_k[i] : 0;
  Setting s;
  if (k < 0 || k >= a.V) k = 0;
  if (k > kSampleMaxK) {
    report_status(a.status, kStatusBadSetting);
    k = kSampleMaxK;
  }
  if (!(T >= 9.765625e-4f)) { k = 1; T = 1.f; }         // greedy
  T = fminf(T, 7.9228163e28f);
  s.k = k;
  s.s = kPerNat / T;
  s.c = 1.4426950408889634 / static_cast<double>(T);
  s.p = p < 1.f ? fmaxf(p, 0.f) : 1.0;                   // (NaN: off)
  s.m = fmax(fmin(static_cast<double>(m), 1.0), kFloor); // (NaN: off)
  if (m != m) s.m = kFloor;
  return s;
}

__device__ __forceinline__ int bin_of(float l, float s) { return static_cast<int>(floorf(fminf(fmaxf(l * s, -static_cast<float>(kFar)), static_cast<float>(kFar)))); }

// order of the logits as unsigned numbers, and a token's place: better tokens have smaller ones
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t u = __float_as_uint(l);
  return u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key ^ ((key >> 31) - 1u | 0x80000000u)); }
__device__ __forceinline__ uint64_t place_of(float l, int idx) { return static_cast<uint64_t>(~key_of(l)) << 32 | static_cast<uint32_t>(idx); }

// The least logit that `reached` holds for (it has to hold from some logit on): by six bits of its key at a time, a lane per candidate.
template <typename F> __device__ __forceinline__ float least_of(F reached) {
  uint32_t key = 0;
#pragma unroll 1
  for (int shift = 26; shift >= -4; shift -= 6) {
    const int by = shift < 0 ? 0 : shift, width = shift < 0 ? 4 : 64;          // (32 bits: five times six, and two)
    const uint32_t lane = threadIdx.x & 63;
    const uint32_t mine = key + (lane << by);
    // (keys of NaN lie below -infinity's and above infinity's)
    const bool below = static_cast<int>(lane) < width && (mine < 0x007FFFFFu || (mine <= 0xFF800000u && !reached(logit_of(mine))));
    const int n = __popcll(__builtin_amdgcn_ballot_w64(below));
    key += shift < 0 ? static_cast<uint32_t>(n) : static_cast<uint32_t>(n > 0 ? n - 1 : 0) << by;
  }
  return logit_of(key);
}

// 2^t, |t| < 1000: 2^f for |f| <= 1/2 by a polynomial of degree 9 through its values at Chebyshev's points, 3.2e-14 off at most.
__device__ __forceinline__ double exp2_of(double t) {
  const double n = rint(t), f = t - n;
  double y = 1.0205905413765595e-07;
  y = fma(y, f, 1.325964524488711e-06);
  y = fma(y, f, 1.5252672924850737e-05);
  y = fma(y, f, 0.0001540343375125101);
  y = fma(y, f, 0.0013333558200794592);
  y = fma(y, f, 0.009618129193934313);
  y = fma(y, f, 0.05550410866465167);
  y = fma(y, f, 0.2402265069564034);
  y = fma(y, f, 0.6931471805599462);
  y = fma(y, f, 1.0);
  return __longlong_as_double(__double_as_longlong(y) + (static_cast<int64_t>(static_cast<int>(n)) << 52));
}
// a weight in units of 2^-45, rounded, on top of the bits of 2^52
constexpr uint64_t kBias = 0x4330000000000000ull;
__device__ __forceinline__ uint64_t biased(double w) { return static_cast<uint64_t>(__double_as_longlong(fma(w, kFix, 4503599627370496.0))); }
// The weights of a row whose best logit is finite: 2^(l c - top c) with one rounding of the exponent (that of top c is the same for every token);
// l from top - 1600 / s on, whose weight of 2^-144 is no unit.
struct Scale {
  double c, k;
};
__device__ __forceinline__ double weight(float l, const Scale& z) { return exp2_of(fma(static_cast<double>(l), z.c, -z.k)); }
__device__ __forceinline__ uint64_t fixed(double w) { return biased(w) - kBias; }
// The same for any row, as it is needed where infinities may meet: 0 below 2^-40.
__device__ __forceinline__ double weight_far(float l, float top, double c) {
  const double d = l == top ? 0.0 : static_cast<double>(l) - static_cast<double>(top);
  const double w = exp2_of(fmax(d * c, -64.0));
  return w >= kFloor ? w : 0.0;
}

// Values of other lanes without LDS (as wave_scan): 0 where there is no such lane.
template <int CTRL, int ROWS> __device__ __forceinline__ uint64_t lane64(uint64_t v) {
  const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(static_cast<uint32_t>(v)), CTRL, ROWS, 0xf, false));
  const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(static_cast<uint32_t>(v >> 32)), CTRL, ROWS, 0xf, false));
  return static_cast<uint64_t>(hi) << 32 | lo;
}
__device__ __forceinline__ uint64_t wave_scan64(uint64_t v) {
  v += lane64<0x111, 0xf>(v);
  v += lane64<0x112, 0xf>(v);
  v += lane64<0x114, 0xf>(v);
  v += lane64<0x118, 0xf>(v);
  v += lane64<0x142, 0xa>(v);
  v += lane64<0x143, 0xc>(v);
  return v;
}
__device__ __forceinline__ double wave_scan64(double v) {
  auto lanes = [](double x, auto f) { return __longlong_as_double(static_cast<long long>(f(static_cast<uint64_t>(__double_as_longlong(x))))); };
  v += lanes(v, [](uint64_t x) { return lane64<0x111, 0xf>(x); });
  v += lanes(v, [](uint64_t x) { return lane64<0x112, 0xf>(x); });
  v += lanes(v, [](uint64_t x) { return lane64<0x114, 0xf>(x); });
  v += lanes(v, [](uint64_t x) { return lane64<0x118, 0xf>(x); });
  v += lanes(v, [](uint64_t x) { return lane64<0x142, 0xa>(x); });
  v += lanes(v, [](uint64_t x) { return lane64<0x143, 0xc>(x); });
  return v;
}
__device__ __forceinline__ uint64_t shfl_xor64(uint64_t v, int m) {
  return static_cast<uint64_t>(static_cast<uint32_t>(__shfl_xor(static_cast<int>(static_cast<uint32_t>(v >> 32)), m))) << 32 | static_cast<uint32_t>(__shfl_xor(static_cast<int>(static_cast<uint32_t>(v)), m));
}
// (uniform)
__device__ __forceinline__ uint64_t wave_sum64(uint64_t v) {
  v = wave_scan64(v);
  return static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(static_cast<uint32_t>(v >> 32)), 63))) << 32 |
         static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(static_cast<uint32_t>(v)), 63));
}
// (in lane 63)
__device__ __forceinline__ uint64_t wave_max64(uint64_t v) {
  v = max(v, lane64<0x111, 0xf>(v));
  v = max(v, lane64<0x112, 0xf>(v));
  v = max(v, lane64<0x114, 0xf>(v));
  v = max(v, lane64<0x118, 0xf>(v));
  v = max(v, lane64<0x142, 0xa>(v));
  v = max(v, lane64<0x143, 0xc>(v));
  return v;
}
// inclusive sum over the workgroup; `part` [kWaves] is free again behind the next barrier
__device__ __forceinline__ uint64_t block_scan64(uint64_t v, uint64_t* part) {
  const int wv = threadIdx.x >> 6;
  v = wave_scan64(v);
  if ((threadIdx.x & 63) == 63) part[wv] = v;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWaves; ++i) v += i < wv ? part[i] : 0;
  return v;
}

__device__ __forceinline__ float as_f32(float v) { return v; }
__device__ __forceinline__ float as_f32(bf16_t v) { return bf16_to_f32(v); }
__device__ __forceinline__ float value(float v) { return v == v ? v + 0.f : -INFINITY; }       // (-0 is 0, NaN is never drawn)

// eight tokens of a lane as they are (NaN too, which no comparison holds for): an instruction of the wave reads consecutive bytes
template <typename T> __device__ __forceinline__ int token_of(int seg, int lane, int e) {
  return sizeof(T) == 4 ? seg * kSeg + 256 * (e >> 2) + 4 * lane + (e & 3) : seg * kSeg + 8 * lane + e;
}
template <typename T> __device__ __forceinline__ void load_seg(const T* row, int V, int seg, float (&x)[8]) {
  const int lane = threadIdx.x & 63;
  T raw[8];
  if ((seg + 1) * kSeg <= V) {
    // (as bytes: a row may begin at any element)
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) __builtin_memcpy(raw + i * (16 / sizeof(T)), row + token_of<T>(seg, lane, i * (16 / static_cast<int>(sizeof(T)))), 16);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = as_f32(raw[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = token_of<T>(seg, lane, e);
      x[e] = i < V ? as_f32(row[i]) : -INFINITY;
    }
  }
}

// Halvings of the bins, up to kFinest, that leave the logits low .. top within kBins of them (their products rounded), and their numbers below kFar.
__device__ __forceinline__ int finer_of(float top, float low, float s) {
  const float span = top > -INFINITY ? (top - low) * s : static_cast<float>(kBins);            // (NaN where they are infinite: no halving either way)
  return max(0, min(min(ilogbf(508.f / fmaxf(span, 0.0625f)), ilogbf(static_cast<float>(kFar) / fmaxf(fabsf(top * s), 1.f))), kFinest));
}

// ------------------------------------------------------------------------------------------------------------ 1: histograms

template <typename T>
__global__ __launch_bounds__(kT) void k_sample_bins(const SampleArgs a) {
  __shared__ uint4 hist[kBins];        // four copies of a bin: the lanes of a wave that meet in a bin add one after the other (64-bit sums in
                                       // one copy, counts and masses together, took 28.7 us for the 144 rows)
  __shared__ float best[kWaves], lowest[kWaves];
  __shared__ int wide;
  const int row = blockIdx.y, chunk = blockIdx.x, lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const T* logits = static_cast<const T*>(a.logits) + static_cast<int64_t>(row) * a.ld;
  const int seg0 = chunk * a.chunk_segs, seg1 = min(seg0 + a.chunk_segs, a.segs);
  constexpr int N = kChunkSegs / kWaves;
  float x[N][8], top = -INFINITY;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int seg = seg0 + wv + i * kWaves;
    if (seg < seg1) {
      load_seg<T>(logits, a.V, seg, x[i]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] = -INFINITY;
    }
  }
  const Setting st = setting_of(a, row);
  for (int j = threadIdx.x; j < kBins; j += kT) hist[j] = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, x[i][e]);
  top = wave_max_dpp(top);
  if (lane == 0) best[wv] = top;
  if (threadIdx.x == 0) wide = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, best[w]);
  const bool counts = st.k > 0, masses = !counts && st.p < 1.0;        // what the borders need
  if (!counts && !masses) {
    if (threadIdx.x == 0) {
      a.chunk_top[static_cast<size_t>(row) * a.chunks + chunk] = make_float4(top, top, 0.f, 0.f);
      if (chunk == 0) a.row_info[row].listed = 0;
    }
    return;                            // uniform
  }
  // Rows whose logits lie close together get finer bins, 2^finer of them in 1/16 nat: as fine as the span of what weighs anything allows
  // (with bins of 1/16 nat only, top-p of 151936 logits of spread 0.3 left 7600 tokens in doubt: 518 us a row in place of 27).
  // (an eighth of the tokens is enough to tell that a row is wide; 4096 nats away are masked ones)
  bool far = false;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float d = (top - x[i][0]) * st.s;
    far |= d >= kWide && d < 4096.f * kPerNat;
  }
  if (__builtin_amdgcn_ballot_w64(far) != 0ull && lane == 0) wide = 1;
  __syncthreads();
  int finer = 0;
  float low = -INFINITY;
  if (!wide && top > -INFINITY) {      // uniform
    low = top;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) low = (top - x[i][e]) * st.s < static_cast<float>(kBins) ? fminf(low, x[i][e]) : low;
    low = -wave_max_dpp(-low);
    if (lane == 0) lowest[wv] = low;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) low = fminf(low, lowest[w]);
    finer = finer_of(top, low, st.s);
  }
  const float s = ldexpf(st.s, finer), step = ldexpf(-1.44269504f / kPerNat, -finer);
  // (whole numbers below kFar, or the row goes another way: their differences are exact)
  const float origin = floorf(top * s);
  uint32_t* const mine = reinterpret_cast<uint32_t*>(hist) + (lane & 3);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (seg0 + wv + i * kWaves >= seg1) break;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float l = x[i][e], prod = l * s, g = floorf(prod), j = origin - g;
      if (j < static_cast<float>(kBins)) {
        uint32_t add = 1;
        if (masses) {                  // uniform
          // how far below the bin's upper edge, in bins: the product's rounding error counts as well, and may be half a bin either way
          const float below = fminf(fmaxf((g - prod) + 1.f - fmaf(l, s, -prod), -1.f), 2.f);
          add = static_cast<uint32_t>(fmaf(__builtin_amdgcn_exp2f(below * step), 65536.f, 0.5f));
        }
        atomicAdd(&mine[4 * static_cast<int>(j)], add);
      }
    }
  }
  __syncthreads();
  const size_t at = static_cast<size_t>(row) * a.chunks + chunk;
  for (int j = threadIdx.x; j < kBins; j += kT) {
    const uint4 h = hist[j];
    a.hist[at * kBins + j] = h.x + h.y + h.z + h.w;
  }
  if (threadIdx.x == 0) {
    a.chunk_top[at] = make_float4(top, low, static_cast<float>(finer), 0.f);
    if (chunk == 0) a.row_info[row].listed = 0;
  }
}

// ------------------------------------------------------------------------------------------------------------ 2: masses and the list

template <typename T>
__global__ __launch_bounds__(kT) void k_sample_mass(const SampleArgs a) {
  __shared__ int cnt_part[kWaves], found[3], n_list, base_list;
  __shared__ double mass_part[kWaves];
  __shared__ float borders[4];
  __shared__ unsigned long long sums[2], merged[kBins];
  __shared__ uint2 list[kListPart];
  const int row = blockIdx.y, chunk = blockIdx.x, lane = threadIdx.x & 63, tid = threadIdx.x;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const T* logits = static_cast<const T*>(a.logits) + static_cast<int64_t>(row) * a.ld;
  const int seg0 = chunk * a.chunk_segs, seg1 = min(seg0 + a.chunk_segs, a.segs);
  float next[8];                                  // (the first tokens are requested with everything else)
  if (seg0 + wv < seg1) load_seg<T>(logits, a.V, seg0 + wv, next);
  const size_t first = static_cast<size_t>(row) * a.chunks;
  const float4 chunk_at = lane < a.chunks ? a.chunk_top[first + lane] : make_float4(-INFINITY, -INFINITY, 0.f, 0.f);
  const float chunk_top = chunk_at.x;
  const Setting st = setting_of(a, row);
  // ---- the row's best logit and its histogram: thread j has bin j, lane c how far chunk c's bins lie behind it
  const float top = wave_max_dpp(chunk_top);
  // (bins as wide as the chunk with the widest ones has them, and as the span of the whole row wants them: those of the others are halves,
  // quarters, .. of them.  Chunks without a token within 32 nats do not count.)
  const bool counts = chunk_top > -INFINITY && (top - chunk_top) * st.s < static_cast<float>(kBins);
  int finer = 0;
  bool equal = false;                             // all tokens that weigh anything are equal (a row of zeros)
  if (__builtin_amdgcn_ballot_w64(counts && chunk_at.z == 0.f) == 0ull) {
    const float low = -wave_max_dpp(counts ? -chunk_at.y : -INFINITY);
    finer = min(finer_of(top, low, st.s), static_cast<int>(-wave_max_dpp(counts ? -chunk_at.z : -static_cast<float>(kFinest))));
    equal = low == top;
  }
  const float s = ldexpf(st.s, finer);
  const int origin = bin_of(top, s);
  const int split = counts ? static_cast<int>(chunk_at.z) - finer : 0;
  const int chunk_origin = bin_of(chunk_top, ldexpf(s, split));
  const int behind = counts ? origin - chunk_origin : kBins;      // (where the grids are the same)
  const bool same = __builtin_amdgcn_ballot_w64(split != 0) == 0ull;
  if (tid < 3) found[tid] = kBins - 1;
  if (tid == 0) n_list = 0;
  if (tid < 2) sums[tid] = 0;
  const int mode = top == -INFINITY ? kModeEmpty : origin >= kFar || origin <= kBins - kFar ? kModeScan : equal ? kModeEqual : st.k > 0 ? kModeTopK : st.p < 1.0 ? kModeTopP : kModeAll;
  const float bottom = top - 100.f * kPerNat / st.s;
  const Scale z = {st.c, static_cast<double>(top) * st.c};
  if (mode == kModeTopK || mode == kModeTopP) {
    uint64_t h = 0;                               // (sums of 2^18 tokens' 2^16)
    double unit = 1.0;
    if (!same) {
      // bins of finer grids, thread j the j-th of every chunk: their counts, or masses below the upper edge of the bin they lie in, are added there
      merged[tid] = 0;
      __syncthreads();
      for (int c = 0; c < a.chunks; ++c) {
        const int by = __builtin_amdgcn_readlane(split, c);
        const int fine = __builtin_amdgcn_readlane(chunk_origin, c) - tid, at = origin - (fine >> by);
        const uint32_t v = __builtin_amdgcn_readlane(static_cast<int>(counts), c) != 0 ? a.hist[(first + c) * kBins + tid] : 0;
        if (v == 0 || at >= kBins) continue;
        uint64_t add = v;
        if (mode == kModeTopP) {
          const int under = (1 << by) - 1 - (fine & ((1 << by) - 1));
          add = static_cast<uint64_t>(static_cast<double>(v) * static_cast<double>(exp2f(static_cast<float>(under) * ldexpf(-1.44269504f / kPerNat, -finer - by))) * 1024.0);
        }
        atomicAdd(&merged[at], static_cast<unsigned long long>(add));
      }
      __syncthreads();
      h = merged[tid];
      if (mode == kModeTopP) unit = 1.0 / 1024.0;
    }
    for (int c0 = 0; same && c0 < a.chunks; c0 += kSampleMaxChunks / 2) {      // (half of the loads in flight: the second half is often empty)
      uint32_t v[kSampleMaxChunks / 2];
      const uint32_t* const hist = a.hist + (first + c0) * kBins;
#pragma unroll
      for (int e = 0; e < kSampleMaxChunks / 2; ++e) {
        v[e] = 0;
        if (c0 + e < a.chunks) {                  // uniform
          const int at = tid - __builtin_amdgcn_readlane(behind, c0 + e);
          if (at >= 0) v[e] = hist[e * kBins + at];
        }
      }
#pragma unroll
      for (int e = 0; e < kSampleMaxChunks / 2; ++e) h += v[e];
    }
    auto first_of = [&](bool reached, int which) {
      const uint64_t m = __builtin_amdgcn_ballot_w64(reached);
      if (m && lane == 0) atomicMin(&found[which], 64 * wv + __ffsll(static_cast<unsigned long long>(m)) - 1);
    };
    // the bins of the borders: the first whose sum reaches them; of top-p those that 2e-5 more or less could make it (a bin's mass is
    // known to some 1e-5: half a unit of 2^-16, T in 32 bits, roundings of the exponentials)
    if (mode == kModeTopK) {
      int cum = wave_scan(static_cast<int>(h));
      if (lane == 63) cnt_part[wv] = cum;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kWaves; ++w) cum += w < wv ? cnt_part[w] : 0;
      first_of(cum >= st.k, 0);
    } else {
      double cum = wave_scan64(unit * static_cast<double>(h) * static_cast<double>(exp2f(static_cast<float>(tid) * ldexpf(-1.44269504f / kPerNat, -finer)))), all = 0.0;
      if (lane == 63) mass_part[wv] = cum;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        cum += w < wv ? mass_part[w] : 0.0;
        all += mass_part[w];
      }
      first_of(cum >= st.p * all * (1.0 - 2e-5), 1);
      first_of(cum >= st.p * all * (1.0 + 2e-5), 2);
    }
    __syncthreads();
  }
  // logits from `sure` on are kept for certain, from `doubt` on the list decides; those below `least` count as none, those below `min_p` are not kept
  if (mode != kModeEmpty && mode != kModeScan) {
    if (wv == 0) {
      const int bin = origin - (mode == kModeTopK ? found[0] : max(found[1], found[2]));
      const float v = mode != kModeTopK && mode != kModeTopP ? NAN : least_of([&](float l) { return bin_of(l, s) >= bin; });
      if (lane == 0) borders[0] = v;
    } else if (wv == 1) {
      const int bin = origin - found[1] + 1;
      const float v = mode != kModeTopP || found[1] == 0 ? NAN : least_of([&](float l) { return bin_of(l, s) >= bin; });
      if (lane == 0) borders[1] = v;
    } else if (wv == 2) {
      const float v = least_of([&](float l) { return l >= top || weight(fmaxf(l, bottom), z) >= kFloor; });
      if (lane == 0) borders[2] = v;
    } else if (wv == 3) {
      const float v = least_of([&](float l) { return l >= top || weight(fmaxf(l, bottom), z) >= st.m; });
      if (lane == 0) borders[3] = v;
    }
  }
  __syncthreads();
  const float doubt = borders[0], least = borders[2], min_p = borders[3], sure = mode == kModeAll || mode == kModeEqual ? min_p : borders[1];
  if (chunk == 0 && tid == 0) {
    SampleRow& r = a.row_info[row];
    r.mode = mode;
    r.top = top;
    r.sure = sure;
    r.doubt = doubt;
    r.least = least;
    r.min_p = min_p;
  }
  if (mode == kModeEmpty || mode == kModeScan) return;       // uniform
  // ---- the chunk's tokens
  uint64_t total = 0, above = 0;
  auto tokens = [&](auto weighed, auto apart) {    // are weights needed, and those above `sure` apart from those that are kept
    const float keep = apart ? min_p : sure;
    for (int seg = seg0 + wv; seg < seg1; seg += kWaves) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = next[e];
      if (seg + kWaves < seg1) load_seg<T>(logits, a.V, seg + kWaves, next);
      if (weighed) {
        uint64_t kept = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint64_t f = biased(weight(x[e] >= least ? x[e] : bottom, z));
          total += f;
          if (apart) above += x[e] >= sure ? f : kBias;
          kept += x[e] >= keep ? f : kBias;
        }
        kept -= 8 * kBias;
        if (!apart) above += kept;
        kept = wave_sum64(kept);
        if (lane == 0) a.seg_mass[static_cast<size_t>(row) * a.segs + seg] = kept;
        total -= 8 * kBias;
        if (apart) above -= 8 * kBias;
      }
      uint64_t in_doubt[8];
      int found_here = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        in_doubt[e] = __builtin_amdgcn_ballot_w64(x[e] >= doubt) & ~__builtin_amdgcn_ballot_w64(x[e] >= sure);
        found_here += __popcll(in_doubt[e]);
      }
      if (found_here) {                            // uniform
        int at = 0;
        if (lane == 0) at = atomicAdd(&n_list, found_here);
        at = __builtin_amdgcn_readfirstlane(at);
        if (at + found_here <= kListPart) {        // (as they are: their places follow when the list is written)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (in_doubt[e]) {                     // uniform
              const uint32_t mine = __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(in_doubt[e] >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(in_doubt[e]), static_cast<uint32_t>(at)));
              if (__builtin_amdgcn_inverse_ballot_w64(in_doubt[e])) list[mine] = make_uint2(__float_as_uint(x[e]), static_cast<uint32_t>(token_of<T>(seg, lane, e)));
              at += __popcll(in_doubt[e]);
            }
        }
      }
    }
  };
  if (mode == kModeTopK) tokens(std::false_type{}, std::false_type{});
  else if (!(min_p > sure)) tokens(std::true_type{}, std::false_type{});
  else tokens(std::true_type{}, std::true_type{});
  if (mode == kModeTopP) {
    total = wave_sum64(total);
    above = wave_sum64(above);
    if (lane == 0) {
      atomicAdd(&sums[0], total);
      atomicAdd(&sums[1], above);
    }
  }
  __syncthreads();
  if (tid == 0) {
    a.chunk_sums[2 * (first + chunk)] = sums[0];
    a.chunk_sums[2 * (first + chunk) + 1] = sums[1];
    // (a list that does not fit is counted as too long, and the last kernel does without it)
    base_list = n_list > 0 ? atomicAdd(&a.row_info[row].listed, n_list <= kListPart ? n_list : kList + 1) : 0;
  }
  __syncthreads();
  if (n_list <= kListPart)
    for (int i = tid; i < n_list; i += kT)
      if (base_list + i < kList) a.list[static_cast<size_t>(row) * kList + base_list + i] = place_of(value(__uint_as_float(list[i].x)), static_cast<int>(list[i].y));
}

// ------------------------------------------------------------------------------------------------------------ 3: the draw

constexpr int kPairs = kT / 4;          // tokens of a list that is compared pair by pair: both borders at once, in place of two selections of two or
                                        // three rounds with six meetings of the workgroup each (7 rows with top-k 20 to 50: 9.8 -> 6.4 us)
struct PickLds {
  uint64_t list[kList];
  uint64_t w[kList];                 // the list's weights
  uint64_t seg[kSampleMaxSegs];
  uint64_t part[kWaves], part2[kWaves];
  unsigned long long digit_mass[256], wide;
  uint32_t digit_count[256];
  int count[kSampleMaxSegs];
  int pick, seg_at, digit, last;
  uint64_t seg_before, cut;
  // results of a round of a selection
  uint32_t key;
  int n_equal;
  uint32_t before;
  uint64_t mass_before;
};

// All segments of a row, four of a wave requested together: f(segment, its tokens of the lane).
template <typename T, typename F> __device__ __forceinline__ void each_seg(const SampleArgs& a, const T* logits, F f) {
  constexpr int kAhead = 4;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int seg = wv; seg < a.segs; seg += kAhead * kWaves) {
    float x[kAhead][8];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (seg + i * kWaves < a.segs) load_seg<T>(logits, a.V, seg + i * kWaves, x[i]);
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (seg + i * kWaves < a.segs) f(seg + i * kWaves, x[i]);
  }
}

// The token at the end of the best `want` ones (by count), or of those whose better ones sum to less than `target`: its key, how many of its equals belong to them, and
// their mass.  Radix selection over the whole row, eight bits at a time.  The workgroup's threads all get the results.
struct Border {
  uint32_t key;
  int equal;             // equals that are kept
  uint64_t mass;         // of everything kept
};
template <typename T>
__device__ Border scan_border(const SampleArgs& a, const T* logits, const Setting& st, float top, PickLds& s, int want, double target) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  uint32_t prefix = 0, before = 0;
  uint64_t mass_before = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) { s.digit_mass[tid] = 0; s.digit_count[tid] = 0; }
    __syncthreads();
    each_seg<T>(a, logits, [&](int, const float (&x)[8]) {
#pragma unroll 1
      for (int e = 0; e < 8; ++e) {
        const uint32_t key = key_of(value(x[e])), d = key >> shift & 255u;
        const double w = weight_far(value(x[e]), top, st.c);
        const bool in = w > 0.0 && !(shift < 24 && key >> (shift + 8) != prefix);
        const uint64_t m = __builtin_amdgcn_ballot_w64(in);
        if (m == 0ull) continue;                  // uniform
        const uint32_t d0 = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(d), __ffsll(static_cast<unsigned long long>(m)) - 1));
        if (__builtin_amdgcn_ballot_w64(in && d != d0) == 0ull) {      // (equal tokens by the thousand are what leads here)
          const uint64_t sum = wave_sum64(in ? fixed(w) : 0);
          if (lane == 0) {
            atomicAdd(&s.digit_count[d0], static_cast<uint32_t>(__popcll(m)));
            atomicAdd(&s.digit_mass[d0], static_cast<unsigned long long>(sum));
          }
        } else if (in) {
          atomicAdd(&s.digit_count[d], 1u);
          atomicAdd(&s.digit_mass[d], static_cast<unsigned long long>(fixed(w)));
        }
      }
    });
    __syncthreads();
    // sums from the highest digit on: waves 0..3
    int c = 0, cum = 0;
    uint64_t m = 0, cmass = 0;
    if (tid < 256) {
      c = static_cast<int>(s.digit_count[255 - tid]);
      m = s.digit_mass[255 - tid];
      cum = wave_scan(c);
      cmass = wave_scan64(m);
      if (lane == 63) { s.count[wv] = cum; s.part[wv] = cmass; }
    }
    if (tid == 0) { s.digit = 256; s.last = 0; }
    __syncthreads();
    if (tid < 256) {
#pragma unroll
      for (int w = 0; w < 3; ++w)
        if (w < wv) { cum += s.count[w]; cmass += s.part[w]; }
      const bool reached = c > 0 && (want > 0 ? before + cum >= static_cast<uint32_t>(want) : static_cast<double>(mass_before + cmass) >= target);
      const uint64_t r = __builtin_amdgcn_ballot_w64(reached), any = __builtin_amdgcn_ballot_w64(c > 0);
      if (r && lane == 0) atomicMin(&s.digit, 64 * wv + __ffsll(static_cast<unsigned long long>(r)) - 1);
      if (any && lane == 0) atomicMax(&s.last, 64 * wv + 63 - __clzll(static_cast<long long>(any)));
    }
    __syncthreads();
    if (tid == (s.digit < 256 ? s.digit : s.last)) {           // (the lowest digit there is, if the border is not reached)
      s.key = prefix << 8 | static_cast<uint32_t>(255 - tid);
      s.n_equal = c;
      s.before = before + static_cast<uint32_t>(cum - c);
      s.mass_before = mass_before + (cmass - m);
    }
    __syncthreads();
    prefix = s.key;
    before = s.before;
    mass_before = s.mass_before;
  }
  const uint64_t w = fixed(weight_far(logit_of(prefix), top, st.c));
  int c = s.n_equal;
  if (want > 0) {
    c = min(c, want - static_cast<int>(before));
  } else if (w > 0) {
    // equal j of them is kept where mass_before + j w < target
    const double room = (target - static_cast<double>(mass_before)) / static_cast<double>(w);
    int n = room < static_cast<double>(c) ? max(static_cast<int>(ceil(room)), 0) : c;
    if (n > 0 && !(static_cast<double>(mass_before + static_cast<uint64_t>(n - 1) * w) < target)) --n;
    else if (n < c && static_cast<double>(mass_before + static_cast<uint64_t>(n) * w) < target) ++n;
    c = n;
  }
  __syncthreads();
  return {prefix, c, mass_before + static_cast<uint64_t>(c) * w};
}

// The place of the last kept token of the list: the want-th best (want > 0), or the last whose better ones sum to less than `target` on top of
// `base`; ~0 where all are kept, 0 where none is.  Radix selection by eight bits of the places at a time, from the highest that differ; it ends
// with the first digit that holds a single token.  All threads get the result.
__device__ uint64_t list_border(PickLds& s, int n, int want, uint64_t base, double target) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (n == 0) return 0;
  if (want <= 0) {
    target = fmax(target, 1.0);                   // (a weight is 32 units at least: the best token is always kept)
    if (static_cast<double>(base) >= target) return 0;
  }
  uint64_t least = 0, most = 0;                   // (of the complements: 0 is what lanes that are not there give)
  for (int i = tid; i < n; i += kT) {
    least = max(least, ~s.list[i]);
    most = max(most, s.list[i]);
  }
  least = wave_max64(least);
  most = wave_max64(most);
  if (lane == 63) { s.part[wv] = least; s.part2[wv] = most; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    least = max(least, s.part[w]);
    most = max(most, s.part2[w]);
  }
  uint64_t lo = ~least;
  int shift = max(0, 56 - __clzll(static_cast<long long>(most - lo)));
  uint32_t before = 0;
  uint64_t mass_before = base;
  for (;;) {
    __syncthreads();
    if (tid < 256) { s.digit_mass[tid] = 0; s.digit_count[tid] = 0; }
    if (tid == 0) s.digit = 256;
    __syncthreads();
    for (int i = tid; i < n; i += kT) {
      const uint64_t d = (s.list[i] - lo) >> shift;
      if (s.list[i] >= lo && d < 256) {
        atomicAdd(&s.digit_count[d], 1u);
        if (want <= 0) atomicAdd(&s.digit_mass[d], static_cast<unsigned long long>(s.w[i]));
      }
    }
    __syncthreads();
    // inclusive sums over the digits: waves 0..3
    int c = 0, cum = 0;
    uint64_t m = 0, cmass = 0;
    if (tid < 256) {
      c = static_cast<int>(s.digit_count[tid]);
      m = s.digit_mass[tid];
      cum = wave_scan(c);
      cmass = wave_scan64(m);
      if (lane == 63) { s.count[wv] = cum; s.part[wv] = cmass; }
    }
    __syncthreads();
    if (tid < 256) {
#pragma unroll
      for (int w = 0; w < 3; ++w)
        if (w < wv) { cum += s.count[w]; cmass += s.part[w]; }
      const bool reached = want > 0 ? before + cum >= static_cast<uint32_t>(want) : static_cast<double>(mass_before + cmass) >= target;
      const uint64_t r = __builtin_amdgcn_ballot_w64(reached);
      if (r && lane == 0) atomicMin(&s.digit, 64 * wv + __ffsll(static_cast<unsigned long long>(r)) - 1);
    }
    __syncthreads();
    const int d = s.digit;
    if (d == 256) return ~0ull;                   // (only in the first round: the border is not reached)
    if (tid == d) {
      s.n_equal = c;
      s.before = before + static_cast<uint32_t>(cum - c);
      s.mass_before = mass_before + (cmass - m);
    }
    __syncthreads();
    lo += static_cast<uint64_t>(d) << shift;
    if (shift == 0) return lo;
    if (s.n_equal == 1) {
      for (int i = tid; i < n; i += kT)
        if (s.list[i] >= lo && (s.list[i] - lo) >> shift == 0) s.cut = s.list[i];
      __syncthreads();
      return s.cut;
    }
    before = s.before;
    mass_before = s.mass_before;
    shift = max(0, shift - 8);
  }
}

// The same for a short list, of both borders at once (k > 0: `total` is of no account): every place against every other, four threads to one.
__device__ uint64_t pairs_border(PickLds& s, int n, int k, double p, uint64_t base, uint64_t total) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i = tid >> 2;
  const uint64_t mine = i < n ? s.list[i] : 0, w = i < n ? s.w[i] : 0;
  int rank = 0;
  uint64_t better = 0;
  for (int j = tid & 3; j < n; j += 4) {
    const bool b = s.list[j] < mine;
    rank += b ? 1 : 0;
    better += b ? s.w[j] : 0;
  }
  rank += __shfl_xor(rank, 1);
  rank += __shfl_xor(rank, 2);
  better += shfl_xor64(better, 1);
  better += shfl_xor64(better, 2);
  bool kept = i < n;
  if (k > 0) {
    kept = kept && rank < k;
    if (p < 1.0) {
      const uint64_t sum = wave_sum64(kept && (tid & 3) == 0 ? w : 0);
      if (lane == 0) s.part[wv] = sum;
      __syncthreads();
      total = 0;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) total += s.part[v];
    }
  }
  if (p < 1.0) kept = kept && static_cast<double>(base + better) < fmax(p * static_cast<double>(total), 1.0);
  const uint64_t last = wave_max64(kept ? mine : 0);
  if (lane == 63) s.part2[wv] = last;
  __syncthreads();
  uint64_t cut = 0;
#pragma unroll
  for (int v = 0; v < kWaves; ++v) cut = max(cut, s.part2[v]);
  return cut;
}

template <typename T>
__global__ __launch_bounds__(kT) void k_sample_pick(const SampleArgs a) {
  extern __shared__ uint4 smem4[];
  PickLds& s = *reinterpret_cast<PickLds*>(smem4);
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  // (what is needed in any case is requested at once)
  uint64_t early[2], seg_mass = 0, total = 0, above = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) early[i] = a.list[static_cast<size_t>(row) * kList + i * kT + tid];
  if (tid < a.segs) seg_mass = a.seg_mass[static_cast<size_t>(row) * a.segs + tid];
  if (lane < a.chunks) {
    total = a.chunk_sums[2 * (static_cast<size_t>(row) * a.chunks + lane)];
    above = a.chunk_sums[2 * (static_cast<size_t>(row) * a.chunks + lane) + 1];
  }
  const SampleRow info = a.row_info[row];
  float u = a.u[row];
  const Setting st = setting_of(a, row);
  const T* logits = static_cast<const T*>(a.logits) + static_cast<int64_t>(row) * a.ld;
  const float top = info.top;
  if (info.mode == kModeEmpty) {                  // uniform
    if (tid == 0) {
      a.token[row] = -1;
      if (a.prob) a.prob[row] = 0.f;
    }
    return;
  }
  float sure = info.sure, doubt = info.doubt;     // kept: logits from `sure` on, and from `doubt` on where the place is not behind `cut`
  uint64_t cut = ~0ull;
  const bool listed = info.mode == kModeTopK || info.mode == kModeTopP;
  const int n = listed ? info.listed : 0;
  const bool scanned = info.mode == kModeScan || n > kList;
  const Scale z = {st.c, static_cast<double>(top) * st.c};
  if (scanned) {
    // ---- without histograms and list: a row whose logits are far from anything (2^20 temperatures), or whose list is too long, as where more than 4096 tokens
    // of nearly one weight lie at the border
    sure = NAN;
    doubt = -INFINITY;
    if (st.k > 0 || st.p < 1.0) {
      Border b = {0, 0, 0};
      if (st.k > 0) b = scan_border<T>(a, logits, st, top, s, st.k, 0.0);
      if (st.p < 1.0) {
        double of = static_cast<double>(b.mass);
        if (info.mode == kModeTopP) {
          of = static_cast<double>(wave_sum64(total));
        } else if (st.k <= 0) {
          if (tid == 0) s.wide = 0;
          __syncthreads();
          uint64_t mine = 0;
          each_seg<T>(a, logits, [&](int, const float (&x)[8]) {
#pragma unroll 1
            for (int e = 0; e < 8; ++e) mine += fixed(weight_far(value(x[e]), top, st.c));
          });
          mine = wave_sum64(mine);
          if (lane == 0) atomicAdd(&s.wide, static_cast<unsigned long long>(mine));
          __syncthreads();
          of = static_cast<double>(s.wide);
        }
        const Border q = scan_border<T>(a, logits, st, top, s, 0, st.p * of);
        const bool equal = st.k > 0 && q.key == b.key;
        b = {q.key, max(equal ? min(q.equal, b.equal) : q.equal, 1), 0};
      }
      // the last of the kept equals, in index order: equals per segment, then in the segment that has it
      each_seg<T>(a, logits, [&](int seg, const float (&x)[8]) {
        int eq = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) eq += __popcll(__builtin_amdgcn_ballot_w64(x[e] > -INFINITY && key_of(value(x[e])) == b.key));
        if (lane == 0) s.count[seg] = eq;
      });
      __syncthreads();
      {
        const int c = tid < a.segs ? s.count[tid] : 0, upto = static_cast<int>(block_scan64(static_cast<uint64_t>(c), s.part));
        if (tid == 0) { s.digit = 0; s.n_equal = INT_MAX; }
        __syncthreads();
        if (upto >= b.equal && upto - c < b.equal) { s.digit = tid; s.n_equal = b.equal - (upto - c); }
        __syncthreads();
      }
      if (wv == 0) {
        int left = s.n_equal, last = INT_MAX;
        const int seg = s.digit;
        for (int r = 0; r < kSeg / 64; ++r) {
          const int i = seg * kSeg + r * 64 + lane;
          const float l = i < a.V ? value(as_f32(logits[i])) : -INFINITY;
          uint64_t eq = __builtin_amdgcn_ballot_w64(l > -INFINITY && key_of(l) == b.key);
          const int c = __popcll(eq);
          if (left > 0 && left <= c) {
            for (int q = 1; q < left; ++q) eq &= eq - 1;
            last = seg * kSeg + r * 64 + __ffsll(static_cast<unsigned long long>(eq)) - 1;
          }
          left -= c;
        }
        if (lane == 0) s.pick = last;
      }
      __syncthreads();
      cut = static_cast<uint64_t>(~b.key) << 32 | static_cast<uint32_t>(s.pick);
    }
    each_seg<T>(a, logits, [&](int seg, const float (&x)[8]) {
      uint64_t kept = 0;
#pragma unroll 1
      for (int e = 0; e < 8; ++e) {
        const double w = weight_far(value(x[e]), top, st.c);
        if (w >= st.m && place_of(value(x[e]), token_of<T>(seg, lane, e)) <= cut) kept += fixed(w);
      }
      kept = wave_sum64(kept);
      if (lane == 0) s.seg[seg] = kept;
    });
    for (int i = a.segs + tid; i < kSampleMaxSegs; i += kT) s.seg[i] = 0;
    __syncthreads();
  } else {
    // ---- the list
    s.seg[tid] = info.mode != kModeTopK ? seg_mass : 0;
    if (listed) {
      for (int i = tid; i < n; i += kT) {
        const uint64_t p = i < kT ? early[0] : i < 2 * kT ? early[1] : a.list[static_cast<size_t>(row) * kList + i];
        s.list[i] = p;
        const float l = logit_of(~static_cast<uint32_t>(p >> 32));
        s.w[i] = l >= info.least ? fixed(weight(l, z)) : 0;
      }
      total = info.mode == kModeTopP ? wave_sum64(total) : 0;
      above = info.mode == kModeTopP ? wave_sum64(above) : 0;
      __syncthreads();
      if (n <= kPairs) {
        cut = pairs_border(s, n, st.k, st.p, above, total);
      } else if (info.mode == kModeTopK) {
        cut = list_border(s, n, st.k, 0, 0.0);
        if (st.p < 1.0) {
          uint64_t mine = 0;
          for (int i = tid; i < n; i += kT) mine += s.list[i] <= cut ? s.w[i] : 0;
          mine = wave_sum64(mine);
          __syncthreads();
          if (lane == 0) s.part[wv] = mine;
          __syncthreads();
          for (int w = 0; w < kWaves; ++w) total += s.part[w];
          __syncthreads();
          cut = min(cut, list_border(s, n, 0, 0, st.p * static_cast<double>(total)));
        }
      } else {
        cut = list_border(s, n, 0, above, st.p * static_cast<double>(total));
      }
      for (int i = tid; i < n; i += kT) {
        const uint64_t p = s.list[i];
        if (p <= cut && logit_of(~static_cast<uint32_t>(p >> 32)) >= info.min_p)
          atomicAdd(reinterpret_cast<unsigned long long*>(&s.seg[static_cast<uint32_t>(p) / kSeg]), static_cast<unsigned long long>(s.w[i]));
      }
    }
    __syncthreads();
  }
  // ---- the segment: the first whose sum is above u times all of it
  static_assert(kSampleMaxSegs == kT && kSeg == kT, "a thread per segment, a thread per token of a segment");
  if (tid == 0) {
    s.pick = INT_MAX;
    s.seg_at = 0;
    s.seg_before = 0;
  }
  const uint64_t mass = s.seg[tid], upto = block_scan64(mass, s.part);
  uint64_t all = 0;
  for (int w = 0; w < kWaves; ++w) all += s.part[w];
  if (info.mode == kModeEqual) {                  // the first ones by index are kept
    const uint64_t one = fixed(weight(top, z));
    uint64_t n_kept = all / one;
    if (st.k > 0) n_kept = min(n_kept, static_cast<uint64_t>(st.k));
    if (st.p < 1.0) n_kept = max(static_cast<uint64_t>(ceil(st.p * static_cast<double>(n_kept))), static_cast<uint64_t>(1));
    all = n_kept * one;
  }
  if (!(u >= 0.f)) u = 0.f;
  u = fminf(u, 0.99999994f);
  uint64_t x = static_cast<uint64_t>(static_cast<double>(all) * static_cast<double>(u));
  if (x >= all) x = all > 0 ? all - 1 : 0;
  if (upto > x && upto - mass <= x) {
    s.seg_at = tid;
    s.seg_before = upto - mass;
  }
  __syncthreads();
  const int idx = s.seg_at * kSeg + tid;
  const float l = idx < a.V ? value(as_f32(logits[idx])) : -INFINITY;
  const double w = scanned ? weight_far(l, top, st.c) : weight(l >= info.min_p ? l : top, z);
  const bool kept = (scanned ? w >= st.m : l >= info.min_p) && (l >= sure || (l >= doubt && place_of(l, idx) <= cut));
  const uint64_t sum = s.seg_before + block_scan64(kept ? fixed(w) : 0, s.part2);
  if (kept && sum > x) atomicMin(&s.pick, tid);
  __syncthreads();
  if (tid == s.pick || (tid == 0 && s.pick == INT_MAX)) {
    a.token[row] = s.pick == INT_MAX ? -1 : idx;
    if (a.prob) a.prob[row] = s.pick == INT_MAX ? 0.f : static_cast<float>(w * kFix / static_cast<double>(all));
  }
}

template <typename T> hipError_t launch_as(const SampleArgs& a, hipStream_t s) {
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_sample_pick<T>), hipFuncAttributeMaxDynamicSharedMemorySize, sizeof(PickLds));
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL((k_sample_bins<T>), dim3(a.chunks, a.M), dim3(kT), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_sample_mass<T>), dim3(a.chunks, a.M), dim3(kT), 0, s, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_sample_pick<T>), dim3(a.M), dim3(kT), sizeof(PickLds), s, a);
  return hipGetLastError();
}

constexpr int kRowChunks = 512;         // chunks of a launch of few rows

size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

}  // namespace

void sample_plan(SampleArgs& a) {
  a.segs = (a.V + kSeg - 1) / kSeg;
  // two workgroups per compute unit where the rows are few, no more than twenty to a row: each of the second kernel's reads the histograms of all.
  // (7 rows: 12 chunks 19.1 us, 20 18.4, 32 19.4; 48 rows: 6 chunks 33.0, 11 32.3, 20 38.5; 144 rows, 5 chunks 64.5, 10 68.0)
  const int least = (a.segs + kChunkSegs - 1) / kChunkSegs;
  const int most = std::max(std::min(kSampleMaxChunks, (a.segs + kWaves - 1) / kWaves), least);
  const int chunks = std::max(std::min((kRowChunks + a.M - 1) / a.M, most), least);
  a.chunk_segs = (a.segs + chunks - 1) / chunks;
  a.chunks = (a.segs + a.chunk_segs - 1) / a.chunk_segs;
  // (the workspace has room for the chunks of any number of rows up to M: ceil(512 / m) m is less than 512 + m)
  a.row_chunks = std::min(static_cast<int64_t>(a.M) * most, std::max(static_cast<int64_t>(a.M) * least, static_cast<int64_t>(kRowChunks) - 1 + a.M));
}

// Lays the workspace out (base null: only its size).
size_t sample_carve(SampleArgs& a, void* base) {
  char* p = static_cast<char*>(base);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* r = p ? p + off : nullptr;
    off += align256(bytes);
    return r;
  };
  const size_t M = static_cast<size_t>(a.M), MC = static_cast<size_t>(a.row_chunks);
  a.hist = reinterpret_cast<uint32_t*>(take(MC * kBins * 4));
  a.chunk_sums = reinterpret_cast<unsigned long long*>(take(MC * 2 * 8));
  a.seg_mass = reinterpret_cast<unsigned long long*>(take(M * a.segs * 8));
  a.list = reinterpret_cast<unsigned long long*>(take(M * kList * 8));
  a.chunk_top = reinterpret_cast<float4*>(take(MC * 16));
  a.row_info = reinterpret_cast<SampleRow*>(take(M * sizeof(SampleRow)));
  return off;
}

hipError_t launch_sample(const SampleArgs& a, hipStream_t s) { return a.f32 ? launch_as<float>(a, s) : launch_as<bf16_t>(a, s); }

}  // namespace sx
