// Rotary positions: the frequencies' table, the rotation of a block's (or a prompt's) heads, keys and values appended to the cache on the
// way, and the entries of a latent cache.
//
// Pair c of a head at position p turns by p f_c.  A table holds f_c / 2 pi as a 64-bit binary fraction of a turn, so that the
// whole turns of p f_c drop out of an integer product exactly: what is left is off by p times the table's own error (a unit of 2^-64 turns, and 32 roundings of
// 64-bit arithmetic, 2^-48 of f_c), and nothing is lost to large angles.  Of the fraction its upper 32 bits are kept (off by up to 2^-32 turns, 1.5e-9, downward: 40 times
// less than a rounding of a value that is not turned at all) and cut to the nearest quarter turn; the rest, within an eighth, goes through the Taylor polynomials of sine and cosine to the eleventh and tenth power (the first
// terms left out are 7e-12 and 2e-10 of theirs at pi / 4, below a rounding).
//
// A value is read once, turned in fp32 and rounded once.  A lane takes two 16-byte pieces of a head (the two halves of its pairs, or
// neighbours), so that a pair never leaves its lane; a wave takes some heads of one token, whose sines and cosines it works out once.
#include "common.hpp"
#include "kernels.hpp"

#include <algorithm>

namespace sx {

namespace {

constexpr int kThreads = 256;

// 16 bytes of storage values
template <typename T> struct Piece;
template <> struct Piece<bf16_t> {
  static constexpr int N = 8;
  __device__ static __forceinline__ void get(const uint4& v, float (&f)[8]) { unpack16(v, f); }
  __device__ static __forceinline__ uint4 put(const float (&f)[8]) {
    return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
  }
  __device__ static __forceinline__ bf16_t one(float f) { return static_cast<bf16_t>(pack_bf16x2(f, f)); }
};
template <> struct Piece<float> {
  static constexpr int N = 4;
  __device__ static __forceinline__ void get(const uint4& v, float (&f)[4]) {
    f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
  }
  __device__ static __forceinline__ uint4 put(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
  __device__ static __forceinline__ float one(float f) { return f; }
};

// amplitude * (cos, sin) of p times a frequency of the table
__device__ __forceinline__ void turn_at(uint32_t p, uint64_t turns, float amplitude, float& cs, float& sn) {
  const uint32_t frac = static_cast<uint32_t>((turns * p) >> 32);
  const uint32_t quarter = (frac + 0x20000000u) >> 30;
  const float x = static_cast<float>(static_cast<int32_t>(frac - (quarter << 30))) * 1.4629180792671596e-09f;      // 2 pi / 2^32
  const float z = x * x;
  const float s = x * fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -2.5052108e-8f, 2.7557319e-6f), -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), 1.f);
  const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.f);
  const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  cs = amplitude * ((quarter + 1) & 2 ? -a : a);
  sn = amplitude * (quarter & 2 ? -b : b);
}

__global__ __launch_bounds__(kThreads) void k_rope_table(const RopeTableArgs a) {
  const int c = threadIdx.x;
  if (c >= a.rot / 2) return;
  const double two_pi = 6.283185307179586476925;
  double f = pow(static_cast<double>(a.theta), -2.0 * c / a.rot);
  const double factor = a.factor, low = a.low, high = a.high, len = a.orig_len;
  if (a.scaling == kRopeLinear) {
    f /= factor;
  } else if (a.scaling == kRopeBands) {
    const double keep = fmin(fmax((len * f / two_pi - low) / (high - low), 0.0), 1.0);
    f *= keep + (1.0 - keep) / factor;
  } else if (a.scaling == kRopeRamp) {
    // pairs that make `high` turns and `low` turns over the original length
    const double per = a.rot / (2.0 * log(static_cast<double>(a.theta)));
    const double first = fmax(floor(per * log(len / (high * two_pi))), 0.0), last = fmin(ceil(per * log(len / (low * two_pi))), a.rot - 1.0);
    const double away = fmin(fmax((c - first) / fmax(last - first, 0.001), 0.0), 1.0);
    f = f * (1.0 - away) + f / factor * away;
  }
  a.turns[c] = static_cast<uint64_t>(f * (18446744073709551616.0 / two_pi));
}

// The pairs of a lane's two pieces: (lo[e], hi[e]), or neighbours in lo and then in hi.
template <int N, bool PAIRS>
__device__ __forceinline__ void turn_pieces(float (&lo)[N], float (&hi)[N], const float (&cs)[N], const float (&sn)[N], int valid) {
#pragma unroll
  for (int e = 0; e < N; ++e) {
    float& x = PAIRS ? (e < N / 2 ? lo[2 * e] : hi[2 * e - N]) : lo[e];
    float& y = PAIRS ? (e < N / 2 ? lo[2 * e + 1] : hi[2 * e + 1 - N]) : hi[e];
    const float u = x * cs[e] - y * sn[e], v = x * sn[e] + y * cs[e];
    x = e < valid ? u : x;                    // (a choice, not a factor of one: what does not turn may be infinite)
    y = e < valid ? v : y;
  }
}

// Rotary position of token t of sequence b, forced into 0 .. 2^31 - 1.
__device__ __forceinline__ uint32_t rotary_position(const int32_t* offset, int pos, int b, int t, int T, int* status) {
  const int64_t p = static_cast<int64_t>(pos) + (offset ? offset[static_cast<int64_t>(b) * T + t] : t);
  if (p < 0 || p > 0x7fffffff) report_status(status, kStatusBadLength);
  return static_cast<uint32_t>(p < 0 ? 0 : p > 0x7fffffff ? 0x7fffffff : p);
}

// Place of entry p of sequence b as (pool block, entry of it), pool blocks being pages or sequences; false: outside the cache, or a page outside the pool.
struct Place {
  int64_t block;
  int at;
};
// (`page`: the page table's word for p, which the caller has asked for, if p is in the cache)
__device__ __forceinline__ bool entry_place(const CachePlace& kv, int b, int64_t p, int page, int* status, Place& out) {
  if (p < 0 || p >= kv.l_max) {
    report_status(status, kStatusBadLength);
    return false;
  }
  if (!kv.paged) {
    out.block = b;
    out.at = static_cast<int>(p);
    return true;
  }
  const uint32_t in_seq = static_cast<uint32_t>(p) / static_cast<uint32_t>(kv.page_size);
  out.block = page;
  out.at = static_cast<int>(p - static_cast<int64_t>(in_seq) * kv.page_size);
  return page_in_pool(page, kv.n_pages, status);
}

enum { kHalves = 0, kNeighbours = 1, kHalvesOdd = 2 };       // kHalvesOdd: half of the rotated values is no whole number of pieces

// A wave takes `per` steps of 64 / LPR rows each of one token, rows being its q heads, k heads and v heads.
template <typename T, int MODE>
__global__ __launch_bounds__(kThreads) void k_rope_rows(const RopeRowsArgs a) {
  constexpr int N = Piece<T>::N;
  arguments_at_once<sizeof(RopeRowsArgs)>();
  const int lane = threadIdx.x & 63;
  const uint32_t task = blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);      // (fewer than 2^26)
  if (task >= static_cast<uint32_t>(a.tasks)) return;
  const uint32_t token = task / static_cast<uint32_t>(a.groups);
  const int group = static_cast<int>(task - token * static_cast<uint32_t>(a.groups));
  const int b = static_cast<int>(token / static_cast<uint32_t>(a.T)), t = static_cast<int>(token - static_cast<uint32_t>(b) * static_cast<uint32_t>(a.T));
  const int64_t bt = token;
  if (a.count && t >= a.count[b]) return;
  const int LPR = a.d / (2 * N), RPW = 64 / LPR;
  const int sub = lane / LPR, i = lane - sub * LPR;
  const int rows = a.Hq + 2 * a.Hkv;
  const int pos = a.pos[b];
  const int64_t p = static_cast<int64_t>(pos) + t;
  int page = -1;
  if (a.Hkv && a.kv.paged && p >= 0 && p < a.kv.l_max) page = a.kv.page_table[static_cast<int64_t>(b) * a.kv.max_pages + static_cast<uint32_t>(p) / static_cast<uint32_t>(a.kv.page_size)];
  const uint32_t turn = rotary_position(a.offset, pos, b, t, a.T, a.status);
  Place at = {0, 0};
  bool stored = false;
  if (a.Hkv) stored = entry_place(a.kv, b, p, page, a.status, at);
  if (sub >= RPW) return;
  // pairs i N .. i N + N - 1; in kHalvesOdd i, i + LPR, ..
  const int half = a.rot / 2;
  float cs[N], sn[N];
  int valid = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const int c = MODE == kHalvesOdd ? i + e * LPR : i * N + e;
    turn_at(turn, a.turns[min(c, half - 1)], a.amplitude, cs[e], sn[e]);
    valid += c < half;
  }
  const int first = group * a.per * RPW + sub;
  const int last = min(rows, (group + 1) * a.per * RPW);
  const T* q = static_cast<const T*>(a.q) + bt * a.q_stride;
  auto source = [&](int r) {
    if (r < a.Hq) return q + static_cast<int64_t>(r) * a.d;
    const int h = r - a.Hq;
    return static_cast<const T*>(h < a.Hkv ? a.k : a.v) + bt * a.kv_stride + static_cast<int64_t>(h < a.Hkv ? h : h - a.Hkv) * a.d;
  };
  auto target = [&](int r) -> T* {
    if (r < a.Hq) return static_cast<T*>(a.q_out) + bt * a.out_stride + static_cast<int64_t>(r) * a.d;
    if (!stored) return nullptr;
    const int h = r - a.Hq;
    const int64_t entries = a.kv.paged ? a.kv.page_size : a.kv.l_max;
    return static_cast<T*>(h < a.Hkv ? a.kc : a.vc) + ((at.block * a.Hkv + (h < a.Hkv ? h : h - a.Hkv)) * entries + at.at) * a.d;
  };
  if constexpr (MODE == kHalvesOdd) {
    for (int r = first; r < last; r += RPW) {
      const T* src = source(r);
      T* dst = target(r);
      if (!dst) continue;
      const bool turned = r < a.Hq + a.Hkv;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int c = i + e * LPR;
        if (c >= half) continue;
        const T u = src[c], v = src[c + half];
        const float x = Elem<T>::load(&u), y = Elem<T>::load(&v);
        dst[c] = turned ? Piece<T>::one(x * cs[e] - y * sn[e]) : u;
        dst[c + half] = turned ? Piece<T>::one(x * sn[e] + y * cs[e]) : v;
      }
      for (int c = a.rot + i; c < a.d; c += LPR) dst[c] = src[c];
    }
    return;
  } else {
    const bool split = MODE == kHalves && valid > 0;          // (kHalves: a lane's pairs are all of the rotated ones or none)
    const int lo_at = split ? i * N : MODE == kHalves ? a.rot + (i - half / N) * 2 * N : i * 2 * N;
    const int hi_at = split ? lo_at + half : lo_at + N;
#pragma unroll 1
    for (int r = first; r < last; r += 2 * RPW) {
      uint4 raw[2][2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const T* src = source(min(r + u * RPW, last - 1));
        raw[u][0] = *reinterpret_cast<const uint4*>(src + lo_at);
        raw[u][1] = *reinterpret_cast<const uint4*>(src + hi_at);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int ru = r + u * RPW;
        T* dst = ru < last ? target(ru) : nullptr;
        if (!dst) continue;
        if (ru < a.Hq + a.Hkv) {
          float lo[N], hi[N];
          Piece<T>::get(raw[u][0], lo);
          Piece<T>::get(raw[u][1], hi);
          turn_pieces<N, MODE == kNeighbours>(lo, hi, cs, sn, valid);
          raw[u][0] = Piece<T>::put(lo);
          raw[u][1] = Piece<T>::put(hi);
        }
        *reinterpret_cast<uint4*>(dst + lo_at) = raw[u][0];
        *reinterpret_cast<uint4*>(dst + hi_at) = raw[u][1];
      }
    }
  }
}

// Entries of a latent cache: a wave brings the latents of U tokens to a root mean square of one, all its lanes on one after the other, multiplies with the gain and turns the key parts,
// LPR lanes a token; behind those, waves that turn the queries' part of some heads of a token.  U = 8 where there are tokens enough: sines and cosines are the most of a token's
// instructions, and with one token four lanes of 64 need them (4 prompts of 4111 tokens at most, 28 MB: 14.1 us with one).
template <typename T, bool PAIRS, int U>
__global__ __launch_bounds__(kThreads) void k_latent_write(const LatentWriteArgs a) {
  constexpr int N = Piece<T>::N, LPR = kLatentRope / (2 * N), RPW = 64 / LPR;       // lanes of a rotated part, parts of a wave
  constexpr int P = sizeof(T) == 2 ? 1 : 2;                                         // pieces of the latent of a lane, at most
  static_assert(U <= RPW, "");
  arguments_at_once<sizeof(LatentWriteArgs)>();
  const int lane = threadIdx.x & 63;
  uint32_t task = blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (task >= static_cast<uint32_t>(a.tasks)) return;
  const bool entry = task < static_cast<uint32_t>(a.entries);
  const uint32_t T_ = static_cast<uint32_t>(a.T), tokens = static_cast<uint32_t>(a.B) * T_;
  const int sub = lane / LPR, i = lane % LPR;
  uint32_t bt;                                      // a lane's token
  int h = 0;                                        // and head
  bool mine;
  if (entry) {
    bt = min(task * U + static_cast<uint32_t>(sub), tokens - 1);
    mine = sub < U && task * U + static_cast<uint32_t>(sub) < tokens;
  } else {
    task -= static_cast<uint32_t>(a.entries);
    bt = task / static_cast<uint32_t>(a.q_groups);
    h = static_cast<int>(task - bt * static_cast<uint32_t>(a.q_groups)) * RPW + sub;
    mine = h < a.H;
    h = min(h, a.H - 1);
  }
  const int b = static_cast<int>(bt / T_), t = static_cast<int>(bt - static_cast<uint32_t>(b) * T_);
  const int pos = a.pos[b];
  mine = mine && (!a.count || t < a.count[b]);
  if (!__builtin_amdgcn_ballot_w64(mine)) return;
  // frequencies and the entry's page are asked for beside the rows, not behind them
  uint64_t turns[N];
#pragma unroll
  for (int e = 0; e < N; ++e) turns[e] = a.turns[i * N + e];
  const int64_t p = static_cast<int64_t>(pos) + t;
  int page = -1;
  if (entry && mine && a.kv.paged && p >= 0 && p < a.kv.l_max) page = a.kv.page_table[static_cast<int64_t>(b) * a.kv.max_pages + static_cast<uint32_t>(p) / static_cast<uint32_t>(a.kv.page_size)];
  const int lo_at = PAIRS ? i * 2 * N : i * N, hi_at = PAIRS ? lo_at + N : lo_at + kLatentRope / 2;
  const int pieces = a.r / N;
  uint4 raw[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)}, lat[U][P], gain[P];
  if (mine) {
    const T* src = entry ? static_cast<const T*>(a.rows) + static_cast<int64_t>(bt) * a.row_stride + a.r
                         : static_cast<const T*>(a.q_rows) + static_cast<int64_t>(bt) * a.q_stride + static_cast<int64_t>(h) * a.head_stride;
    raw[0] = *reinterpret_cast<const uint4*>(src + lo_at);
    raw[1] = *reinterpret_cast<const uint4*>(src + hi_at);
  }
  const uint64_t live = __builtin_amdgcn_ballot_w64(mine);
  if (entry) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint4* p = reinterpret_cast<const uint4*>(static_cast<const T*>(a.rows) + static_cast<int64_t>(task * U + u) * a.row_stride);
#pragma unroll
      for (int k = 0; k < P; ++k) lat[u][k] = (live >> (u * LPR) & 1) && lane + k * 64 < pieces ? p[lane + k * 64] : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < P; ++k) gain[k] = a.gain && lane + k * 64 < pieces ? static_cast<const uint4*>(a.gain)[lane + k * 64] : make_uint4(0, 0, 0, 0);
  }
  uint32_t turn = 0;
  Place at = {0, 0};
  if (mine) {
    turn = rotary_position(a.offset, pos, b, t, a.T, a.status);
    if (entry) mine = entry_place(a.kv, b, p, page, a.status, at);
  }
  float cs[N], sn[N], lo[N], hi[N];
#pragma unroll
  for (int e = 0; e < N; ++e) turn_at(turn, turns[e], a.amplitude, cs[e], sn[e]);
  Piece<T>::get(raw[0], lo);
  Piece<T>::get(raw[1], hi);
  turn_pieces<N, PAIRS>(lo, hi, cs, sn, N);
  const int64_t row = at.block * (a.kv.paged ? a.kv.page_size : a.kv.l_max) + at.at;       // of a lane's token in the pool
  if (mine) {
    T* dst = entry ? static_cast<T*>(a.c) + row * (a.r + kLatentRope) + a.r
                   : static_cast<T*>(a.q_out) + (static_cast<int64_t>(bt) * a.H + h) * (a.r + kLatentRope) + a.r;
    *reinterpret_cast<uint4*>(dst + lo_at) = Piece<T>::put(lo);
    *reinterpret_cast<uint4*>(dst + hi_at) = Piece<T>::put(hi);
  }
  if (!entry) return;
  const float per_value = 1.f / static_cast<float>(a.r);      // (a power of two)
  const uint64_t placed = __builtin_amdgcn_ballot_w64(mine);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (!(placed >> (u * LPR) & 1)) continue;       // (uniform)
    const int64_t to = static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(row >> 32), u * LPR))) << 32 |
                                            static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(row), u * LPR)));
    if (a.gain) {
      float x[P][N], ssq = 0.f;
#pragma unroll
      for (int k = 0; k < P; ++k) {
        Piece<T>::get(lat[u][k], x[k]);
#pragma unroll
        for (int e = 0; e < N; ++e) ssq = fmaf(x[k][e], x[k][e], ssq);
      }
      const float inv = rsqrtf(wave_sum_dpp(ssq) * per_value + a.eps);
#pragma unroll
      for (int k = 0; k < P; ++k) {
        float g[N];
        Piece<T>::get(gain[k], g);
#pragma unroll
        for (int e = 0; e < N; ++e) x[k][e] = x[k][e] * inv * g[e];
        lat[u][k] = Piece<T>::put(x[k]);
      }
    }
    uint4* dst = reinterpret_cast<uint4*>(static_cast<T*>(a.c) + to * (a.r + kLatentRope));
#pragma unroll
    for (int k = 0; k < P; ++k)
      if (lane + k * 64 < pieces) dst[lane + k * 64] = lat[u][k];
  }
}

template <typename T>
void launch_rows_as(const RopeRowsArgs& a, unsigned grid, hipStream_t s) {
  if (a.neighbours) hipLaunchKernelGGL((k_rope_rows<T, kNeighbours>), dim3(grid), dim3(kThreads), 0, s, a);
  else if (a.rot % (2 * Piece<T>::N) == 0) hipLaunchKernelGGL((k_rope_rows<T, kHalves>), dim3(grid), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((k_rope_rows<T, kHalvesOdd>), dim3(grid), dim3(kThreads), 0, s, a);
}

}  // namespace

hipError_t launch_rope_table(const RopeTableArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(k_rope_table, dim3(1), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

// Waves from which on one takes several steps: 32 a compute unit.
constexpr int64_t kRopeWaves = 8192;
bool rope_rows_plan(RopeRowsArgs& a) {
  const int per_step = 64 / (a.d / (a.f32 ? 8 : 16));             // rows of a wave's step
  const int steps = (a.Hq + 2 * a.Hkv + per_step - 1) / per_step;
  const int64_t tokens = static_cast<int64_t>(a.B) * a.T;
  if (tokens > kLaunchWaves) return false;
  // few tokens: a step per wave, so that the call is as short as one; many: more of a token's heads in one wave, which shares their sines and cosines
  a.per = static_cast<int>(std::min<int64_t>(steps, std::max<int64_t>(1, tokens * steps / kRopeWaves)));
  a.groups = (steps + a.per - 1) / a.per;
  a.tasks = tokens * a.groups;
  return a.tasks <= kLaunchWaves;
}

hipError_t launch_rope_rows(const RopeRowsArgs& a, hipStream_t s) {
  const unsigned grid = static_cast<unsigned>((a.tasks + 3) / 4);
  if (a.f32) launch_rows_as<float>(a, grid, s);
  else launch_rows_as<bf16_t>(a, grid, s);
  return hipGetLastError();
}

// Tokens from which a wave takes eight.
constexpr int64_t kManyTokens = 4096;
bool latent_write_plan(LatentWriteArgs& a) {
  const int64_t tokens = static_cast<int64_t>(a.B) * a.T;
  if (tokens > kLaunchWaves) return false;
  a.many = tokens >= kManyTokens;
  a.entries = a.many ? (tokens + 7) / 8 : tokens;
  const int rows = a.f32 ? 8 : 16;                                // rotated parts of a wave
  a.q_groups = (a.H + rows - 1) / rows;
  a.tasks = a.entries + tokens * a.q_groups;
  return a.tasks <= kLaunchWaves;
}

template <typename T, bool PAIRS>
static void launch_latent_as(const LatentWriteArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>((a.tasks + 3) / 4)), block(kThreads);
  if (a.many) hipLaunchKernelGGL((k_latent_write<T, PAIRS, 8>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((k_latent_write<T, PAIRS, 1>), grid, block, 0, s, a);
}

hipError_t launch_latent_write(const LatentWriteArgs& a, hipStream_t s) {
  if (a.f32) {
    if (a.neighbours) launch_latent_as<float, true>(a, s);
    else launch_latent_as<float, false>(a, s);
  } else {
    if (a.neighbours) launch_latent_as<bf16_t, true>(a, s);
    else launch_latent_as<bf16_t, false>(a, s);
  }
  return hipGetLastError();
}

}  // namespace sx
