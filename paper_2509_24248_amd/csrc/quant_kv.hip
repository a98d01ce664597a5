// The 8-bit KV cache: rows quantised as they are written, and the compaction that closes a round over them.
//
// A row (one token of one KV head, d values) is stored as d e4m3 codes and one scale byte s, and stands for code 2^(s - 127).
// With amax = m 2^E the row's largest finite magnitude, 1 <= m < 2, s = E + 127 - 8 + (m > 1.75): the least power of two that
// brings the row within e4m3's 448 = 1.75 2^8.  A power of two because multiplying by it is exact: a code is one rounding of the
// value (to nearest even, at most 2^-4 of it; what lies more than 2^14 below the row's largest has e4m3's subnormal step, 2^-9), the
// same whatever order or machine computes it, and because it is the scale that the block-scaled matrix instructions
// multiply with (attn_quant.hip).  e4m3 is a floating type, so a finer scale would only move values within a binade.
#include "common.hpp"
#include "kernels.hpp"
#include "quant.hpp"

namespace sx {

namespace {

typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kTok = 16;        // tokens of a wave of the writing kernel

// maximum over the 16 (or 8) lanes that hold a row
template <int CTRL> __device__ __forceinline__ uint32_t row_umax(uint32_t v) {
  return max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xf, 0xf, false)));
}

// Row of entry p of (sequence b, KV head h) in the pools, or -1: outside the cache, or a page outside the pool.
__device__ __forceinline__ int64_t quant_row(const QuantKv& kv, int b, int h, int64_t p, int* status) {
  if (!kv.paged) return (static_cast<int64_t>(b) * kv.Hkv + h) * kv.l_max + p;
  const uint32_t in_seq = static_cast<uint32_t>(p) / static_cast<uint32_t>(kv.page_size);
  const int page = kv.page_table[static_cast<size_t>(b) * kv.max_pages + in_seq];
  if (!page_in_pool(page, kv.n_pages, status)) return -1;
  return (static_cast<int64_t>(page) * kv.Hkv + h) * kv.page_size + (p - static_cast<int64_t>(in_seq) * kv.page_size);
}

// A wave takes sixteen tokens of K or V of one head: D / 8 lanes a row, eight values a lane, all loads of the wave requested together.
// Bound by memory: 4 prompts of 4111 tokens, 8 heads, bf16 (76 MB): 13.8 to 14.4 us = 5.3 to 5.5 TB/s, a copy's rate 5.3 (with every value looked at
// for being finite, not only the wave's largest, 16.6: the vector unit was busy for 89 % of them); of fp32 ones (126 MB) 19.7 us = 6.4 TB/s; 64-wide
// heads 9.1 us (38 MB) and 11.0 (63 MB); a block of 56 tokens: 3.6 us, a launch and two dependent loads.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void k_quant_write(const QuantWriteArgs a) {
  constexpr int LPR = D / 8, RPI = 64 / LPR, U = kTok / RPI;     // lanes of a row, rows of an instruction, instructions
  const int lane = threadIdx.x & 63;
  const int64_t task = static_cast<int64_t>(blockIdx.x) * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (task >= a.tasks) return;
  const int which = static_cast<int>(task & 1);
  const uint32_t rest = static_cast<uint32_t>(task >> 1);
  const uint32_t bg = rest / static_cast<uint32_t>(a.kv.Hkv), h = rest - bg * a.kv.Hkv;
  const uint32_t b = bg / static_cast<uint32_t>(a.groups), t0 = (bg - b * a.groups) * kTok;
  const int count = a.count ? min(a.count[b], a.T) : a.T;
  const int pos = a.pos[b];
  const int sub = lane / LPR, c = lane % LPR;
  const T* src = static_cast<const T*>(which ? a.v : a.k) + (static_cast<int64_t>(b) * a.T + t0) * a.token_stride + h * D + c * 8;
  uint4 raw[U][sizeof(T) / 2];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int t = u * RPI + sub;
    const bool in = static_cast<int>(t0) + t < count;
    const uint4* p = reinterpret_cast<const uint4*>(src + static_cast<int64_t>(in ? t : 0) * a.token_stride);
#pragma unroll
    for (unsigned i = 0; i < sizeof(T) / 2; ++i) raw[u][i] = in ? p[i] : make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int t = static_cast<int>(t0) + u * RPI + sub;
    float x[8];
    if constexpr (sizeof(T) == 2) {
      unpack16(raw[u][0], x);
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x[4 * i] = __uint_as_float(raw[u][i].x); x[4 * i + 1] = __uint_as_float(raw[u][i].y);
        x[4 * i + 2] = __uint_as_float(raw[u][i].z); x[4 * i + 3] = __uint_as_float(raw[u][i].w);
      }
    }
    uint32_t amax = 0;              // magnitudes compare like their bits
    if constexpr (sizeof(T) == 2) {
      auto larger = [](uint32_t p, uint32_t q) { return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, p), __builtin_bit_cast(u16x2_t, q))); };
      constexpr uint32_t kMag = 0x7FFF7FFFu;
      const uint32_t two = larger(larger(raw[u][0].x & kMag, raw[u][0].y & kMag), larger(raw[u][0].z & kMag, raw[u][0].w & kMag));
      amax = max(two << 16, two & 0xFFFF0000u);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = max(amax, __float_as_uint(x[e]) & 0x7FFFFFFFu);
    }
    const bool odd = __builtin_amdgcn_ballot_w64(amax >= 0x7F800000u) != 0ull;          // (uniform) some value of the wave is not finite
    if (odd) {
      amax = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t bits = __float_as_uint(x[e]) & 0x7FFFFFFFu;
        amax = max(amax, bits < 0x7F800000u ? bits : 0u);
      }
    }
    amax = row_umax<0xB1>(amax);                       // lanes 1, 2, 4 (and 8) apart
    amax = row_umax<0x4E>(amax);
    amax = row_umax<0x141>(amax);
    if constexpr (LPR == 16) amax = row_umax<0x140>(amax);
    const int s = quant_scale_byte(amax);
    const float inv = quant_scale_inverse(s);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * inv, x[4 * i + 1] * inv, static_cast<int>(w[i]), false);
      w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * inv, x[4 * i + 3] * inv, static_cast<int>(w[i]), true);
    }
    // a value that is not finite has the NaN code with its sign
    if (odd) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t bits = __float_as_uint(x[e]);
        if ((bits & 0x7FFFFFFFu) >= 0x7F800000u) {
          const int sh = 8 * (e & 3);
          w[e >> 2] = (w[e >> 2] & ~(0xFFu << sh)) | ((0x7Fu | (bits >> 24 & 0x80u)) << sh);
        }
      }
    }
    if (t >= count) continue;
    const int64_t p = static_cast<int64_t>(pos) + t;
    if (p < 0 || p >= a.kv.l_max) {
      report_status(a.status, kStatusBadLength);
      continue;
    }
    const int64_t row = quant_row(a.kv, b, h, p, a.status);
    if (row < 0) continue;
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(which ? a.kv.v : a.kv.k) + row * D + c * 8) = make_uint2(w[0], w[1]);
    if (c == 0) static_cast<uint8_t*>(which ? a.kv.vs : a.kv.ks)[row] = static_cast<uint8_t>(s);
  }
}

// A wave per layer, sequence and KV head, and one per sequence that copies its hidden row.  Lane j holds path entry j and where its row
// comes from and goes to; the rows are then moved by all lanes, D / 16 of them to one, and all are read before any is written.  U: sixteen-byte
// pieces of a lane.  Latency is all there is, so few waves with few instructions count: 4 sequences of 16 nodes, 36 layers, 8 heads: 3.7 us, 16 of
// 9 nodes, 64 layers, paged: 6.8 us (a workgroup of four waves per layer and head, pieces divided among its threads: 18.4 and 34.2).
template <int D, int U>
__global__ __launch_bounds__(kThreads) void k_quant_compact(const QuantCompactArgs a) {
  const int lane = threadIdx.x & 63;
  int task = static_cast<int>(blockIdx.x) * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (task >= a.tasks) return;
  if (task >= a.moves) {
    const int b = task - a.moves;
    int node = a.last_node[b];
    if (node < 0 || node >= a.n_q) report_status(a.status, kStatusBadNode);
    node = max(0, min(node, a.n_q - 1));
    const uint4* src = reinterpret_cast<const uint4*>(static_cast<const char*>(a.block_hidden) + (static_cast<size_t>(b) * a.n_q + node) * a.hidden_row_bytes);
    uint4* dst = reinterpret_cast<uint4*>(static_cast<char*>(a.hidden_next) + static_cast<size_t>(b) * a.hidden_row_bytes);
#pragma unroll 8
    for (int i = lane; i < (a.hidden_row_bytes >> 4); i += 64) dst[i] = src[i];
    return;
  }
  const int layer = task / (a.B * a.kv.Hkv);
  task -= layer * a.B * a.kv.Hkv;
  const int b = task / a.kv.Hkv, h = task - b * a.kv.Hkv;
  const int L = a.ctx_len[b];
  const int m = max(0, min(a.accept_len[b], a.n_q - 1));
  const int node = lane < a.n_q ? a.accept_path[static_cast<size_t>(b) * a.n_q + lane] : -1;
  if (L < 0 || static_cast<int64_t>(L) + a.n_q > a.kv.l_max) {
    report_status(a.status, kStatusBadLength);
    return;
  }
  const uint64_t away = __builtin_amdgcn_ballot_w64(lane < m && node != lane + 1);
  if (!away) return;
  const int first = __ffsll(static_cast<unsigned long long>(away)) - 1, rows = m - first;      // rows that may move
  // rows of path entry `lane`; -1 where nothing moves
  int64_t from = -1, to = -1;
  if (lane >= first && lane < m) {
    if (node >= 1 && node < a.n_q) {
      from = quant_row(a.kv, b, h, L + node, a.status);
      to = quant_row(a.kv, b, h, L + 1 + lane, a.status);
      if (from < 0) to = -1;
    } else {
      report_status(a.status, kStatusBadNode);
    }
  }
  char* const pool[2] = {static_cast<char*>(a.kv.k) + layer * a.layer_stride, static_cast<char*>(a.kv.v) + layer * a.layer_stride};
  uint8_t* const ks = static_cast<uint8_t*>(a.kv.ks) + layer * a.scale_stride;
  uint8_t* const vs = static_cast<uint8_t*>(a.kv.vs) + layer * a.scale_stride;
  uint8_t k_scale = 0, v_scale = 0;
  if (to >= 0) { k_scale = ks[from]; v_scale = vs[from]; }
  constexpr int LPR = D / 16;
  const int items = 2 * rows * LPR;                    // K rows, then V rows
  auto row_of = [](int64_t row, int j) {
    return static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(__shfl(static_cast<int>(row >> 32), j))) << 32 | static_cast<uint32_t>(__shfl(static_cast<int>(row), j)));
  };
  uint4 buf[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    buf[u] = make_uint4(0, 0, 0, 0);
    if (64 * u < items) {                              // uniform
      const int r = (64 * u + lane) / LPR, v = r >= rows;
      const int j = min(first + r - (v ? rows : 0), 63);
      const int64_t dst = row_of(to, j), src = row_of(from, j);
      if (64 * u + lane < items && dst >= 0) buf[u] = *reinterpret_cast<const uint4*>(pool[v] + src * D + (lane % LPR) * 16);
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // (nothing is written before everything has arrived)
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (64 * u < items) {
      const int r = (64 * u + lane) / LPR, v = r >= rows;
      const int64_t dst = row_of(to, min(first + r - (v ? rows : 0), 63));
      if (64 * u + lane < items && dst >= 0) *reinterpret_cast<uint4*>(pool[v] + dst * D + (lane % LPR) * 16) = buf[u];
    }
  }
  if (to >= 0) { ks[to] = k_scale; vs[to] = v_scale; }
}

template <typename T>
hipError_t launch_write(const QuantWriteArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>((a.tasks + kThreads / 64 - 1) / (kThreads / 64)));
  if (a.d == 128) hipLaunchKernelGGL((k_quant_write<T, 128>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((k_quant_write<T, 64>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

// Sets the launch's task count; false: more than one launch takes.
bool quant_write_plan(QuantWriteArgs& a) {
  a.groups = (a.T - 1) / kTok + 1;
  const int64_t all = static_cast<int64_t>(a.B) * a.groups;
  if (all > kLaunchWaves || all * a.kv.Hkv > kLaunchWaves / 2) return false;
  a.tasks = 2 * all * a.kv.Hkv;
  return true;
}

hipError_t launch_quant_write(const QuantWriteArgs& a, hipStream_t s) { return a.f32 ? launch_write<float>(a, s) : launch_write<bf16_t>(a, s); }

hipError_t launch_quant_compact(const QuantCompactArgs& args, hipStream_t s) {
  QuantCompactArgs a = args;
  a.moves = a.n_layers * a.B * a.kv.Hkv;
  a.tasks = a.moves + (a.block_hidden ? a.B : 0);
  const dim3 grid((a.tasks + kThreads / 64 - 1) / (kThreads / 64));
  // pieces of a lane: 2 (n_q - 1) rows of d bytes over 64 lanes at most; four of them (a block of 17 at d = 128) take 34 registers, all waves of
  // a unit, sixteen 88
  const bool few = 2 * (a.n_q - 1) * (a.d / 16) <= 4 * 64;
  if (a.d == 128) {
    if (few) hipLaunchKernelGGL((k_quant_compact<128, 4>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((k_quant_compact<128, 16>), grid, dim3(kThreads), 0, s, a);
  } else {
    if (few) hipLaunchKernelGGL((k_quant_compact<64, 4>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((k_quant_compact<64, 16>), grid, dim3(kThreads), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace sx
