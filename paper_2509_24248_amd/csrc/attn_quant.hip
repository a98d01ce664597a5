// Verification attention over the 8-bit cache (quant_kv.hip), on the matrix cores.
//
// The keys of the launch are dealt to the workgroups in equal shares (attn_sched.hpp); a workgroup takes one (sequence, KV head)
// unit's key range at a time, against all R = G * n_q query rows that share the head, so that the cache is read once.  It has NK
// rings of S LDS slots; ring kg takes the 32-key tiles kg, kg + NK, .. of the range, brought in by direct global->LDS loads S - 1 tiles ahead.
// The ring's NR waves own RTW 16-row tiles of the queries each:
//   S^T = K Q^T : block-scaled matrix instruction, 16 keys x 16 rows x 128 products.  A = the codes as they lie in the cache, with
//                 the keys' scale bytes as its scales.  B = the queries as a sum of e4m3 parts, each with its own power of two:
//                 a part takes four bits of what is left, so two parts hold a bf16 value that is a normal number of the first: from 2^-14 of
//                 the row's power of two on, 2^-13 of its largest value.  What lies below has the lesser part's least step, and is off by half of it,
//                 2^-21.8 of the largest value, at most.  The products are exact and no key is converted.  (The instruction drops what lies 2^-23
//                 below its largest product, some 1e-5 of a score, which the rounding to bf16 hides and fp32 results do not: there, keys are
//                 converted to bf16, exactly, and the queries are three bf16 parts.  With six e4m3 parts the tiny fp32 shape was off by 3.4e-5.
//                 One bf16 part of the queries and converted keys would hold any bf16 value too: 8 sequences of 2048 .. 16384 tokens 34.0 -> 36.4 us
//                 at 28 rows, 57.1 -> 65.6 at 72, 16 of 8192 .. 32768 195 -> 226.)
//   softmax     : online, per wave, in log2 units; lane (row, q) owns 8 keys of its row;
//   O^T += V^T P^T : A = V codes, transposed on the way out of LDS (eight keys of a column per lane) and converted to bf16,
//                 which is exact; B = the probabilities times the keys' scales (powers of two: exact) in PP bf16 parts.
// 64-wide heads need half the products: the instruction's second half then takes the same codes with the next part of the queries.
//
// What bounds it.  Few rows: memory (8 sequences of 2k to 16k tokens, 28 rows a head, 153 MB: 31 us = 4.9 TB/s, and 4.7 for the merge).  Many:
// instructions.  16 rows x 32 keys take a wave some 129 vector instructions of 4.4 cycles - 32 convert V, 8 exponentials of 8.4 - and 256 cycles of
// matrix instructions on a unit that issues one or the other: 16 sequences of 8k to 32k, 72 rows: 193 to 199 us for 681 MB, 129 at a copy's rate.
// Short: the split from the lengths, its first loads and the merge (one sequence of 4096: 8.8 and 3.6 us).
// Tried: both operands of the next tile in registers across the barrier (no gain); two workgroups of five waves per compute unit (slower); three or
// four row tiles to a wave, one wave a SIMD (slower: 5.3 cycles an instruction); tiles unrolled over the ring's slots (spills).
#include "attn_sched.hpp"
#include "common.hpp"
#include "kernels.hpp"
#include "quant.hpp"
#include "stream.hpp"

#include <float.h>

#include <algorithm>

namespace sx {

namespace {

typedef int v2i_t __attribute__((ext_vector_type(2)));
typedef int v8i_t __attribute__((ext_vector_type(8)));
typedef float v2f_t __attribute__((ext_vector_type(2)));
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((address_space(3))) v2i_t* lds_v2i_t;

constexpr int kMaxGroups = 2048;     // groups of 16 keys of a paged segment, whose places in the pool are kept in LDS (8 KB)
constexpr int kTileKeys = 32;
constexpr size_t kRingLds = 128 * 1024;

__host__ __device__ constexpr int slot_bytes(int hd) { return 2 * kTileKeys * hd; }    // K codes, then V codes
constexpr int kScaleSlot = 2 * kTileKeys;        // K scale bytes, then V scale bytes
// Slots of a ring.
__host__ __device__ constexpr int ring_slots(int hd, int nk) { return static_cast<int>(kRingLds) / (nk * slot_bytes(hd)) > 8 ? 8 : static_cast<int>(kRingLds) / (nk * slot_bytes(hd)); }

// XOR swizzles of the 16-byte chunks of a tile row, so that the 16 rows (K) or 16 rows x 1 chunk (V) that an instruction reads at once lie on
// different banks: 128-wide rows are two to the 256 bytes of all banks, 64-wide ones four.
template <int HD> __device__ __forceinline__ int swz_k(int key) { return HD == 128 ? (key >> 1) & 7 : (key >> 2) & 3; }
template <int HD> __device__ __forceinline__ int swz_v(int key) {      // (V reads take keys 4 q .. + 3 and 16 + 4 q .. + 3 together)
  return HD == 128 ? ((key >> 1) & 3) | ((key >> 4) & 1) << 2 : ((key >> 2) & 1) | ((key >> 4) & 1) << 1;
}

__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }   // (hands a NaN on)
__device__ __forceinline__ float max3_nan(float a, float b, float c) { return max_nan(max_nan(a, b), c); }

__device__ __forceinline__ uint32_t two_bf16(uint32_t codes, bool hi) {
  const bf16x2_t v = hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.0f, false);
  return __builtin_bit_cast(uint32_t, v);
}

// 16 keys x 16 rows: a with the scale bytes of `sa` (byte 0), b with byte OP of `sb`
template <int OP> __device__ __forceinline__ f32x4_t mfma_scaled(v8i_t a, v8i_t b, f32x4_t c, int sa, int sb) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, sa, OP, sb);
}

// vmcnt <= n: a load of each of the last n requests may still be on its way
template <int N> __device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(vmcnt_imm(N)); }
// waits until at most `tiles` tiles of PER requests each are (a uniform number up to MOST)
template <int PER, int MOST> __device__ __forceinline__ void wait_tiles(int tiles) {
  if constexpr (MOST <= 0) {
    wait_loads<0>();
  } else {
    if (tiles >= MOST) wait_loads<(PER * MOST > 63 ? 63 : PER * MOST)>();
    else wait_tiles<PER, MOST - 1>(tiles);
  }
}

// four bytes per lane: lane l's land at lds_base + 4 l
__device__ __forceinline__ void load_to_lds4(const void* src, const void* lds_base) {
  const uint32_t l = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_ptr_t)lds_base));
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(l), "v"(src) : "memory");
}

// parts of the queries: bf16 ones in two e4m3 parts, fp32 ones in three bf16 parts; and bf16 parts of the probabilities
template <typename T> struct Parts { static constexpr int q = sizeof(T) == 2 ? 2 : 3, p = sizeof(T) == 2 ? 1 : 3; };

constexpr int ml_floats(int nk, int rows) { return nk > 1 ? 2 * nk * rows : 0; }
__host__ __device__ constexpr size_t quant_lds_bytes(int hd, int nk, int rows, int B, bool paged) {
  const size_t s = static_cast<size_t>(nk) * ring_slots(hd, nk);
  return s * slot_bytes(hd) + s * kScaleSlot + static_cast<size_t>(nk > 1 ? 2 * nk * rows : 0) * sizeof(float) + static_cast<size_t>(attn_sched_words(B)) * sizeof(int) +
         (paged ? static_cast<size_t>(kMaxGroups) * sizeof(int) : 0);
}

template <int HD, typename T, int NK, int NR, int RTW, int KT>
__global__ __launch_bounds__(64 * NK * NR, NK * NR <= 8 ? 2 : (NK * NR + 3) / 4) void k_quant_attn(const QuantAttnArgs a) {
  constexpr int S = ring_slots(HD, NK);
  constexpr int RP = 16 * NR * RTW;               // query rows covered (padded)
  constexpr int kSlot = slot_bytes(HD);
  constexpr int kChunks = HD / 16;                // 16-byte chunks of a row
  constexpr int kKeysPP = 1024 / HD;              // keys of a 1 KB piece
  constexpr int kTileP = kTileKeys / kKeysPP;     // pieces of a K (or V) tile
  constexpr int kPieces = (2 * kTileP + NR - 1) / NR;      // pieces that a wave requests of a tile, at most
  static_assert(NK == 1 || NR * RTW <= S, "a ring's slots hold its sums");
  static_assert(S >= 2 * KT && S % KT == 0, "a step is requested while the one before it is worked on");
  constexpr int kVAhead = NK * NR <= 8 ? 8 : 3;       // V reads in front of their use, as many as the registers allow
  constexpr int kReq = 2 * kTileP / NR + 1;       // requests of a wave per tile, at least
  constexpr bool kCodes = sizeof(T) == 2;         // keys are multiplied as codes
  constexpr int NP = Parts<T>::q, PP = Parts<T>::p;
  constexpr int NM = HD == 128 ? NP : 1;          // block-scaled matrix instructions for 16 keys x 16 rows
  constexpr int kKS = HD / 32;                    // k steps of bf16 ones
  constexpr int kDT = HD / 16;
  extern __shared__ uint4 smem4[];
  char* smem = reinterpret_cast<char*>(smem4);
  char* scales = smem + NK * S * kSlot;
  float* ml_lds = reinterpret_cast<float*>(scales + NK * S * kScaleSlot);
  int* sched_lds = reinterpret_cast<int*>(ml_lds + ml_floats(NK, RP));
  uint32_t* group_lds = reinterpret_cast<uint32_t*>(sched_lds + attn_sched_words(a.B));
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kg = wv / NR, rr = wv % NR;
  const int G = a.G, R = G * a.n_q;
  const AttnTable table = attn_sched_build(a, sched_lds);
  const AttnLine line = attn_sched_line(a, table);
  if (static_cast<int>(blockIdx.x) >= line.W) return;   // the whole workgroup leaves together
  const int x_hi = attn_sched_lo(line, blockIdx.x + 1);
  bool again = false;                             // a segment before this one used the rings
  AttnSeg seg = attn_sched_next(a, table, true, line.pad, attn_sched_lo(line, blockIdx.x), x_hi);
  if (seg.next < x_hi) attn_sched_keep(a, table);
  for (; seg.s1 > seg.s0; seg = attn_sched_next(a, table, false, line.pad, seg.next, x_hi)) {
  attn_sched_publish(a, seg);
  // (what follows from the lane is worked out anew for every segment, and for its end: held through the tiles it is registers)
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));
  const int fr = lane & 15, fq = lane >> 4;
  const int g = seg.g, b = seg.b;
  const int L = __builtin_amdgcn_readfirstlane(seg.L);
  const int s0 = seg.s0, s1 = __builtin_amdgcn_readfirstlane(seg.s1);
  const int ntl = (s1 - s0 + kTileKeys - 1) / kTileKeys;   // tiles of the segment
  const int nit = (ntl + NK - 1) / NK;            // tiles of every ring, at most
  const int mine = (ntl - kg + NK - 1) / NK;      // tiles of this ring
  char* ring = smem + kg * (S * kSlot);
  char* ring_s = scales + kg * (S * kScaleSlot);

  // ---- this wave's query rows (rows past the last one repeat it and are not stored): lane (row, q) holds columns 16 q .. + 15 and, of
  // 128-wide heads, 64 + 16 q .. + 15; in the converted form 32 s + 8 q .. + 7 of every k step s
  constexpr int kQ = HD / 4;                      // columns of a lane
  float x[RTW][kQ];
  uint64_t rowmask[RTW];
#pragma unroll
  for (int t = 0; t < RTW; ++t) {
    const int r = min(16 * (rr * RTW + t) + fr, R - 1);
    const int i = (r * a.g_inv) >> 16;            // r / G
    const T* qp = static_cast<const T*>(a.q) + ((static_cast<size_t>(b) * a.n_q + i) * a.Hq + g * G + (r - i * G)) * HD;
#pragma unroll
    for (int c = 0; c < kQ; c += 4) {
      const T* p = qp + (kCodes ? 16 * fq + (c & 15) + (c >> 4) * 64 : 8 * fq + (c & 7) + (c >> 3) * 32);
      if constexpr (sizeof(T) == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        x[t][c] = __uint_as_float(v.x << 16); x[t][c + 1] = __uint_as_float(v.x & 0xFFFF0000u);
        x[t][c + 2] = __uint_as_float(v.y << 16); x[t][c + 3] = __uint_as_float(v.y & 0xFFFF0000u);
      } else {
        const float4 v = *reinterpret_cast<const float4*>(p);
        x[t][c] = v.x; x[t][c + 1] = v.y; x[t][c + 2] = v.z; x[t][c + 3] = v.w;
      }
    }
    rowmask[t] = a.mask ? a.mask[static_cast<size_t>(b) * a.mask_stride + i] : ((2ull << i) - 1ull);
  }

  // ---- the places of the segment's groups of 16 keys to LDS, in units of 16 rows of the pool (a page is a multiple of 16 entries): loads from there
  // do not count against the vector-memory counter that paces the tile loads, and a wave needs no multiplication for a request.
  const uint32_t group0 = static_cast<uint32_t>(s0) >> 4;
  if (a.paged) {
    const uint32_t per = static_cast<uint32_t>(a.page_size) >> 4;           // groups of a page
    const int ng = (s1 - s0 + 15) >> 4;
    const int32_t* ptab = a.page_table + static_cast<size_t>(b) * a.max_pages;
    for (int i = threadIdx.x; i < ng; i += 64 * NK * NR) {
      const uint32_t at = group0 + i, n = a.page_shift >= 0 ? at >> (a.page_shift - 4) : at / per;
      group_lds[i] = (static_cast<uint32_t>(checked_page(ptab[n], a.n_pages, a.status)) * static_cast<uint32_t>(a.Hkv) + g) * per + (at - n * per);
    }
  }
  if (a.paged || again) __syncthreads();          // the groups are there, and the rings are free of the segment before
  again = true;

  // ---- requests of a tile.  Piece j holds kKeysPP keys from kKeysPP (j % kTileP) on (K, then V), lane l fetches key l / kChunks of them, chunk
  // (l % kChunks) ^ swizzle(key).  A wave has the same pieces of every tile; of an address only the group's place is new.
  const int lkey = lane / kChunks, lpos = lane % kChunks;
  uint64_t k_pool = reinterpret_cast<uint64_t>(a.k), v_pool = reinterpret_cast<uint64_t>(a.v), ks_pool = reinterpret_cast<uint64_t>(a.ks), vs_pool = reinterpret_cast<uint64_t>(a.vs);
  // (selected as values: left alone the compiler selects the arguments' addresses and loads through them for every tile, which waits for all
  // requests in flight)
  asm volatile("" : "+s"(k_pool), "+s"(v_pool), "+s"(ks_pool), "+s"(vs_pool));
  uint64_t piece_at[kPieces];
#pragma unroll
  for (int u = 0; u < kPieces; ++u) {
    const int j = rr + u * NR, key = kKeysPP * (j & (kTileP - 1)) + lkey;
    const bool is_v = j >= kTileP;
    piece_at[u] = (is_v ? v_pool : k_pool) + ((key & 15) * HD + ((lpos ^ (is_v ? swz_v<HD>(key) : swz_k<HD>(key))) << 4));
  }
  // scale bytes: lanes 0..7 four keys' K scales each, lanes 8..15 V scales
  const uint64_t scale_at = (lane & 8 ? vs_pool : ks_pool) + 4 * (lane & 3);
  const uint32_t unit_group = static_cast<uint32_t>((static_cast<uint64_t>(b) * a.Hkv + g) * static_cast<uint64_t>(a.l_max) >> 4) + group0;      // (contiguous)
  auto issue = [&](int it) {
    if (it >= mine) return;                       // uniform per wave
    const int first = kTileKeys * (it * NK + kg); // the tile's first key in the segment
    const int n = s1 - s0 - first;                // keys from there to the end
    uint32_t g0, g1;                              // places of the tile's two groups
    if (a.paged) {
      g0 = group_lds[first >> 4];
      g1 = group_lds[(first >> 4) + (n > 16 ? 1 : 0)];
    } else {
      g0 = unit_group + (first >> 4);
      g1 = g0 + (n > 16 ? 1 : 0);
    }
    char* slot = ring + (it % S) * kSlot;
    if (n >= kTileKeys) {
#pragma unroll
      for (int u = 0; u < kPieces; ++u) {
        const int j = rr + u * NR;
        if (2 * kTileP % NR != 0 && j >= 2 * kTileP) break;
        const uint32_t at = kKeysPP * (j & (kTileP - 1)) & 16 ? g1 : g0;
        load_to_lds16(reinterpret_cast<const void*>(piece_at[u] + static_cast<uint64_t>(at) * (16 * HD)), slot + j * 1024);
      }
    } else {
      // keys past the range repeat the last one and are masked
#pragma unroll
      for (int u = 0; u < kPieces; ++u) {
        const int j = rr + u * NR;
        if (2 * kTileP % NR != 0 && j >= 2 * kTileP) break;
        const int key = kKeysPP * (j & (kTileP - 1)) + lkey, to = min(key, n - 1);
        const bool is_v = j >= kTileP;
        const uint64_t at = (is_v ? v_pool : k_pool) + static_cast<uint64_t>(to & 16 ? g1 : g0) * (16 * HD) + (to & 15) * HD + ((lpos ^ (is_v ? swz_v<HD>(key) : swz_k<HD>(key))) << 4);
        load_to_lds16(reinterpret_cast<const void*>(at), slot + j * 1024);
      }
    }
    // (the bytes behind the last entry are inside the cache: pages and contiguous caches are multiples of 16 entries)
    if (lane < 16) load_to_lds4(reinterpret_cast<const void*>(scale_at + (static_cast<uint64_t>(lane & 4 ? g1 : g0) << 4)), ring_s + (it % S) * kScaleSlot);
  };

  f32x4_t oacc[kDT][RTW];
  float m_run[RTW], l_run[RTW];
#pragma unroll
  for (int t = 0; t < RTW; ++t) {
    m_run[t] = -FLT_MAX;
    l_run[t] = 0.f;
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt) oacc[dt][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const float sl2 = a.scale * 1.44269504088896340736f;    // scores are kept in log2 units

  // ---- the queries' parts.  Codes: a row's scale as in the cache, then four bits at a time; v8i m of a row is the whole of part m (128-wide
  // heads), or parts 0 and 1; scale bytes of instruction m: byte m.
  v8i_t qf[RTW][NM];
  int qs[RTW];
  uint4 qb[RTW][NP][kKS];
#pragma unroll
  for (int t = 0; t < RTW; ++t) {
    if constexpr (kCodes) {
      float big = 0.f;
#pragma unroll
      for (int c = 0; c < kQ; ++c) big = fmaxf(big, fabsf(x[t][c]));
      // (from 5 on, so that the lesser part, four powers of two below, has a scale byte too: of rows below 2^-114 both are exact to 2^-136)
      const int s = min(max(quant_scale_byte(__float_as_uint(quad_row_max(big))), 5), 254);
      const float inv = quant_scale_inverse(s);
#pragma unroll
      for (int c = 0; c < kQ; ++c) x[t][c] *= inv;
#pragma unroll
      for (int p = 0; p < NP; ++p) {
#pragma unroll
        for (int c = 0; c < kQ; c += 4) {
          int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[t][c], x[t][c + 1], 0, false);
          w = __builtin_amdgcn_cvt_pk_fp8_f32(x[t][c + 2], x[t][c + 3], w, true);
          if constexpr (HD == 128) qf[t][p][c / 4] = w;
          else qf[t][0][p * 4 + c / 4] = w;
          if (p + 1 < NP) {
            const v2f_t lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
            x[t][c] = (x[t][c] - lo[0]) * 16.f; x[t][c + 1] = (x[t][c + 1] - lo[1]) * 16.f;
            x[t][c + 2] = (x[t][c + 2] - hi[0]) * 16.f; x[t][c + 3] = (x[t][c + 3] - hi[1]) * 16.f;
          }
        }
      }
      // (lanes q hold the scales of products 32 q .. + 31)
      qs[t] = HD == 128 ? s | (s - 4) << 8 : s - 4 * (fq >> 1);
    } else {
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int s = 0; s < kKS; ++s) {
          float* y = x[t] + 8 * s;
          qb[t][p][s] = make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
          float hi[8];
          unpack16(qb[t][p][s], hi);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] -= hi[e];
        }
    }
  }
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));       // from here on vmcnt counts tile requests only
#pragma unroll 1
  for (int it = 0; it < S - KT; ++it) issue(it);

  // a lane's part of the operand addresses
  // (one for K and one for V, a read is the exclusive or with its number: held in registers they are a dozen)
  int k_at = fr * HD + (kCodes ? (fq ^ swz_k<HD>(fr)) << 4 : (((fq >> 1) ^ swz_k<HD>(fr)) << 4) + (fq & 1) * 8);
  const int v_key = (fr >> 1) < 4 ? 4 * fq + (fr >> 1) : 16 + 4 * fq + (fr >> 1) - 4;
  int v_at = v_key * HD + (fr & 1) * 8 + (swz_v<HD>(v_key) << 4);

  uint4 kreg[2][HD / 64];
  int ksc[2];
  v2i_t vreg[kDT];
  uint32_t ksw[2], vsw[2];
  auto read_k = [&](int it) {
    const char* k_lds = ring + (it % S) * kSlot;
    const char* s_lds = ring_s + (it % S) * kScaleSlot;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if constexpr (kCodes) {
        // chunks q and, of 128-wide heads, q + 4 of key 16 j + row   (swz_k(16 + key) == swz_k(key))
#pragma unroll
        for (int c = 0; c < HD / 64; ++c) kreg[j][c] = *reinterpret_cast<const uint4*>(k_lds + (k_at ^ (c << 6)) + j * 16 * HD);
        ksc[j] = *reinterpret_cast<const uint8_t*>(s_lds + 16 * j + fr);
      } else {
        // eight codes of every k step
#pragma unroll
        for (int s = 0; s < kKS; ++s) {
          const uint2 c = *reinterpret_cast<const uint2*>(k_lds + (k_at ^ (s << 5)) + j * 16 * HD);
          if (s & 1) { kreg[j][s >> 1].z = c.x; kreg[j][s >> 1].w = c.y; }
          else { kreg[j][s >> 1].x = c.x; kreg[j][s >> 1].y = c.y; }
        }
        ksw[j] = *reinterpret_cast<const uint32_t*>(s_lds + 16 * j + 4 * fq);
      }
    }
  };
  auto read_v = [&](int it, int dt) {
    vreg[dt] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i_t)(lds_ptr_t)(ring + (it % S) * kSlot + kSlot / 2 + (v_at ^ (dt << 4))));
  };
  auto read_vs = [&](int it) {
#pragma unroll
    for (int j = 0; j < 2; ++j) vsw[j] = *reinterpret_cast<const uint32_t*>(ring_s + (it % S) * kScaleSlot + kTileKeys + 16 * j + 4 * fq);
  };
#pragma unroll 1
  for (int it0 = 0; it0 < nit; it0 += KT) {
    // this wave's pieces of the KT tiles from it0 on have landed once at most those of the tiles requested behind them are outstanding (loads
    // return in order); behind the barrier everyone's have, and the slots of the KT tiles before are free
    wait_tiles<kReq, S - 2 * KT>(min(it0 + S - KT, mine) - (it0 + KT));
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    if constexpr (NR > 1) __builtin_amdgcn_s_barrier();
    else __builtin_amdgcn_s_waitcnt(0xC07F);      // lgkmcnt(0): of one wave, the tiles before are read
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll 1
    for (int k = 0; k < KT; ++k) issue(it0 + S - KT + k);
#pragma unroll 1
    for (int it = it0; it < min(it0 + KT, mine); ++it) {
    read_k(it);
    read_vs(it);
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" : "+v"(k_at), "+v"(v_at));
    const int t0 = s0 + kTileKeys * (it * NK + kg);

    // ---- S^T = K Q^T, both halves of 16 keys
    f32x4_t sacc[2][RTW];
    if constexpr (kCodes) {
      v8i_t kf[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint4 lo = kreg[j][0], hi = kreg[j][HD / 64 - 1];          // (64-wide heads: the same codes twice)
        kf[j] = v8i_t{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
      }
#pragma unroll
      for (int p = NM - 1; p >= 0; --p)                // (the lesser part first, and all of it: an accumulator's second product waits for the first)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int t = 0; t < RTW; ++t) {
            const f32x4_t c = p == NM - 1 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : sacc[j][t];
            sacc[j][t] = p == 1 ? mfma_scaled<1>(kf[j], qf[t][p], c, ksc[j], qs[t]) : mfma_scaled<0>(kf[j], qf[t][p], c, ksc[j], qs[t]);
          }
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float ks[4] = {quant_scale<0>(ksw[j]), quant_scale<1>(ksw[j]), quant_scale<2>(ksw[j]), quant_scale<3>(ksw[j])};
        f32x4_t part[RTW][NP];
#pragma unroll
        for (int t = 0; t < RTW; ++t)
#pragma unroll
          for (int p = 0; p < NP; ++p) part[t][p] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < kKS; ++s) {
          const uint4 r = kreg[j][s >> 1];
          const uint32_t c0 = s & 1 ? r.z : r.x, c1 = s & 1 ? r.w : r.y;
          const uint4 ka = make_uint4(two_bf16(c0, false), two_bf16(c0, true), two_bf16(c1, false), two_bf16(c1, true));
#pragma unroll
          for (int t = 0; t < RTW; ++t)
#pragma unroll
            for (int p = 0; p < NP; ++p)
              part[t][p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, ka), __builtin_bit_cast(bf16x8_t, qb[t][p][s]), part[t][p], 0, 0, 0);
        }
#pragma unroll
        for (int t = 0; t < RTW; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) sacc[j][t][e] = ((part[t][2][e] + part[t][1][e]) + part[t][0][e]) * ks[e];
      }
    }
    const float vs[8] = {quant_scale<0>(vsw[0]), quant_scale<1>(vsw[0]), quant_scale<2>(vsw[0]), quant_scale<3>(vsw[0]),
                         quant_scale<0>(vsw[1]), quant_scale<1>(vsw[1]), quant_scale<2>(vsw[1]), quant_scale<3>(vsw[1])};
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int dt = 0; dt < min(kVAhead, kDT); ++dt) read_v(it, dt);
    __builtin_amdgcn_sched_barrier(0);

    // ---- online softmax; lane (row, q) owns keys t0 + 16 j + 4 q + e of its row.  The reference of the exponents moves only when a score
    // exceeds its row's by more than kSlack.  Probabilities of one bf16 part have none: the largest is then 1, which bf16 holds, and its rounding
    // is what a peaked row's error would be made of: a result whose value is all in that key's is off by half a step, with a slack by up to 2.5.
    // (Root mean square error against 64 bits, beyond that of fp32 arithmetic rounded to bf16, with a slack of 8 / none: 8 sequences of 300 .. 900, 72
    // rows 3.5 / 0.5 %; 8 of 2048 .. 16384, 28 rows 2.7 / 0.25 %, 16 rows 1.1 / 0.3 %; 64-wide, 8 of 1000 .. 8000, 64 rows 1.4 / 0.3 %; with two parts
    // 0.1 % everywhere.  What it costs, 8 sequences of 2048 .. 16384: up to 16 rows nothing, 28 rows 34.2 -> 34.7 us, 48 rows 40.6 -> 41.8, 72 rows 57.2 ->
    // 59.8, 128 rows 71.2 -> 76.2; 16 of 8192 .. 32768, 72 rows 188 -> 194.  Two parts: 35.8, 44.5, 63.8, 83.6; 223.)
    constexpr float kSlack = PP == 1 ? 0.f : 8.f;
    const bool plain = t0 + kTileKeys <= min(L, s1) && sl2 > 0.f;
    float z[RTW][8], unit = sl2;
#pragma unroll
    for (int t = 0; t < RTW; ++t)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) z[t][4 * j + e] = sacc[j][t][e];
    if (!plain) {
      unit = 1.f;
#pragma unroll
      for (int t = 0; t < RTW; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int p = t0 + 16 * (e >> 2) + 4 * fq + (e & 3);
          bool vis = p < s1;
          if (vis && p >= L) vis = (rowmask[t] >> (p - L)) & 1ull;
          z[t][e] = vis ? z[t][e] * sl2 : -INFINITY;
        }
    }
    float mt[RTW];
    bool grown = false;
#pragma unroll
    for (int t = 0; t < RTW; ++t) {
      mt[t] = max3_nan(max3_nan(z[t][0], z[t][1], z[t][2]), max3_nan(z[t][3], z[t][4], z[t][5]), max_nan(z[t][6], z[t][7])) * unit;
      grown |= mt[t] > m_run[t] + kSlack;
    }
    if (__builtin_amdgcn_ballot_w64(grown) != 0ull) {            // (one test for all of a wave's rows, so that what follows is one stretch of code)
#pragma unroll
      for (int t = 0; t < RTW; ++t) {
        const float m_new = fmaxf(m_run[t], quad_row_max(mt[t]));
        const float al = __builtin_amdgcn_exp2f(m_run[t] - m_new);
        m_run[t] = m_new;
        l_run[t] *= al;
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt) {
          oacc[dt][t][0] *= al; oacc[dt][t][1] *= al;
          oacc[dt][t][2] *= al; oacc[dt][t][3] *= al;
        }
      }
    }
    uint4 pf[RTW][PP];
#pragma unroll
    for (int t = 0; t < RTW; ++t) {
      float pr[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) pr[e] = __builtin_amdgcn_exp2f(fmaf(z[t][e], unit, -m_run[t]));
      l_run[t] += ((pr[0] + pr[1]) + (pr[2] + pr[3])) + ((pr[4] + pr[5]) + (pr[6] + pr[7]));
#pragma unroll
      for (int e = 0; e < 8; ++e) pr[e] *= vs[e];
#pragma unroll
      for (int p = 0; p < PP; ++p) {
        pf[t][p] = make_uint4(pack_bf16x2(pr[0], pr[1]), pack_bf16x2(pr[2], pr[3]), pack_bf16x2(pr[4], pr[5]), pack_bf16x2(pr[6], pr[7]));
        if (p + 1 < PP) {
          float hi[8];
          unpack16(pf[t][p], hi);
#pragma unroll
          for (int e = 0; e < 8; ++e) pr[e] -= hi[e];
        }
      }
    }

    // ---- O^T += V^T P^T: a column tile is converted while the one before it is multiplied, into registers of its own
    auto convert = [&](int dt) { return make_uint4(two_bf16(vreg[dt][0], false), two_bf16(vreg[dt][0], true), two_bf16(vreg[dt][1], false), two_bf16(vreg[dt][1], true)); };
    uint4 va = convert(0), vb;
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt) {
      if (dt + kVAhead < kDT) read_v(it, dt + kVAhead);
      if (dt + 1 < kDT) vb = convert(dt + 1);
      __builtin_amdgcn_sched_barrier(0);          // (all conversions first would take four registers for every one of these)
#pragma unroll
      for (int p = PP - 1; p >= 0; --p)
#pragma unroll
        for (int t = 0; t < RTW; ++t)
          oacc[dt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, va), __builtin_bit_cast(bf16x8_t, pf[t][p]), oacc[dt][t], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      va = vb;
    }
    }
  }

  // ---- the segment's partial result.  Several rings: each leaves its sums in its own slots (16-byte pieces of a row swizzled), every wave adds some
  // rows, in the order of the rings.
  int lane_e = threadIdx.x & 63;
  asm volatile("" : "+v"(lane_e));
  const int fr_e = lane_e & 15, fq_e = lane_e >> 4;
  const size_t unit = static_cast<size_t>(blockIdx.x) + static_cast<size_t>(b) * a.Hkv + g;   // partial slot of segment (w, u)
#pragma unroll
  for (int t = 0; t < RTW; ++t) l_run[t] = quad_row_sum(l_run[t]);
  if constexpr (NK == 1) {
#pragma unroll
    for (int t = 0; t < RTW; ++t) {
      const int r = 16 * (rr * RTW + t) + fr_e;
      if (r >= R) continue;
      if (fq_e == 0) *reinterpret_cast<float2*>(a.part_ml + (unit * R + r) * 2) = make_float2(m_run[t], l_run[t]);
      float* dst = a.part_o + (unit * R + r) * HD + 4 * fq_e;
#pragma unroll
      for (int dt = 0; dt < kDT; ++dt) *reinterpret_cast<float4*>(dst + 16 * dt) = make_float4(oacc[dt][t][0], oacc[dt][t][1], oacc[dt][t][2], oacc[dt][t][3]);
    }
    __syncthreads();                              // (the schedule's table is there for the next segment)
  } else {
    if constexpr (NR > 1) __syncthreads();        // the ring's last tile is read by all its waves
#pragma unroll
    for (int t = 0; t < RTW; ++t) {
      const int r = 16 * (rr * RTW + t) + fr_e;
      if (fq_e == 0) *reinterpret_cast<float2*>(ml_lds + 2 * (kg * RP + r)) = make_float2(m_run[t], l_run[t]);
#pragma unroll
      for (int dt = 0; dt < kDT; ++dt)
        *reinterpret_cast<float4*>(ring + r * (4 * HD) + (((4 * dt + fq_e) ^ fr_e) << 4)) = make_float4(oacc[dt][t][0], oacc[dt][t][1], oacc[dt][t][2], oacc[dt][t][3]);
    }
    __syncthreads();
    constexpr int C4 = HD / 4, RPW = 64 / C4;     // 16-byte pieces of a row, rows that a wave adds at a time
    const int c4 = lane_e % C4;
#pragma unroll 1
    for (int r = RPW * wv + lane_e / C4; r < R; r += RPW * NK * NR) {
      float2 ml[NK];
      float4 o[NK];
#pragma unroll
      for (int k = 0; k < NK; ++k) {
        ml[k] = *reinterpret_cast<const float2*>(ml_lds + 2 * (k * RP + r));
        o[k] = *reinterpret_cast<const float4*>(smem + k * (S * kSlot) + r * (4 * HD) + ((c4 ^ (r & 15)) << 4));
      }
      float mm = ml[0].x;
#pragma unroll
      for (int k = 1; k < NK; ++k) mm = fmaxf(mm, ml[k].x);
      float sum = 0.f;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < NK; ++k) {
        const float f = __builtin_amdgcn_exp2f(ml[k].x - mm);
        sum = fmaf(f, ml[k].y, sum);
        v.x = fmaf(f, o[k].x, v.x); v.y = fmaf(f, o[k].y, v.y);
        v.z = fmaf(f, o[k].z, v.z); v.w = fmaf(f, o[k].w, v.w);
      }
      *reinterpret_cast<float4*>(a.part_o + (unit * R + r) * HD + 4 * c4) = v;
      if (c4 == 0) *reinterpret_cast<float2*>(a.part_ml + (unit * R + r) * 2) = make_float2(mm, sum);
    }
  }
  }
}

// ---------------------------------------------------------------------------------------------------- merging the segments

// Row of entry p of a unit in the pools.
__device__ __forceinline__ size_t quant_entry(const QuantAttnArgs& a, int b, int g, int p) {
  if (!a.paged) return (static_cast<size_t>(b) * a.Hkv + g) * a.l_max + p;
  const int n = static_cast<int>(static_cast<uint32_t>(p) / static_cast<uint32_t>(a.page_size));
  const int page = checked_page(a.page_table[static_cast<size_t>(b) * a.max_pages + n], a.n_pages, a.status);
  return (static_cast<size_t>(page) * a.Hkv + g) * a.page_size + (p - n * a.page_size);
}

__device__ __forceinline__ void two_f32(uint32_t codes, bool hi, float* f) {
  const v2f_t v = hi ? __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(codes), true) : __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(codes), false);
  f[0] = v[0];
  f[1] = v[1];
}

// One output row again, by one wave, key by key and with hidden keys left out.  The matrix instructions multiply every value of a tile with a
// probability, hidden ones with 0, so that a NaN among entries that a row does not see (a block's entries that were never written)
// reaches its sums, and infinite products of queries in parts are NaN: rows whose result is not finite are taken here, and are NaN
// only where what they see makes them so.
template <typename T, int D>
__device__ __forceinline__ void quant_row_again(const QuantAttnArgs& a, int b, int i, int h) {
  constexpr int LPK = D / 8, KPW = 64 / LPK;      // lanes of a key, keys of a wave
  const int lane = threadIdx.x & 63;
  const int kq = lane / LPK, c = lane % LPK;
  const int g = h / a.G, L = attn_ctx_len(a, b), n = L + a.n_blk;
  const size_t row = ((static_cast<size_t>(b) * a.n_q + i) * a.Hq + h) * D;
  const uint64_t seen = a.mask ? a.mask[static_cast<size_t>(b) * a.mask_stride + i] : ((2ull << i) - 1ull);
  float q[8], acc[8], m = -INFINITY, sum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    q[e] = Elem<T>::load(static_cast<const T*>(a.q) + row + 8 * c + e);
    acc[e] = 0.f;
  }
#pragma unroll 1
  for (int p0 = 0; p0 < n; p0 += KPW) {
    const int p = p0 + kq;
    const bool vis = p < n && (p < L || (seen >> (p - L) & 1ull));
    const size_t at = quant_entry(a, b, g, min(p, n - 1));
    const uint2 kr = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.k) + at * D + 8 * c);
    const uint2 vr = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.v) + at * D + 8 * c);
    const float ks = quant_scale<0>(static_cast<const uint8_t*>(a.ks)[at]), vs = quant_scale<0>(static_cast<const uint8_t*>(a.vs)[at]);
    float kf[8], vf[8], x = 0.f;
    two_f32(kr.x, false, kf); two_f32(kr.x, true, kf + 2); two_f32(kr.y, false, kf + 4); two_f32(kr.y, true, kf + 6);
    two_f32(vr.x, false, vf); two_f32(vr.x, true, vf + 2); two_f32(vr.y, false, vf + 4); two_f32(vr.y, true, vf + 6);
#pragma unroll
    for (int e = 0; e < 8; ++e) x = fmaf(q[e], kf[e] * ks, x);
#pragma unroll
    for (int o = 1; o < LPK; o <<= 1) x += __shfl_xor(x, o, 64);
    x = vis ? x * a.scale : -INFINITY;
    float mt = x;
#pragma unroll
    for (int o = LPK; o < 64; o <<= 1) mt = fmaxf(mt, __shfl_xor(mt, o, 64));
    const float m_new = fmaxf(m, mt);
    float al = 1.f, pr = 0.f;
    if (m_new != -INFINITY) {
      al = m == -INFINITY ? 0.f : expf(m - m_new);
      pr = expf(x - m_new);
    }
    if (x != x) pr = x;
    m = m_new;
    sum = fmaf(sum, al, pr);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = fmaf(pr, vis ? vf[e] * vs : 0.f, acc[e] * al);
  }
#pragma unroll
  for (int o = LPK; o < 64; o <<= 1) {
    sum += __shfl_xor(sum, o, 64);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += __shfl_xor(acc[e], o, 64);
  }
  if (kq == 0) {
    T* dst = static_cast<T*>(a.out) + row + 8 * c;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float v = sum == 0.f ? 0.f : acc[e] / sum;
      if constexpr (sizeof(T) == 2) dst[e] = static_cast<bf16_t>(pack_bf16x2(v, v));
      else dst[e] = v;
    }
  }
}

// Exact log-sum-exp merge of the segments of one (sequence, query, head), WPR waves per output row.  Latency is all there is: the unit's
// first and last workgroup, one round to memory for (max, sum) pairs and the first partial outputs, a meeting of the waves.
// Lane s of every wave holds the weights of segments s, s + 64, ..; half a wave (128-wide heads; a quarter of 64-wide ones) has a segment's row.
constexpr int kEarly = 6;        // partial outputs requested with the (max, sum) pairs, per group of lanes

template <typename T, int D, int WPR>
__global__ __launch_bounds__(256) void k_quant_combine(const QuantAttnArgs a) {
  constexpr int C4 = D / 4, GPW = 64 / C4, NG = WPR * GPW;     // float4 columns; groups of a wave and of a row
  __shared__ float4 gs[WPR > 1 ? NG : 1][C4];
  arguments_at_once<sizeof(QuantAttnArgs)>();
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = WPR == 4 ? static_cast<int>(blockIdx.x) : static_cast<int>(blockIdx.x) * 4 + wv;
  if (row >= a.B * a.n_q * a.Hq) return;          // (one wave per row)
  const int b = row / (a.n_q * a.Hq), ih = row - b * (a.n_q * a.Hq), i = ih / a.Hq, h = ih - i * a.Hq;
  const int R = a.G * a.n_q, g = h / a.G, r = i * a.G + h - g * a.G;
  typedef const __attribute__((address_space(4))) int* words_t;           // (scalar loads: nothing writes these words meanwhile)
  const int u = b * a.Hkv + g;
  const words_t ends = (words_t)a.sched + 2 * u;
  const int w_first = ends[0], n_seg = ends[1] - w_first + 1;
  const size_t slot = static_cast<size_t>(w_first) + u;
  const float* ml_p = a.part_ml + (slot * R + r) * 2;
  const size_t ml_step = 2 * static_cast<size_t>(R), po_step = static_cast<size_t>(R) * D;
  const int sg = (WPR == 4 ? wv * GPW : 0) + lane / C4, c4 = lane % C4;
  const float* po = a.part_o + (slot * R + r) * D + c4 * 4;
  float2 ml = *reinterpret_cast<const float2*>(ml_p + min(lane, n_seg - 1) * ml_step);
  float4 o[kEarly];
#pragma unroll
  for (int k = 0; k < kEarly; ++k) o[k] = *reinterpret_cast<const float4*>(po + min(sg + k * NG, n_seg - 1) * po_step);
  float mmax = ml.x;
  for (int s = 64 + lane; s < n_seg; s += 64) mmax = fmaxf(mmax, ml_p[s * ml_step]);
  mmax = wave_max_dpp(mmax);
  float den = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s0 = 0; s0 < n_seg; s0 += 64) {
    if (s0 > 0) ml = *reinterpret_cast<const float2*>(ml_p + min(s0 + lane, n_seg - 1) * ml_step);
    const float w = s0 + lane < n_seg ? __builtin_amdgcn_exp2f(ml.x - mmax) : 0.f;
    den += w != 0.f || ml.y != ml.y ? w * ml.y : 0.f;             // (a NaN counts whatever its weight)
    const int n = min(64, n_seg - s0);
    for (int sb = 0; sb < n; sb += kEarly * NG) {                 // (uniform)
      const int s = sb + sg;
      if (s0 + sb > 0) {
#pragma unroll
        for (int k = 0; k < kEarly; ++k) o[k] = *reinterpret_cast<const float4*>(po + (s0 + min(s + k * NG, n - 1)) * po_step);
      }
#pragma unroll
      for (int k = 0; k < kEarly; ++k) {
        float wk = __shfl(w, min(s + k * NG, n - 1), 64);
        if (s + k * NG >= n) wk = 0.f;
        if (wk != 0.f) {
          acc.x = fmaf(wk, o[k].x, acc.x); acc.y = fmaf(wk, o[k].y, acc.y);
          acc.z = fmaf(wk, o[k].z, acc.z); acc.w = fmaf(wk, o[k].w, acc.w);
        }
      }
    }
  }
  den = wave_sum_dpp(den);
  if constexpr (WPR > 1) {
    gs[sg][c4] = acc;
    __syncthreads();
    if (wv > 0) return;
    acc = gs[0][c4];                              // (the first wave's lanes all hold the row then, group 0 stores it)
#pragma unroll
    for (int k = 1; k < NG; ++k) { acc.x += gs[k][c4].x; acc.y += gs[k][c4].y; acc.z += gs[k][c4].z; acc.w += gs[k][c4].w; }
  } else {
#pragma unroll
    for (int off = C4; off < 64; off <<= 1) {
      acc.x += __shfl_xor(acc.x, off, 64); acc.y += __shfl_xor(acc.y, off, 64);
      acc.z += __shfl_xor(acc.z, off, 64); acc.w += __shfl_xor(acc.w, off, 64);
    }
  }
  // a row that sees nothing has a sum of 0 and is all zeros
  const float inv = den == 0.f ? 0.f : 1.0f / den;
  if constexpr (sizeof(T) == 2) {
    acc.x *= inv; acc.y *= inv; acc.z *= inv; acc.w *= inv;
  } else if (den != 0.f) {
    acc.x /= den; acc.y /= den; acc.z /= den; acc.w /= den;
  }
  const float all = (acc.x + acc.y) + (acc.z + acc.w);
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(fabsf(all) < INFINITY)) != 0ull, 0)) {
    quant_row_again<T, D>(a, b, i, h);
    return;
  }
  if (lane < C4) {
    T* dst = static_cast<T*>(a.out) + static_cast<size_t>(row) * D + c4 * 4;
    // (as bytes: the caller's buffer may begin at any element)
    if constexpr (sizeof(T) == 2) {
      const uint2 v = make_uint2(pack_bf16x2(acc.x, acc.y), pack_bf16x2(acc.z, acc.w));
      __builtin_memcpy(dst, &v, sizeof(v));
    } else {
      __builtin_memcpy(dst, &acc, sizeof(acc));
    }
  }
}

// ---------------------------------------------------------------------------------------------------- launches

int row_tiles(const QuantAttnArgs& a) { return (a.G * a.n_q + 15) / 16; }

template <int HD, typename T, int NK, int NR, int RTW, int KT>
hipError_t launch_one(const QuantAttnArgs& a, hipStream_t s) {
  static_assert(quant_lds_bytes(HD, NK, 16 * NR * RTW, kAttnMaxSeqs, true) <= 160 * 1024, "the LDS of a compute unit");
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_quant_attn<HD, T, NK, NR, RTW, KT>), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL((k_quant_attn<HD, T, NK, NR, RTW, KT>), dim3(a.wgrid), dim3(64 * NK * NR), quant_lds_bytes(HD, NK, 16 * NR * RTW, a.B, a.paged != 0), s, a);
  return hipGetLastError();
}

// The form by the number of 16-row tiles: the fewest waves that hold all rows as one ring's, and as many rings as sixteen waves and the LDS of
// a compute unit take.  One wave of a SIMD alone issues every 5.3 cycles, four together every 2.6 to 4.4, so twelve to sixteen waves are
// wanted, evenly over the four SIMDs (five tiles on two rings, three waves to some SIMDs and two to others: 61.5 us, not 57.3); a wave of two tiles (from seven on) shares the conversion of V.  Microseconds of a call over 8 sequences of 2048 .. 16384 tokens,
// 8 KV heads, 128-wide (64-wide), against the next form's at the same rows:
//   rows 16: 31.7, not 34.0 (20.5, 26.5)   28: 34.7, 39.7 (27.0, 31.6)   48: 42.1, 47.4 (32.7, 35.6)   64: 48.6, 58.6 (36.7, 41.2)
//        72: 59.3, 66.3 (42.4, 46.1)   96: 66.9, 74.6 (47.2, 52.5)   128: 76.8, 78.2 with eight waves of one tile (54.3, 55.6)
// Probabilities are one bf16 part, off by half a step (2^-8) at most, as the results are rounded anyway: with the largest of a row exact (kSlack) the
// error against 64 bits is 0.1 to 0.5 % above that of fp32 arithmetic rounded to bf16 (3 to 4 % where a row sees some fifty keys), with two parts
// 0.1 %, at 35.8 us for 28 rows and 63.8 for 72.  With a slack of 8: a step of two tiles (four of 64-wide heads) halves the barriers where the ring's slots
// allow it: 96 rows 64.6 -> 62.1 (48.8 -> 46.2), 112 rows 71.6 -> 68.9; below it gains nothing or costs (48 rows 40.8 -> 43.0).
template <int HD> hipError_t launch_bf16(const QuantAttnArgs& a, hipStream_t s) {
  constexpr int K2 = HD == 64 ? 4 : 2;            // tiles of a step
  switch (row_tiles(a)) {
    case 1: return launch_one<HD, bf16_t, 8, 1, 1, 1>(a, s);
    case 2: return launch_one<HD, bf16_t, 4, 2, 1, 1>(a, s);
    case 3: return launch_one<HD, bf16_t, 4, 3, 1, 1>(a, s);
    case 4: return launch_one<HD, bf16_t, 4, 4, 1, 1>(a, s);
    case 5: return launch_one<HD, bf16_t, 3, 5, 1, HD == 64 ? 4 : 1>(a, s);
    case 6: return launch_one<HD, bf16_t, 2, 6, 1, K2>(a, s);
    default: return launch_one<HD, bf16_t, 2, 4, 2, K2>(a, s);
  }
}

// fp32: three parts of queries and probabilities take 172 to 187 registers of a lane, more than twelve or sixteen waves have; four to eight waves (eight
// for one or two row tiles, which would fit, were not measured).  8 sequences of 500 .. 4000 tokens, 128-wide, against the
// form of twice the rows: 16 rows 18.1 us, not 24.6; 28 rows 25.3, 31.5; 64 rows 35.6, 49.9.  64-wide: 28 rows 18.9, 24.7; 64 rows 27.1, 34.8.
hipError_t launch_f32(const QuantAttnArgs& a, hipStream_t s) {
  const int tiles = row_tiles(a);
  if (a.d == 64) return tiles <= 2 ? launch_one<64, float, 4, 1, 2, 1>(a, s) : tiles <= 4 ? launch_one<64, float, 2, 2, 2, 1>(a, s) : launch_one<64, float, 2, 4, 2, 1>(a, s);
  if (tiles <= 1) return launch_one<128, float, 4, 1, 1, 1>(a, s);
  if (tiles <= 2) return launch_one<128, float, 2, 2, 1, 1>(a, s);
  return tiles <= 4 ? launch_one<128, float, 2, 4, 1, 1>(a, s) : launch_one<128, float, 1, 8, 1, 1>(a, s);
}

// Four waves to an output row while the rows are few: latency is what counts then (one sequence, 28 rows a head: 12.0 us a call, not 13.0);
// one wave where there are enough rows to fill the chip (8 sequences of 28 rows a head: 36.3 us, not 38.2; of 96 rows: 62.1, 69.6).
template <typename T, int D> hipError_t launch_combine(const QuantAttnArgs& a, hipStream_t s) {
  const int64_t units = static_cast<int64_t>(a.B) * a.Hkv, rows = static_cast<int64_t>(a.B) * a.n_q * a.Hq;
  if (rows * units > 256 * static_cast<int64_t>(a.wgrid)) hipLaunchKernelGGL((k_quant_combine<T, D, 1>), dim3(static_cast<unsigned>((rows + 3) / 4)), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_quant_combine<T, D, 4>), dim3(static_cast<unsigned>(rows)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

bool quant_attn_plan(QuantAttnArgs& a, int num_cus) {
  // Not kOnePart, whose launches of middling size spread over 256 workgroups because shorter segments are nearer: with the largest probability of a row
  // exact it makes no difference (six shapes of 3 to 8 sequences of 300 to 4000 entries: errors within 0.03 % of each other, times within 1.5 %).
  a.use_mfma = kTwoPart;
  a.G = a.Hq / a.Hkv;
  a.g_inv = (65536 + a.G - 1) / a.G;
  // a workgroup's start at a unit costs some eight granules: with 4, 8, 14 the 8 sequences of 28 rows took 36.9, 34.7, 34.8 us
  a.pad = 8;
  a.wide_from = 2400;                             // (1000 .. 5000 are alike)
  a.page_shift = (a.page_size & (a.page_size - 1)) == 0 ? 31 - __builtin_clz(static_cast<unsigned>(a.page_size)) : -1;
  if (a.B > kAttnMaxSeqs || a.l_max < a.n_blk) return false;
  const int64_t units = static_cast<int64_t>(a.B) * a.Hkv;
  if (units * a.G * a.n_q > kLaunchWaves) return false;            // (the merge: a wave per row, of as many as that)
  const int64_t gmax = (a.l_max + kAttnGran - 1) / kAttnGran;      // granules of the longest possible unit
  if (units * (gmax + a.pad) >= (1ll << 30)) return false;
  const AttnLine line = attn_sched_line(static_cast<int>(a.B * gmax), a.B, a.Hkv, a.pad, a.wide_from, 0, num_cus);
  int64_t w = line.W;
  if (line.T > kAttnSpread && w < kAttnSpread) w = std::min<int64_t>(kAttnSpread, num_cus);   // (fewer granules may take more workgroups)
  if (a.paged) {                                  // a segment's groups have to fit LDS
    const int64_t seg_gran = kMaxGroups * 16 / kAttnGran;
    w = std::max(w, (line.T + seg_gran - 1) / seg_gran);
  }
  if (w > kAttnMaxGrid) return false;
  a.wgrid = static_cast<int>(w);
  return true;
}

hipError_t launch_quant_attn(const QuantAttnArgs& a, hipStream_t s) {
  const hipError_t e = a.dtype == 0 ? launch_f32(a, s) : a.d == 128 ? launch_bf16<128>(a, s) : launch_bf16<64>(a, s);
  if (e != hipSuccess) return e;
  if (a.dtype == 0) return a.d == 128 ? launch_combine<float, 128>(a, s) : launch_combine<float, 64>(a, s);
  return a.d == 128 ? launch_combine<bf16_t, 128>(a, s) : launch_combine<bf16_t, 64>(a, s);
}

}  // namespace sx
