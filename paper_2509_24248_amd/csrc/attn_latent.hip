// Verification attention over a latent cache: an entry is one vector of LD + 64 values, the key of every query head whole and the value with its
// first LD, so all R = n_q_heads n_q query rows of a sequence share it.
//
//   s_j = scale q . (c_j | k_j),  o = sum_j softmax_j(s) c_j          2 (2 LD + 64) operations a row and entry of (LD + 64) e bytes
//
// Read once, an entry has 2 R (2 LD + 64) / (LD + 64) operations an element: up to some 80 rows the bytes take longer, beyond that the products.
//
// The rows of a sequence are cut into blocks; a workgroup takes an equal share of all keys of all (sequence, block) units (attn_sched.hpp, the blocks in the place
// of KV heads).  Inside it the tiles of 32 keys (fp32: 16) lie in LDS once, as they lie in memory, and are read twice from there:
//   S^T = C Q^T    : A operand = entries (row = key), B operand = the rows' queries, held in registers;
//   softmax        : online, per wave, in log2 units;
//   O^T += C^T P^T : A operand = the same tile by columns (ds_read_b64_tr_b16; fp32: plain reads, a key's sixteen columns to sixteen lanes), B operand = P^T
//                    straight from the softmax registers.
// fp32 uses the fp32 matrix instructions: neither entries nor probabilities lose a digit.
//
// A workgroup has four waves, one per SIMD with all of its registers.  Tiles are brought in by direct global -> LDS loads, up to four slots ahead.  Rows of a block:
//   16 or 32: four rings of one wave or two of two, each with keys of its own, added at the end in their order;
//   64      : one ring of four waves, sixteen rows each (fp32; bf16 in software-pipelined form);
//   128     : bf16, two tiles of sixteen rows a wave: 256 registers of accumulators and 144 of queries.
// Partial results go to memory as the accumulators lie (1 KB for 16 rows x 16 columns: one store instruction) and are merged by a second kernel.
//
// Measured (whole calls, LD = 512, bf16): 16 sequences x 16448 entries, 128 rows, 303 MB and 73 GFLOP: 97 us, 3.1 TB/s and 755 TFLOP/s (a library product of 8192 reaches 1257).
// Beyond some 80 rows no unit is full: of the cycles of the attention kernel over 16 contexts of 8192 to 32768 entries the matrix instructions are busy for 45 %, vector instructions for 24, LDS for
// 23, and 23 are spent waiting, at 1.6 GHz, where the power limit holds the clock.  With one wave to a SIMD (its accumulators are half of the registers) nothing fills what the order of that wave's
// instructions leaves open.  The merge is 15 us of such a call's 120.
#include "attn_sched.hpp"
#include "common.hpp"
#include "kernels.hpp"
#include "stream.hpp"

#include <float.h>
#include <limits.h>
#include <algorithm>

namespace sx {

namespace {

constexpr int kLds = 160 * 1024;
constexpr int kPe = kLatentRope;

typedef short s16x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

template <typename T> struct Tile;
// A tile lies in LDS in groups of 8 keys (fp32: 4), a group in 1 KB blocks of 128 bytes (256) of each of them: what one load instruction brings in, lane l the 16-byte chunk
// l % 8 (16) of key l / 8 (16), so that a lane's source is one offset for all blocks.  The chunks of a key's part are swizzled.  A row read takes a chunk of sixteen keys, four lanes' worth of
// chunks at a time, and the LDS serves the lanes 0-3, 12-15, 20-27 of each 32 together, then the others: keys 0-3 and 12-15 of one chunk with 4-11 of its neighbour.  A transpose read takes an
// even chunk and the next of eight keys.  With 2 (key / 2 % 4) + key / 4 % 2 neither has two lanes on a bank; with key / 8 for the last bit, which serves the transpose read alone, row reads took
// twice their time and 35 % of all LDS cycles were conflicts.
template <> struct Tile<bf16_t> {
  static constexpr int kKeys = 32, kGroup = 8, kPart = 128;
  __host__ __device__ static constexpr int swz(int key) { return ((key >> 1 & 3) << 1) | (key >> 2 & 1); }
  __host__ __device__ static constexpr int flip(int) { return 0; }                            // of a lane's source, from group to group
};
template <> struct Tile<float> {
  static constexpr int kKeys = 16, kGroup = 4, kPart = 256;
  __host__ __device__ static constexpr int swz(int key) { return key & 15; }
  __host__ __device__ static constexpr int flip(int group) { return group << 6; }
};

constexpr int slot_bytes(int ld, int e) { return (e == 2 ? 32 : 16) * (ld + kPe) * e; }
// LDS: the rings' slots, (max, sum) pairs of up to 64 rows for their merge, the schedule's table.  Slots of a ring: as many as find room, four at most.
constexpr int kPairsBytes = 64 * 8, kTableBytes = attn_sched_words(kAttnMaxSeqs) * 4;
constexpr int kPairsAt = kLds - kTableBytes - kPairsBytes, kTableAt = kLds - kTableBytes;
__host__ __device__ constexpr int stages_of(int ld, int e, int nk) {
  const int most = kPairsAt / (nk * slot_bytes(ld, e));
  return most < 1 ? 1 : most > 4 ? 4 : most;
}

// Where the tiles of a segment come from.  Paged: a lane holds where 16 keys lie in the pool (in units of 16 entries), for 64 of them; the next 64 are on their way.
template <typename T, int LD, bool PAGED>
struct Source {
  static constexpr int kKeys = Tile<T>::kKeys, kGroup = Tile<T>::kGroup, kPart = Tile<T>::kPart;
  static constexpr int kRowB = (LD + kPe) * static_cast<int>(sizeof(T)), kBlocks = kRowB / kPart;    // 1 KB blocks of a group
  static constexpr int kLanes = kPart / 16;                                                          // lanes of a key
  const LatentAttnArgs& a;
  int b, s0, s1;
  int lane_key, lane_chunk;    // what a lane brings in of a group: key, and byte of its part
  int ids, ids_next, chunk, id0, id1;
  __device__ __forceinline__ Source(const LatentAttnArgs& args) : a(args) {
    const int lane = threadIdx.x & 63;
    lane_key = lane / kLanes;
    lane_chunk = ((lane % kLanes) ^ Tile<T>::swz(lane_key)) << 4;
  }
  __device__ __forceinline__ int ids_at(int c) const {        // first key of the lane's sixteen
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));                  // (worked out where it is wanted, not held)
    return min(s0 + 16 * (64 * c + lane), s1 - 1) & ~15;
  }
  __device__ __forceinline__ int page_in_seq(int p) const { return static_cast<int>(static_cast<uint32_t>(p) / static_cast<uint32_t>(a.page_size)); }
  __device__ __forceinline__ int fetch(int c) const { return a.page_table[static_cast<int64_t>(b) * a.max_pages + page_in_seq(ids_at(c))]; }
  // A fetched page as sixteens of the pool, apart from the fetch: whatever is asked for between does not wait for it.
  __device__ __forceinline__ int sixteens(int page, int c) const {
    const int p = ids_at(c);
    return checked_page(page, a.n_pages, a.status) * (a.page_size >> 4) + ((p - page_in_seq(p) * a.page_size) >> 4);
  }
  __device__ __forceinline__ void begin(int seq, int from, int to) {
    b = seq; s0 = from; s1 = to;
    ids = ids_next = id0 = id1 = 0;
    chunk = -1;
    if (PAGED) ids_next = fetch(0);
  }
  // Tile ti of the segment, one that has keys, in front of its entries or blocks.  (Calls go up by less than 1024 keys.)
  __device__ __forceinline__ void locate(int ti) {
    if (!PAGED) return;
    const int blk = kKeys * ti >> 4;
    if (__builtin_expect(blk >> 6 != chunk, 0)) {
      chunk = blk >> 6;
      ids = sixteens(ids_next, chunk);
      if (s0 + 1024 * (chunk + 1) < s1) ids_next = fetch(chunk + 1);
    }
    id0 = __builtin_amdgcn_readlane(ids, blk & 63);
    if (kKeys == 32) id1 = __builtin_amdgcn_readlane(ids, (blk & 63) + 1);
  }
  __device__ __forceinline__ const char* entry(int ti, int key) const {
    if (!PAGED) return static_cast<const char*>(a.k) + (static_cast<int64_t>(b) * a.l_max + s0 + kKeys * ti + key) * kRowB;
    return static_cast<const char*>(a.k) + (static_cast<int64_t>(key < 16 ? id0 : id1) * 16 + (key & 15)) * kRowB;
  }
  // A group of a tile with keys (after locate): a base and a lane's offset.  Keys past the range repeat the group's last one, a group without any the tile's first: they are masked later.
  // (No branch: between matrix instructions one costs 30 cycles.)
  struct Group {
    const char* base;
    uint32_t off;
  };
  __device__ __forceinline__ Group group_of(int ti, int group) const {
    const int last = s1 - 1 - s0 - kKeys * ti;
    const int first = group * kGroup <= last ? group * kGroup : 0;
    return {entry(ti, first), static_cast<uint32_t>(min(lane_key, last - first) * kRowB + (lane_chunk ^ Tile<T>::flip(group)))};
  }
  __device__ __forceinline__ static void load(const Group& g, int group, int block, const char* slot) {
    load_to_lds16(g.base + block * kPart, g.off, slot + (group * kBlocks + block) * 1024);
  }
  __device__ __forceinline__ void load_group(int ti, int group, const char* slot) const {
    const Group g = group_of(ti, group);
#pragma unroll
    for (int block = 0; block < kBlocks; ++block) load(g, group, block, slot);
  }
  // Operand addresses in a tile.  rows: chunk quad ks of key fr (+ 16 half).  columns: the transpose read of chunks 2 dt, 2 dt + 1 of key 4 fq + fr / 4 (+ 16 half); fp32: value
  // 16 dt + fr of key 4 fq + e.
  __device__ static __forceinline__ int place(int key) { return (key / kGroup) * (kBlocks * 1024) + key % kGroup * kPart; }
  __device__ static __forceinline__ int rows_at(int fr, int fq) { return place(fr) + ((fq ^ Tile<T>::swz(fr)) << 4); }
  __device__ static __forceinline__ int columns_at(int fr, int fq) {
    if (sizeof(T) == 4) return place(4 * fq) + ((((fr >> 2) ^ Tile<T>::swz(4 * fq)) << 4) | ((fr & 3) << 2));
    const int key = 4 * fq + (fr >> 2);
    return place(key) + (((((fr & 3) >> 1) ^ Tile<T>::swz(key)) << 4) | ((fr & 1) << 3));
  }
  static constexpr int kHalf = (16 / kGroup) * kBlocks * 1024;                    // bytes between the halves of 16 keys
  static constexpr int kQuads = kPart / 64;                                       // chunk quads of a block
  __device__ static __forceinline__ const char* row_read(const char* tile, int rows_at, int ks, int half) {
    return tile + (rows_at ^ (ks % kQuads << 6)) + (ks / kQuads) * 1024 + half * kHalf;
  }
  __device__ static __forceinline__ const char* column_read(const char* tile, int columns_at, int dt, int e) {
    if (sizeof(T) == 4) return tile + ((columns_at ^ (e << 4) ^ ((dt & 3) << 6)) + e * kPart) + (dt >> 2) * 1024;
    return tile + (columns_at ^ ((dt & 3) << 5)) + (dt >> 2) * 1024 + e * kHalf;
  }
};

// The lane's number, worked out where it is wanted, not held.
__device__ __forceinline__ int lane_here() {
  int none = 0;
  asm volatile("" : "+v"(none));
  return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, none));
}

// Registers of a lane for accumulators and queries.  Up to 190 everything is done in 256 ordinary ones; beyond that the accumulators are in the other 256, which
// only matrix instructions work on: see the rescaling.
constexpr int held_registers(int ld, int e, int rtw) { return rtw * (ld / 4 + (ld + kPe) * e / 16); }
constexpr bool in_agprs(int ld, int e, int rtw) { return held_registers(ld, e, rtw) > 190; }

// Until at most `blocks` blocks of GROUPS loads each are outstanding (a constant where it is called: the instruction has no other form).
template <int GROUPS>
__device__ __forceinline__ void wait_blocks(int blocks) {
  switch (blocks) {
    case 8: __builtin_amdgcn_s_waitcnt(vmcnt_imm(8 * GROUPS)); break;
    case 7: __builtin_amdgcn_s_waitcnt(vmcnt_imm(7 * GROUPS)); break;
    case 6: __builtin_amdgcn_s_waitcnt(vmcnt_imm(6 * GROUPS)); break;
    case 5: __builtin_amdgcn_s_waitcnt(vmcnt_imm(5 * GROUPS)); break;
    case 4: __builtin_amdgcn_s_waitcnt(vmcnt_imm(4 * GROUPS)); break;
    case 3: __builtin_amdgcn_s_waitcnt(vmcnt_imm(3 * GROUPS)); break;
    case 2: __builtin_amdgcn_s_waitcnt(vmcnt_imm(2 * GROUPS)); break;
    case 1: __builtin_amdgcn_s_waitcnt(vmcnt_imm(GROUPS)); break;
    default: __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
  }
}

// NK = 4 / NR rings, each of NR waves with sixteen rows, and each with its own tiles of the segment.
template <typename T, int LD, int NR, bool PAGED>
__device__ __forceinline__ void ring_segments(const LatentAttnArgs& a, const AttnTable& table, const AttnLine& line, AttnSeg seg, int x_hi, char* smem) {
  constexpr int NK = 4 / NR;
  constexpr bool kF32 = sizeof(T) == 4;
  constexpr int S = stages_of(LD, sizeof(T), NK);
  constexpr int kKeys = Tile<T>::kKeys, kRowB = Source<T, LD, PAGED>::kRowB;
  constexpr int kSlot = slot_bytes(LD, sizeof(T));
  constexpr int kGroups = 4 / NR;                   // groups of a tile that a wave brings in
  constexpr int kPieces = kGroups * Source<T, LD, PAGED>::kBlocks;
  constexpr int kKS = kRowB / 64, kDT = LD / 16, kHalves = kKeys / 16;
  constexpr float kSlack = 8.f;                     // of the softmax reference, log2 units: see attn_mfma.hip
  float* ml_lds = reinterpret_cast<float*>(smem + kPairsAt);
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kg = wv / NR, rr = wv % NR;
  const int fr = lane & 15, fq = lane >> 4;
  Source<T, LD, PAGED> src(a);
  const float sl2 = a.scale * 1.44269504088896340736f;
  bool again = false;
  for (; seg.s1 > seg.s0; seg = attn_sched_next(a, table, false, line.pad, seg.next, x_hi)) {
    attn_sched_publish(a, seg);
    const int b = seg.b, row0 = seg.g * a.block_rows;
    const int R = min(a.block_rows, a.rows - row0);
    const int L = __builtin_amdgcn_readfirstlane(seg.L);
    const int s0 = seg.s0, s1 = __builtin_amdgcn_readfirstlane(seg.s1);
    const int ntl = (s1 - s0 + kKeys - 1) / kKeys;
    const int nit = (ntl + NK - 1) / NK;
    char* ring = smem + kg * (S * kSlot);

    src.begin(b, s0, s1);                           // (the page ids in front of the queries: the first tile waits for them)
    // ---- the rows' queries and mask words (rows past the last repeat it and are not stored)
    uint4 qf[kKS];
    const int row = row0 + min(16 * rr + fr, R - 1);
    const uint4* qp = reinterpret_cast<const uint4*>(static_cast<const char*>(a.q) + (static_cast<int64_t>(b) * a.rows + row) * kRowB) + fq;
#pragma unroll
    for (int ks = 0; ks < kKS; ++ks) qf[ks] = qp[4 * ks];
    // (a load either way, without a mask of a query's bytes: a branch would wait for the queries in front of the first tiles)
    const int i = row / a.Hq;
    const uint64_t* mask_at = a.mask ? a.mask + static_cast<int64_t>(b) * a.mask_stride : static_cast<const uint64_t*>(a.q);
    const uint64_t rowmask = mask_at[a.mask ? i : 0];
    if (again) __syncthreads();                     // the rings are free of the segment before
    again = true;

    auto locate = [&](int it) {
      if (it * NK + kg < ntl) src.locate(it * NK + kg);
    };
    auto issue = [&](int it) {                      // (after locate of the same tile)
      const int ti = it * NK + kg;
      if (ti >= ntl) return;
      char* slot = ring + (it % S) * kSlot;
      if constexpr (S == 1) {                       // one part of all keys after the other, as the products take them
        typename Source<T, LD, PAGED>::Group g[kGroups];
#pragma unroll
        for (int u = 0; u < kGroups; ++u) g[u] = src.group_of(ti, u);
#pragma unroll
        for (int block = 0; block < src.kBlocks; ++block)
#pragma unroll
          for (int u = 0; u < kGroups; ++u) src.load(g[u], u, block, slot);
      } else {
#pragma unroll
        for (int u = 0; u < kGroups; ++u) src.load_group(ti, rr * kGroups + u, slot);
      }
    };
    // A ring of one slot: its wave takes a part of the tile as soon as that is there.  (What was asked for in front of the tile comes first.)
    auto landed = [&](int block) {
      if constexpr (S == 1) {
        if (block >= src.kBlocks) return;
        wait_blocks<kGroups>(src.kBlocks - 1 - block);
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        __builtin_amdgcn_sched_barrier(0);
      }
    };

    f32x4_t oacc[kDT];
    float m_run = -FLT_MAX, l_run = 0.f;
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt) oacc[dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // A short segment has all its tiles in flight at once, behind the queries; of a longer one the first, so that the wait for the queries is not one for a
    // whole ring.
    const int together = S <= 2 || nit < S ? S : 1;
#pragma unroll 1
    for (int it = 0; it < together; ++it) {
      locate(it);
      issue(it);
    }
    int k_at = src.rows_at(fr, fq), v_at = src.columns_at(fr, fq);
    if constexpr (S > 1) __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));           // from here on vmcnt counts tile loads only
    if constexpr (S > 2) {
#pragma unroll 1
      for (int it = together; it < S; ++it) {
        locate(it);
        issue(it);
      }
    }

#pragma unroll 1
    for (int it = 0; it < nit; ++it) {
      if (S > 1 && it > 0) locate(it + S - 1);
      // this wave's pieces of tile `it` have landed once at most those of the S - 2 tiles behind it are outstanding (the first has already)
      if (S == 2 || (S > 2 && it + S - 1 >= nit)) __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
      else if (S > 2 && it > 0) __builtin_amdgcn_s_waitcnt(vmcnt_imm(S <= 2 ? 0 : (S - 2) * kPieces));
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_s_waitcnt(0xC07F);           // lgkmcnt(0): tile it - 1 is read
      if constexpr (NR > 1) __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      if (S > 1 && it > 0) issue(it + S - 1);
      const int ti = it * NK + kg;
      if (ti < ntl) {
        const int t0 = s0 + kKeys * ti;
        const char* tile = ring + (it % S) * kSlot;
        asm volatile("" : "+v"(k_at), "+v"(v_at));  // (worked out per read from these two, not held)
        // ---- S^T = C Q^T
        f32x4_t sacc[kHalves];
#pragma unroll
        for (int j = 0; j < kHalves; ++j) sacc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        constexpr int kReads = kHalves * kKS, kAhead = kF32 ? 4 : 8, kOfBlock = 4;          // reads; those of a 1 KB block of every group
        static_assert(kHalves * src.kQuads == kOfBlock && kAhead % kOfBlock == 0, "");
        landed(kAhead / kOfBlock - 1);
        auto kread = [&](int i) { return *reinterpret_cast<const uint4*>(src.row_read(tile, k_at, i / kHalves, i % kHalves)); };
        uint4 kf[kReads];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) kf[i] = kread(i);
#pragma unroll
        for (int i = 0; i < kReads; ++i) {
          if (i % kOfBlock == 0) landed((i + kAhead) / kOfBlock);
          if (i + kAhead < kReads) kf[i + kAhead] = kread(i + kAhead);
          __builtin_amdgcn_sched_barrier(0);
          f32x4_t& c = sacc[i % kHalves];
          if constexpr (kF32) {
            const f32x4_t x = __builtin_bit_cast(f32x4_t, kf[i]), y = __builtin_bit_cast(f32x4_t, qf[i / kHalves]);
#pragma unroll
            for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], c, 0, 0, 0);
          } else {
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf[i]), __builtin_bit_cast(bf16x8_t, qf[i / kHalves]), c, 0, 0, 0);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        // ---- online softmax; lane (row fr, fq) owns the keys t0 + 16 j + 4 fq + e
        const bool plain = t0 + kKeys <= min(L, s1);
        float x[4 * kHalves];
#pragma unroll
        for (int j = 0; j < kHalves; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) x[4 * j + e] = sacc[j][e] * sl2;
        if (!plain) {
          int given = __builtin_amdgcn_readfirstlane(a.mask != nullptr);
          asm volatile("" : "+s"(given));           // (chosen here, not in front of the loop)
          const uint64_t word = given ? rowmask : (2ull << i) - 1ull;
#pragma unroll
          for (int j = 0; j < kHalves; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int p = t0 + 16 * j + 4 * fq + e;
              bool seen = p < s1;
              if (seen && p >= L) seen = (word >> (p - L)) & 1ull;
              x[4 * j + e] = seen ? x[4 * j + e] : -INFINITY;
            }
        }
        float mt = x[0];
#pragma unroll
        for (int e = 1; e < 4 * kHalves; ++e) mt = max_nan(mt, x[e]);
        if (__builtin_amdgcn_ballot_w64(mt > m_run + kSlack) != 0ull) {
          const float m_new = fmaxf(m_run, quad_row_max(mt));
          const float al = __builtin_amdgcn_exp2f(m_run - m_new);
          m_run = m_new;
          l_run *= al;
#pragma unroll
          for (int dt = 0; dt < kDT; ++dt) {
            oacc[dt][0] *= al; oacc[dt][1] *= al;
            oacc[dt][2] *= al; oacc[dt][3] *= al;
            if constexpr (in_agprs(LD, sizeof(T), 1)) {         // four at a time there and back: all at once are as many registers again
              asm volatile("" : "+a"(oacc[dt]));
              __builtin_amdgcn_sched_barrier(0);
            }
          }
        }
        // Probabilities: fp32 as they are; bf16 two bf16 parts (16 bits), for which the matrix instructions have the time.
        float pr[4 * kHalves];
        uint4 pf, pl;
#pragma unroll
        for (int e = 0; e < 4 * kHalves; ++e) pr[e] = __builtin_amdgcn_exp2f(x[e] - m_run);
        if constexpr (kF32) {
          l_run += (pr[0] + pr[1]) + (pr[2] + pr[3]);
        } else {
          pf = make_uint4(pack_bf16x2(pr[0], pr[1]), pack_bf16x2(pr[2], pr[3]), pack_bf16x2(pr[4], pr[5]), pack_bf16x2(pr[6], pr[7]));
          float hi[8];
          unpack16(pf, hi);
          pl = make_uint4(pack_bf16x2(pr[0] - hi[0], pr[1] - hi[1]), pack_bf16x2(pr[2] - hi[2], pr[3] - hi[3]),
                          pack_bf16x2(pr[4] - hi[4], pr[5] - hi[5]), pack_bf16x2(pr[6] - hi[6], pr[7] - hi[7]));
          l_run += ((pr[0] + pr[1]) + (pr[2] + pr[3])) + ((pr[4] + pr[5]) + (pr[6] + pr[7]));
        }
        // ---- O^T += C^T P^T
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (kF32) {
          float vf[kDT][4];
          auto vread = [&](int dt) {
#pragma unroll
            for (int e = 0; e < 4; ++e) vf[dt][e] = *reinterpret_cast<const float*>(src.column_read(tile, v_at, dt, e));
          };
          constexpr int kVAhead = 2;
#pragma unroll
          for (int dt = 0; dt < kVAhead; ++dt) vread(dt);
#pragma unroll
          for (int dt = 0; dt < kDT; ++dt) {
            if (dt + kVAhead < kDT) vread(dt + kVAhead);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int e = 0; e < 4; ++e) oacc[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[dt][e], pr[e], oacc[dt], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
          }
        } else {
          s16x4_t vlo[kDT], vhi[kDT];
          auto vread = [&](int dt) {
            vlo[dt] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(lds_ptr_t)src.column_read(tile, v_at, dt, 0));
            vhi[dt] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(lds_ptr_t)src.column_read(tile, v_at, dt, 1));
          };
          constexpr int kVAhead = 4;
#pragma unroll
          for (int dt = 0; dt < kVAhead; ++dt) vread(dt);
#pragma unroll
          for (int dt = 0; dt < kDT; ++dt) {
            if (dt + kVAhead < kDT) vread(dt + kVAhead);
            __builtin_amdgcn_sched_barrier(0);
            const uint2 l2 = __builtin_bit_cast(uint2, vlo[dt]), h2 = __builtin_bit_cast(uint2, vhi[dt]);
            const bf16x8_t va = __builtin_bit_cast(bf16x8_t, make_uint4(l2.x, l2.y, h2.x, h2.y));
            oacc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, __builtin_bit_cast(bf16x8_t, pf), oacc[dt], 0, 0, 0);
            oacc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, __builtin_bit_cast(bf16x8_t, pl), oacc[dt], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
      if constexpr (S == 1) {                       // (rings of one slot, one wave: the others' loads are on their way meanwhile)
        static_assert(S > 1 || NR == 1, "a slot alone belongs to one wave");
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_s_waitcnt(0xC07F);
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        locate(it + 1);
        issue(it + 1);
      }
    }

    // ---- the segment's partial result
    const int64_t slot = static_cast<int64_t>(blockIdx.x) + static_cast<int64_t>(b) * a.Hkv + seg.g;
    const int tiles = a.block_rows / 16;            // row tiles of a block
    if constexpr (NK == 1) {
      const float l = quad_row_sum(l_run);
      if (rr < tiles) {
        if (fq == 0) *reinterpret_cast<float2*>(a.part_ml + ((slot * tiles + rr) * 16 + fr) * 2) = make_float2(m_run, l);
        float* dst = a.part_o + ((slot * tiles + rr) * kDT * 64 + lane) * 4;
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt) *reinterpret_cast<f32x4_t*>(dst + dt * 256) = oacc[dt];
      }
    } else {
      // the rings leave their sums in their own slots, and every wave adds some fragments in the order of the rings
      static_assert(NR * 16 * LD * 4 <= S * kSlot, "a ring's slots hold its sums");
      const float l = quad_row_sum(l_run);
      if constexpr (NR > 1) __syncthreads();        // (waves of a ring write where others may still read)
      if (fq == 0) *reinterpret_cast<float2*>(ml_lds + 2 * ((kg * NR + rr) * 16 + fr)) = make_float2(m_run, l);
#pragma unroll
      for (int dt = 0; dt < kDT; ++dt) *reinterpret_cast<f32x4_t*>(ring + ((rr * kDT + dt) * 64 + lane) * 16) = oacc[dt];
      __syncthreads();
#pragma unroll 1
      for (int tile = 0; tile < tiles; ++tile) {
        float f[NK], mm = -FLT_MAX, sum = 0.f;
#pragma unroll
        for (int k = 0; k < NK; ++k) {
          f[k] = ml_lds[2 * ((k * NR + tile) * 16 + fr)];
          mm = fmaxf(mm, f[k]);
        }
#pragma unroll
        for (int k = 0; k < NK; ++k) {
          f[k] = __builtin_amdgcn_exp2f(f[k] - mm);
          sum = fmaf(f[k], ml_lds[2 * ((k * NR + tile) * 16 + fr) + 1], sum);
        }
        if (wv == 0 && fq == 0) *reinterpret_cast<float2*>(a.part_ml + ((slot * tiles + tile) * 16 + fr) * 2) = make_float2(mm, sum);
        constexpr int kEach = kDT / 4;              // fragments of a wave, all read together
        f32x4_t v[kEach];
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
          for (int u = 0; u < kEach; ++u) {
            const f32x4_t o = *reinterpret_cast<const f32x4_t*>(smem + k * (S * kSlot) + ((tile * kDT + wv * kEach + u) * 64 + lane) * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[u][e] = k ? fmaf(f[k], o[e], v[u][e]) : f[k] * o[e];
          }
        float* dst = a.part_o + (((slot * tiles + tile) * kDT + wv * kEach) * 64 + lane) * 4;
#pragma unroll
        for (int u = 0; u < kEach; ++u) *reinterpret_cast<f32x4_t*>(dst + u * 256) = v[u];
      }
    }
  }
}

// bf16, 64 or 128 rows: four waves of RTW 16-row tiles on one ring of four slots, software-pipelined.  With one wave to a SIMD nothing else fills
// the time of the softmax, so the products of tile t's probabilities with its values are interleaved with the exponentials of tile t + 1, and the loads of tile t + 3
// with the products of tile t + 1 with the queries in front of that; one barrier a tile.
//
// The reference of a row's exponentials is the maximum of its first tile and stays: floating-point probabilities lose nothing by being large, so up to
// 2^kReach is fine, and the accumulators are never rescaled (256 registers that only matrix instructions work on, there and back, take longer than a tile).  A
// segment with a score beyond that is taken again with its rows' true maxima, which the first pass has found.
template <int LD, int RTW, bool PAGED>
__device__ __forceinline__ void pipe_segments(const LatentAttnArgs& a, const AttnTable& table, const AttnLine& line, AttnSeg seg, int x_hi, char* smem) {
  typedef Source<bf16_t, LD, PAGED> Src;
  constexpr int S = 4, kSlot = slot_bytes(LD, 2), kKeys = 32;
  static_assert(stages_of(LD, 2, 1) == S, "four slots");
  constexpr int kKS = Src::kRowB / 64, kReads = 2 * kKS, kDT = LD / 16, kBlocks = Src::kBlocks;
  // Probabilities: two bf16 parts (16 bits) with 64 rows, with 128 one (8 bits), normalised with its own sum, so that the rounding is no bias.  Two would be a third more of the products and sixteen registers
  // more than there are: 139 us where one takes 117 (16 sequences x 20480 entries, 128 rows), 214 for 169 (8 x 9216, 1024 rows); blocks of 64 rows with two parts take 147 and 240.  One leaves
  // results 1.15 to 1.33 times as far from 64 bits as their own rounding to bf16 does (with two: 1.00).
  constexpr bool kSplitP = RTW == 1;
  constexpr float kReach = 60.f;                    // log2; sums of 2^31 such probabilities times values of 2^30 stay in range
  // With 128 rows of 512 columns the accumulators are all 256 registers that matrix instructions alone work on, and the compiler has no form that puts
  // other results elsewhere: the scores' instructions are written out.
  constexpr bool kWritten = LD == 512 && RTW == 2;
  int* votes = reinterpret_cast<int*>(smem + kPairsAt);
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 15, fq = lane >> 4;
  Src src(a);
  const float sl2 = a.scale * 1.44269504088896340736f;
  bool again = false;
  for (; seg.s1 > seg.s0; seg = attn_sched_next(a, table, false, line.pad, seg.next, x_hi)) {
    attn_sched_publish(a, seg);
    const int b = seg.b, row0 = seg.g * a.block_rows;
    const int R = min(a.block_rows, a.rows - row0);
    const int L = __builtin_amdgcn_readfirstlane(seg.L);
    const int s0 = seg.s0, s1 = __builtin_amdgcn_readfirstlane(seg.s1);
    const int ntl = (s1 - s0 + kKeys - 1) / kKeys;
    src.begin(b, s0, s1);                           // (the page ids in front of the queries: the first tile waits for them)
    uint4 qf[kKS][RTW];
    const char* q0 = static_cast<const char*>(a.q) + (static_cast<int64_t>(b) * a.rows + row0) * Src::kRowB;
#pragma unroll
    for (int t = 0; t < RTW; ++t) {
      const uint32_t off = static_cast<uint32_t>(min(16 * (wv * RTW + t) + fr, R - 1) * Src::kRowB + fq * 16);      // (rows past the last repeat it and are not stored)
#pragma unroll
      for (int ks = 0; ks < kKS; ++ks) qf[ks][t] = *reinterpret_cast<const uint4*>(q0 + off + 64 * ks);
    }
    float known[RTW];                               // second pass: the rows' maxima
#pragma unroll 1
    for (int pass = 0;; ++pass) {
    if (again) __syncthreads();                     // the ring is free of the segment before
    again = true;
    if (pass) src.begin(b, s0, s1);
    auto slot_of = [&](int ti) { return smem + (ti & (S - 1)) * kSlot; };
    // Every step asks for a tile, behind the last one for that again: the count of what is outstanding is then always the same.
    auto issue = [&](int ti) {
      const int t = min(ti, ntl - 1);
      src.locate(t);
      src.load_group(t, wv, slot_of(ti));
    };
    issue(0);
    int k_at = Src::rows_at(fr, fq), v_at = Src::columns_at(fr, fq);
    f32x4_t oacc[kDT][RTW];
    float ref[RTW], l_run[RTW], most[RTW];          // reference, sum of the probabilities, largest score (times sl2: the first two)
#pragma unroll
    for (int t = 0; t < RTW; ++t) {
      l_run[t] = 0.f;
      most[t] = -INFINITY;
#pragma unroll
      for (int dt = 0; dt < kDT; ++dt) oacc[dt][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));       // (the queries and the first tile) from here on vmcnt counts tile loads only
    issue(1);
    issue(2);

    f32x4_t sn[2][RTW];                             // scores of the next tile: key half, row tile
    auto score = [&](f32x4_t& c, const uint4& k, const uint4& q, bool first) {
      const bf16x8_t x = __builtin_bit_cast(bf16x8_t, k), y = __builtin_bit_cast(bf16x8_t, q);
      if constexpr (kWritten) {
        if (first) asm("v_mfma_f32_16x16x32_bf16 %0, %1, %2, 0" : "=&v"(c) : "v"(x), "v"(y));
        else asm("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(c) : "v"(x), "v"(y));
      } else {
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, first ? f32x4_t{0.f, 0.f, 0.f, 0.f} : c, 0, 0, 0);
      }
    };
    // the scores are there (the compiler does not know how long the written instructions take: eight passes, 11 wait states to an ordinary read)
    auto scored = [&] {
      if constexpr (kWritten) asm volatile("s_nop 15" : "+v"(sn[0][0]), "+v"(sn[1][0]), "+v"(sn[0][RTW - 1]), "+v"(sn[1][RTW - 1]));
    };
    auto mask_tile = [&](int ti) {                  // keys past the range and block entries that a row does not see
      const int t0 = s0 + kKeys * ti;
      if (__builtin_expect(t0 + kKeys <= min(L, s1), 1)) return;
#pragma unroll
      for (int t = 0; t < RTW; ++t) {
        const int ln = lane_here();                 // (once or twice a segment; of each row tile anew, for what is worked out from it is not held then)
        __builtin_amdgcn_sched_barrier(0);
        const int i = (row0 + min(16 * (wv * RTW + t) + (ln & 15), R - 1)) / a.Hq;
        const uint64_t word = a.mask ? a.mask[static_cast<int64_t>(b) * a.mask_stride + i] : ((2ull << i) - 1ull);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int p = t0 + 16 * j + 4 * (ln >> 4) + e;
            bool seen = p < s1;
            if (seen && p >= L) seen = (word >> (p - L)) & 1ull;
            sn[j][t][e] = seen ? sn[j][t][e] : -INFINITY;
          }
      }
    };
    constexpr int kAhead = 8, kVAhead = 4;
    uint4 kf[kReads];
    auto kread = [&](const char* tile, int i) { kf[i] = *reinterpret_cast<const uint4*>(Src::row_read(tile, k_at, i / 2, i % 2)); };

    uint32_t pw[RTW][4], pn[RTW][4], rw[RTW][4], rn[RTW][4];          // probabilities of a tile and of the next, two to a word; what they are rounded by
    float pr[2];
    auto weigh = [&](int n, uint32_t (&p)[RTW][4], uint32_t (&rest)[RTW][4]) {      // exponential n: row tile n / 8, key half n / 4 % 2
      const int t = n / 8, e = n % 8;
      const float x = sn[e >> 2][t][e & 3];
      most[t] = max_nan(most[t], x);
      pr[e & 1] = __builtin_amdgcn_exp2f(fmaf(x, sl2, -ref[t]));
      if (!(e & 1)) return;
      const uint32_t word = pack_bf16x2(pr[0], pr[1]);
      const float lo = __uint_as_float(word << 16), hi = __uint_as_float(word & 0xFFFF0000u);
      p[t][e >> 1] = word;
      if constexpr (kSplitP) {
        rest[t][e >> 1] = pack_bf16x2(pr[0] - lo, pr[1] - hi);
        l_run[t] += pr[0] + pr[1];
      } else {
        l_run[t] += lo + hi;                        // the probabilities as the values are multiplied with them
      }
    };
    // ---- the first tile's scores
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_s_waitcnt(0xC07F);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int i = 0; i < kAhead; ++i) kread(smem, i);
#pragma unroll
    for (int i = 0; i < kReads; ++i) {
      if (i + kAhead < kReads) kread(smem, i + kAhead);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < RTW; ++t) score(sn[i % 2][t], kf[i], qf[i / 2][t], i < 2);
      __builtin_amdgcn_sched_barrier(0);
    }
    scored();
    mask_tile(0);
#pragma unroll
    for (int t = 0; t < RTW; ++t) {
      float mt = sn[0][t][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) mt = max_nan(mt, sn[e >> 2][t][e & 3]);
      ref[t] = pass ? known[t] : fmaxf(-FLT_MAX, quad_row_max(mt * sl2));
    }
#pragma unroll
    for (int n = 0; n < 8 * RTW; ++n) weigh(n, pw, rw);

#pragma unroll 1
    for (int ti = 0;; ++ti) {
      const int tl = min(ti + S - 1, ntl - 1);
      src.locate(tl);
      const typename Src::Group group = src.group_of(tl, wv);
      char* to = slot_of(ti + S - 1);
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(kBlocks));         // tile ti + 1 has landed: at most this wave's blocks of tile ti + 2 are outstanding
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_s_waitcnt(0xC07F);           // lgkmcnt(0): tile ti - 1 is read
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      const char* tile = slot_of(ti);
      const char* next = slot_of(ti + 1);
      asm volatile("" : "+v"(k_at), "+v"(v_at));    // (worked out per read from these two, not held)
      s16x4_t vlo[kDT], vhi[kDT];
      auto vread = [&](int dt) {
        vlo[dt] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(lds_ptr_t)Src::column_read(tile, v_at, dt, 0));
        vhi[dt] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(lds_ptr_t)Src::column_read(tile, v_at, dt, 1));
      };
      // ---- scores of tile ti + 1, loads of tile ti + 3.  (Behind the last tile: of what lies in the slot, all of it masked; a copy of the code without would be one
      // of the products below as well, and the accumulators of two do not stay in place.)
#pragma unroll
      for (int i = 0; i < kAhead; ++i) kread(next, i);
#pragma unroll
      for (int i = 0; i < kReads; ++i) {
        if (i + kAhead < kReads) kread(next, i + kAhead);
        if (i >= kReads - kVAhead) vread(i - (kReads - kVAhead));
        if (i % 4 == 0) Src::load(group, wv, i / 4, to);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < RTW; ++t) score(sn[i % 2][t], kf[i], qf[i / 2][t], i < 2);
        __builtin_amdgcn_sched_barrier(0);
      }
      scored();
      mask_tile(ti + 1);
      // ---- O^T += C^T P^T of tile ti, exponentials of tile ti + 1
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int dt = 0; dt < kDT; ++dt) {
        if (dt + kVAhead < kDT) vread(dt + kVAhead);
        __builtin_amdgcn_sched_barrier(0);
        const uint2 l2 = __builtin_bit_cast(uint2, vlo[dt]), h2 = __builtin_bit_cast(uint2, vhi[dt]);
        const bf16x8_t va = __builtin_bit_cast(bf16x8_t, make_uint4(l2.x, l2.y, h2.x, h2.y));
#pragma unroll
        for (int t = 0; t < RTW; ++t) {
          const bf16x8_t p = __builtin_bit_cast(bf16x8_t, make_uint4(pw[t][0], pw[t][1], pw[t][2], pw[t][3]));
          oacc[dt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, p, oacc[dt][t], 0, 0, 0);
          if constexpr (kSplitP) {
            const bf16x8_t r = __builtin_bit_cast(bf16x8_t, make_uint4(rw[t][0], rw[t][1], rw[t][2], rw[t][3]));
            oacc[dt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, r, oacc[dt][t], 0, 0, 0);
          }
        }
        constexpr int kEach = (8 * RTW + kDT - 1) / kDT;
#pragma unroll
        for (int n = dt * kEach; n < (dt + 1) * kEach; ++n)
          if (n < 8 * RTW) weigh(n, pn, rn);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int t = 0; t < RTW; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          pw[t][e] = pn[t][e];
          if constexpr (kSplitP) rw[t][e] = rn[t][e];
        }
      if (ti + 1 >= ntl) break;
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));       // (nothing is on its way to the ring any more)
    // (a maximum that is not a number counts as one out of reach: its row is worked out again by the merging kernel)
    bool far = false;
#pragma unroll
    for (int t = 0; t < RTW; ++t) {
      const float top = most[t] * sl2;
      known[t] = top != top ? top : fmaxf(-FLT_MAX, quad_row_max(top));
      far = far || !(known[t] - ref[t] <= kReach);
    }
    if (pass == 0) {                                // (static LDS, which the workgroup vote takes, has no room beside the slots)
      const bool mine = __builtin_amdgcn_ballot_w64(far) != 0ull;
      if (lane_here() == 0) votes[wv] = mine;
      __syncthreads();
      if (votes[0] | votes[1] | votes[2] | votes[3]) continue;
    }

    // ---- the segment's partial result
    const int64_t slot = static_cast<int64_t>(blockIdx.x) + static_cast<int64_t>(b) * a.Hkv + seg.g;
    const int tiles = a.block_rows / 16;
#pragma unroll
    for (int t = 0; t < RTW; ++t) {
      const float l = quad_row_sum(l_run[t]);
      const int rt = wv * RTW + t;
      if (rt >= tiles) continue;
      const int ln = lane_here();
      if (ln < 16) *reinterpret_cast<float2*>(a.part_ml + ((slot * tiles + rt) * 16 + ln) * 2) = make_float2(ref[t], l);
      float* dst = a.part_o + (slot * tiles + rt) * (kDT * 256);
#pragma unroll
      for (int dt = 0; dt < kDT; ++dt) *reinterpret_cast<f32x4_t*>(dst + dt * 256 + ln * 4) = oacc[dt][t];
    }
    break;
    }
  }
}

// Rows of a workgroup.  Few granules (64 entries for the whole rows of a sequence; the lengths are known here only): what counts is how many workgroups share them and what each
// writes for the merge, 2 KB a row with 512 columns, so they take 16 rows, each with four rings of keys, or 32 with two; the caches are small then and their
// second reader finds them in a cache of the chip.  Many: 64 or 128 (MOST), as many as the sequences have.  Whole calls, LD = 512, granules of MOST rows, 16 / 32 / MOST rows a workgroup:
//   112 rows   3: 12.9 / 13.4 / 18.9 us   17: 15.4 / 16.1 / 20.2   65: 18.1 / 20.2 / 24.2   126: 20.9 / 21.5 / 28.1   160: 28.4 / 25.2 / 30.6   257: 35.0 / 28.2 / 31.3   501: 38.0 / 40.6 / 41.7
//   1025: 61 / 63 / 46         128 rows 256 (8 sequences): 34.9 / 35.3 / 39.3   504: 46.1 / 40.3 / 39.3   4112 (16): 314 / 165 / 97         64 rows 252: 26.2 / 23.3 / 24.8   2016: 84 / 57 / 51
constexpr int kFewGran = 160, kSomeGran = 512;
__host__ __device__ __forceinline__ int rows_of_block(int rows, int most) {
  const int blocks = (rows + most - 1) / most;
  return ((rows + blocks - 1) / blocks + 15) & ~15;
}

template <typename T, int LD, int MOST, bool PAGED>
__global__ __launch_bounds__(256, MOST <= 32 && !in_agprs(LD, sizeof(T), 1) ? 2 : 1) void k_latent_attn(const LatentAttnArgs args) {
  extern __shared__ uint4 smem4[];
  char* smem = reinterpret_cast<char*>(smem4);
  LatentAttnArgs a = args;
  const AttnTable table = attn_sched_build(a, reinterpret_cast<int*>(smem + kTableAt));
  int most = MOST;
  if (MOST > 16) {
    const int gran = (a.B <= 64 ? __builtin_amdgcn_readlane(table.upto, 63) : __builtin_amdgcn_readfirstlane(table.S[a.B])) * ((a.rows + MOST - 1) / MOST);
    most = gran < kFewGran ? 16 : MOST > 32 && gran < kSomeGran ? 32 : MOST;
  }
  a.block_rows = rows_of_block(a.rows, most);
  a.Hkv = (a.rows + a.block_rows - 1) / a.block_rows;
  if (blockIdx.x == 0 && threadIdx.x == 0) a.sched[0] = a.block_rows;         // for the merging kernel
  a.sched += 2;
  const AttnLine line = attn_sched_line(a, table);
  if (static_cast<int>(blockIdx.x) >= line.W) return;         // the whole workgroup leaves together
  const int x_hi = attn_sched_lo(line, blockIdx.x + 1);
  const AttnSeg seg = attn_sched_next(a, table, true, line.pad, attn_sched_lo(line, blockIdx.x), x_hi);
  if (seg.next < x_hi) attn_sched_keep(a, table);
  if constexpr (MOST > 32) {
    if (most == MOST) {
      if constexpr (sizeof(T) == 4) ring_segments<T, LD, 4, PAGED>(a, table, line, seg, x_hi, smem);
      else pipe_segments<LD, MOST / 64, PAGED>(a, table, line, seg, x_hi, smem);
      return;
    }
  }
  if constexpr (MOST > 16) {
    if (most == 32) {
      ring_segments<T, LD, 2, PAGED>(a, table, line, seg, x_hi, smem);
      return;
    }
  }
  ring_segments<T, LD, 1, PAGED>(a, table, line, seg, x_hi, smem);
}

__device__ __forceinline__ float load_value(const bf16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ float load_value(const float* p) { return *p; }

// Sixteen columns of one output row key by key, from the entries that it sees: for rows that are not finite, since the products above multiply what is masked with zero.
template <typename T, int LD>
__device__ __forceinline__ void latent_row_again(const LatentAttnArgs& a, int b, int row, int dt, float (&lds)[4][18]) {
  constexpr int E = LD / 64;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int L = attn_ctx_len(a, b), i = row / a.Hq;
  const uint64_t word = a.mask ? a.mask[static_cast<int64_t>(b) * a.mask_stride + i] : ((2ull << i) - 1ull);
  const T* q = static_cast<const T*>(a.q) + (static_cast<int64_t>(b) * a.rows + row) * (LD + kPe);
  float qv[E + 1], acc = 0.f, m = -INFINITY, sum = 0.f;
#pragma unroll
  for (int e = 0; e <= E; ++e) qv[e] = load_value(q + 64 * e + lane);
  for (int p = wv; p < L + a.n_blk; p += 4) {
    if (p >= L && !((word >> (p - L)) & 1ull)) continue;
    int64_t at = static_cast<int64_t>(b) * a.l_max + p;
    if (a.paged) {
      const int in_seq = p / a.page_size;
      at = static_cast<int64_t>(checked_page(a.page_table[static_cast<int64_t>(b) * a.max_pages + in_seq], a.n_pages, a.status)) * a.page_size + (p - in_seq * a.page_size);
    }
    const T* c = static_cast<const T*>(a.k) + at * (LD + kPe);
    float s = 0.f;
#pragma unroll
    for (int e = 0; e <= E; ++e) s = fmaf(qv[e], load_value(c + 64 * e + lane), s);
    s = wave_sum_dpp(s) * a.scale * 1.44269504088896340736f;
    const float m_new = max_nan(m, s);
    const float old = m == m_new ? 1.f : exp2f(m - m_new), w = s == -INFINITY ? 0.f : exp2f(s - m_new);
    m = m_new;
    sum = sum * old + w;
    acc = acc * old + w * load_value(c + 16 * dt + (lane & 15));
  }
  __syncthreads();
  if (lane < 16) lds[wv][lane] = acc;
  if (lane == 0) {
    lds[wv][16] = m;
    lds[wv][17] = sum;
  }
  __syncthreads();
  float mm = -INFINITY;
  for (int k = 0; k < 4; ++k) mm = max_nan(mm, lds[k][16]);
  float den = 0.f, v = 0.f;
  for (int k = 0; k < 4; ++k) {
    const float w = lds[k][16] == -INFINITY ? 0.f : exp2f(lds[k][16] - mm);          // (a wave that saw nothing, or scores of minus infinity only)
    if (w == 0.f) continue;
    den += w * lds[k][17];
    v += w * lds[k][lane & 15];
  }
  v = mm == -INFINITY ? 0.f : v / den;
  if (threadIdx.x < 16) {
    T* out = static_cast<T*>(a.out) + (static_cast<int64_t>(b) * a.rows + row) * LD + 16 * dt + lane;
    if constexpr (sizeof(T) == 2) *out = static_cast<bf16_t>(pack_bf16x2(v, v));
    else *out = v;
  }
}

// Merge the segments of sixteen rows: exact log-sum-exp combination.  Partial results lie as the matrix instructions leave them, a 1 KB fragment for sixteen rows and
// sixteen columns, and are read and added that way: (max, sum) pairs and fragments of a wave's segments in one round of requests, the WS waves that share a fragment's
// segments in a fixed order.  (What is not there is not asked for: with the last segment again in its place the merge of 272 segments of 128 rows x 512 columns, 71 MB, took 17.3
// us, 15.4 this way; with four waves a fragment there 24.6.)
// A segment's sum counts whatever its weight: it is finite or, of a key that the row sees (what is masked weighs nothing), NaN, and maxima pass NaN over, so that a segment
// whose scores are all NaN is left with the lowest maximum.
template <typename T, int LD, int WS>
__global__ __launch_bounds__(256) void k_latent_combine(const LatentAttnArgs a) {
  constexpr int kDT = LD / 16, kPer = 4 / WS, kCombAhead = WS == 1 ? 8 : 12;
  __shared__ f32x4_t part[4][64];
  __shared__ float2 part_ml[4][16];
  __shared__ float again[4][18];
  __shared__ int odd_rows;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 15, fq = lane >> 4;
  const int block_rows = a.sched[0], tiles = block_rows / 16, blocks = (a.rows + block_rows - 1) / block_rows;
  const int b = blockIdx.y, g = blockIdx.x / tiles, tile = blockIdx.x - g * tiles, u = b * blocks + g;
  const int row = blockIdx.x * 16 + fr;
  const int w_first = a.sched[2 + 2 * u], n = __builtin_amdgcn_readfirstlane(a.sched[3 + 2 * u] - w_first + 1);
  const int64_t first = (static_cast<int64_t>(w_first) + u) * tiles + tile;
  const float* pm = a.part_ml + first * 32 + fr * 2;
  const float* po = a.part_o + first * (kDT * 256) + lane * 4;
  const int64_t po_step = static_cast<int64_t>(tiles) * (kDT * 256), pm_step = static_cast<int64_t>(tiles) * 32;
#pragma unroll 1
  for (int d0 = blockIdx.z * kPer; d0 < kDT; d0 += gridDim.z * kPer) {
    const int dt = d0 + wv / WS;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    float m = -FLT_MAX, den = 0.f;
#pragma unroll 1
    for (int s0 = wv % WS; s0 < n; s0 += WS * kCombAhead) {
      f32x4_t o[kCombAhead];
      float2 ml[kCombAhead];
#pragma unroll
      for (int e = 0; e < kCombAhead; ++e) {
        o[e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        ml[e] = make_float2(-FLT_MAX, 0.f);
      }
#pragma unroll
      for (int e = 0; e < kCombAhead; ++e) {
        const int s = s0 + e * WS;
        if (s >= n) break;                          // (uniform)
        o[e] = *reinterpret_cast<const f32x4_t*>(po + s * po_step + dt * 256);
        ml[e] = *reinterpret_cast<const float2*>(pm + s * pm_step);
      }
      __builtin_amdgcn_sched_barrier(0);
      float m_new = m;
#pragma unroll
      for (int e = 0; e < kCombAhead; ++e) m_new = fmaxf(m_new, ml[e].x);
      const float old = __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      den *= old;
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c] *= old;
#pragma unroll
      for (int e = 0; e < kCombAhead; ++e) {
        if (s0 + e * WS >= n) break;
        const float w = __builtin_amdgcn_exp2f(ml[e].x - m);
        den = fmaf(w, ml[e].y, den);
        if (w != 0.f) {                             // (a weight of nothing counts nothing, whatever is there)
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[c] = fmaf(w, o[e][c], acc[c]);
        }
      }
    }
    if constexpr (WS > 1) {
      part[wv][lane] = acc;
      if (fq == 0) part_ml[wv][fr] = make_float2(m, den);
      __syncthreads();
      if (wv % WS == 0) {
        float2 ml[WS];
        float top = m;
#pragma unroll
        for (int k = 0; k < WS; ++k) {
          ml[k] = part_ml[wv + k][fr];
          top = fmaxf(top, ml[k].x);
        }
        den = 0.f;
        acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < WS; ++k) {
          const float w = __builtin_amdgcn_exp2f(ml[k].x - top);
          den = fmaf(w, ml[k].y, den);
          if (w == 0.f) continue;
          const f32x4_t v = part[wv + k][lane];
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[c] = fmaf(w, v[c], acc[c]);
        }
      }
    }
    bool odd = false;
    if (wv % WS == 0 && row < a.rows) {
      const float inv = den == 0.f ? 0.f : 1.f / den;          // (a row that sees nothing)
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c] *= inv;
      T* dst = static_cast<T*>(a.out) + (static_cast<int64_t>(b) * a.rows + row) * LD + 16 * dt + 4 * fq;
      if constexpr (sizeof(T) == 2) {
        const uint2 v = make_uint2(pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3]));
        __builtin_memcpy(dst, &v, sizeof(v));
      } else {
        __builtin_memcpy(dst, &acc, sizeof(acc));
      }
      odd = !(fabsf((acc[0] + acc[1]) + (acc[2] + acc[3])) < INFINITY) || !(fabsf(den) < INFINITY);
    }
    if (__syncthreads_or(odd)) {                       // rows that are not finite, one after the other, for every fragment of this step
#pragma unroll 1
      for (int f = 0; f < kPer; ++f) {
        if (threadIdx.x == 0) odd_rows = 0;
        __syncthreads();
        if (odd && wv / WS == f) atomicOr(&odd_rows, 1 << fr);
        __syncthreads();
        int left = odd_rows;
        while (left) {
          const int r = __ffs(left) - 1;
          left &= left - 1;
          latent_row_again<T, LD>(a, b, blockIdx.x * 16 + r, d0 + f, again);
        }
        __syncthreads();
      }
    }
  }
}

// Rows that a workgroup takes where there is work for all of them.
int most_rows(const LatentAttnArgs& a) { return a.rows <= 16 ? 16 : a.rows <= 32 ? 32 : a.rows <= 64 || a.dtype == 0 ? 64 : 128; }

template <typename T, int LD, int MOST, bool PAGED>
hipError_t launch_attn_as(const LatentAttnArgs& a, hipStream_t s) {
  // set once per process; a function-local static is initialised under the language's own lock, so first calls from several host threads are safe
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_latent_attn<T, LD, MOST, PAGED>), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL((k_latent_attn<T, LD, MOST, PAGED>), dim3(a.wgrid), dim3(256), kLds, s, a);
  return hipGetLastError();
}
template <typename T, int LD, int MOST>
hipError_t launch_most(const LatentAttnArgs& a, hipStream_t s) {
  return a.paged ? launch_attn_as<T, LD, MOST, true>(a, s) : launch_attn_as<T, LD, MOST, false>(a, s);
}

template <typename T, int LD>
hipError_t launch_ld(const LatentAttnArgs& a, hipStream_t s) {
  hipError_t e;
  const int most = most_rows(a);
  if (most == 16) e = launch_most<T, LD, 16>(a, s);
  else if (most == 32) e = launch_most<T, LD, 32>(a, s);
  else if (most == 64) e = launch_most<T, LD, 64>(a, s);
  else if constexpr (sizeof(T) == 2) e = launch_most<T, LD, 128>(a, s);
  else e = hipErrorInvalidValue;
  if (e != hipSuccess) return e;
  // a fragment's segments to four waves where there are few fragments; many: several fragments a workgroup, some 4096 of those
  const unsigned tiles = static_cast<unsigned>((a.rows + 15) / 16);
  const int64_t fragments = static_cast<int64_t>(tiles) * a.B;
  constexpr int kDT = LD / 16;
  if (fragments * kDT < 4096) {
    hipLaunchKernelGGL((k_latent_combine<T, LD, 4>), dim3(tiles, a.B, kDT), dim3(256), 0, s, a);
  } else {
    const unsigned z = static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>(kDT / 4, 4096 / fragments)));
    hipLaunchKernelGGL((k_latent_combine<T, LD, 1>), dim3(tiles, a.B, z), dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t launch_as(const LatentAttnArgs& a, hipStream_t s) {
  switch (a.d) {
    case 128: return launch_ld<T, 128>(a, s);
    case 256: return launch_ld<T, 256>(a, s);
    case 512: return launch_ld<T, 512>(a, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

bool latent_attn_plan(LatentAttnArgs& a, int num_cus) {
  a.rows = a.Hq * a.n_q;
  a.block_rows = rows_of_block(a.rows, most_rows(a));
  a.Hkv = (a.rows + a.block_rows - 1) / a.block_rows;
  a.pad = 2;
  a.wide_from = INT_MAX;
  a.use_mfma = 0;
  if (a.B > kAttnMaxSeqs || a.l_max < a.n_blk) return false;
  // (smaller blocks are taken of few granules only, some 8 kSomeGran of theirs at most)
  const int64_t gmax = (a.l_max + kAttnGran - 1) / kAttnGran;
  if (static_cast<int64_t>(a.B) * a.Hkv * (gmax + a.pad) >= (1ll << 30)) return false;
  // one workgroup per compute unit; fewer where even the longest possible caches have no granule for each
  const int64_t most = static_cast<int64_t>(a.B) * ((a.rows + 15) / 16) * gmax;
  a.wgrid = static_cast<int>(std::min<int64_t>(most, num_cus));
  return true;
}

// Partial results: a slot per workgroup and one per unit, of the rows of a block, whichever block is taken.
static size_t up256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }
static size_t slot_rows(const LatentAttnArgs& a) {
  size_t rows = 0;
  for (const int most : {16, 32, 64, 128}) {
    if (most > most_rows(a)) break;
    const size_t block = rows_of_block(a.rows, most), blocks = (a.rows + block - 1) / block;
    rows = std::max(rows, (static_cast<size_t>(a.wgrid) + static_cast<size_t>(a.B) * blocks) * block);
  }
  return rows;
}
static size_t sched_bytes(const LatentAttnArgs& a) { return up256((2 + static_cast<size_t>(a.B) * ((a.rows + 15) / 16) * 2) * sizeof(int)); }

size_t latent_attn_workspace_bytes(const LatentAttnArgs& a) {
  return up256(slot_rows(a) * a.d * sizeof(float)) + up256(slot_rows(a) * 2 * sizeof(float)) + sched_bytes(a);
}

void latent_attn_carve(LatentAttnArgs& a, void* workspace) {
  char* p = static_cast<char*>(workspace);
  a.part_o = reinterpret_cast<float*>(p);
  p += up256(slot_rows(a) * a.d * sizeof(float));
  a.part_ml = reinterpret_cast<float*>(p);
  p += up256(slot_rows(a) * 2 * sizeof(float));
  a.sched = reinterpret_cast<int*>(p);
}

hipError_t launch_latent_attn(const LatentAttnArgs& a, hipStream_t s) { return a.dtype == 1 ? launch_as<bf16_t>(a, s) : launch_as<float>(a, s); }

}  // namespace sx
