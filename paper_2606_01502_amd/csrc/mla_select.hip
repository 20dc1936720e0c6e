// What chooses the blocks a query row attends: the mean keys of whole blocks, the
// scores of a request's blocks by them, and the choice of the best.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "mla_mx4.h"
#include "mla_select.h"

namespace mla {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ uint16_t bf16_bits(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ float low_half(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_half(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// ---- mean keys.
//
// The mean of a block is the sum of its 64 entries over 64, in fp32, rounded once to
// bf16, in which the scores' matrix products take it.  fp8: the sum of 64 codes is
// exact in fp32 (multiples of 2^-9 below 2^15), the block's scale comes after it.
//
// Several workgroups look at the same 1024 slots and share out the blocks that end
// there in their order, so that each has its part both of a prompt's tokens, every
// 64th of which ends a block, and of a list of ends.  A block's 18 loads a thread are
// all out before the first sum: a stream through HBM, bound by the launch and two
// trips where few blocks are whole.  100,003 tokens that complete 1562 fp8 blocks (58
// MB) take 16.1 us, 3.7 TB/s (20.9 with every n-th slot to a workgroup, which gave some
// of them three blocks and others none); 128 tokens that complete two 3.6.
constexpr int kMeanCols = kDLat + kDPe;

// Adds the eight bf16 of v to a.
__device__ __forceinline__ void add8(float (&a)[8], u32x4_t v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a[2 * i] += low_half(v[i]);
    a[2 * i + 1] += high_half(v[i]);
  }
}

// Adds the sixteen e4m3 codes of v to a.
__device__ __forceinline__ void add16(float (&a)[16], u32x4_t v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[i], false);
    const f32x2_t hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[i], true);
    a[4 * i] += lo[0];
    a[4 * i + 1] += lo[1];
    a[4 * i + 2] += hi[0];
    a[4 * i + 3] += hi[1];
  }
}

template <int N>
__device__ __forceinline__ void over_lanes(float (&a)[N], int from) {
  for (int o = from; o < 64; o <<= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] += __shfl_xor(a[i], o);
}

// The sums of block b's columns, each wave's in sums[wave].
template <int KV>
__device__ __forceinline__ void block_sums(const MeansParams& p, int64_t b, float (*sums)[kMeanCols]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if constexpr (KV == kKvFp8Shared) {  // (either kind of scales)
    const u32x4_t* const lat = (const u32x4_t*)(p.ckv + b * (kBlock * kDLat));
    const u32x4_t* const rope = (const u32x4_t*)(p.kpe + b * (kBlock * kDPe));
    u32x4_t v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = lat[(wave * 8 + j) * 64 + lane];
    const u32x4_t w = rope[wave * 64 + lane];
    float a[16] = {}, r[16] = {};
#pragma unroll
    for (int j = 0; j < 8; ++j) add16(a, v[j]);
    add16(r, w);
    over_lanes(a, 32);
    over_lanes(r, 4);
    if (lane < 32)
#pragma unroll
      for (int i = 0; i < 16; ++i) sums[wave][16 * lane + i] = a[i];
    if (lane < 4)
#pragma unroll
      for (int i = 0; i < 16; ++i) sums[wave][kDLat + 16 * lane + i] = r[i];
  } else {
    float a[8] = {}, r[8] = {};
    u32x4_t w[2];
    const u32x4_t* const rope = (const u32x4_t*)(p.kpe + b * (kBlock * kDPe * 2));
    if constexpr (KV == kKvMx4) {
      const uint8_t* const rows = p.ckv + (b * kBlock + wave * 16) * kMx4Row;
      uint32_t c[16], e[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        c[j] = *(const uint32_t*)(rows + j * kMx4Row + 4 * lane);
        e[j] = rows[j * kMx4Row + kDLat / 2 + (lane >> 2)];
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) w[j] = rope[(wave * 2 + j) * 64 + lane];
#pragma unroll
      for (int j = 0; j < 16; ++j) add8(a, mx4x8_bf16(c[j], mx4_scale(e[j])));
    } else {
      const u32x4_t* const lat = (const u32x4_t*)(p.ckv + b * (kBlock * kDLat * 2));
      u32x4_t v[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = lat[(wave * 16 + j) * 64 + lane];
#pragma unroll
      for (int j = 0; j < 2; ++j) w[j] = rope[(wave * 2 + j) * 64 + lane];
#pragma unroll
      for (int j = 0; j < 16; ++j) add8(a, v[j]);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) add8(r, w[j]);
    over_lanes(r, 8);
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[wave][8 * lane + i] = a[i];
    if (lane < 8)
#pragma unroll
      for (int i = 0; i < 8; ++i) sums[wave][kDLat + 8 * lane + i] = r[i];
  }
}

template <int KV>
__global__ __launch_bounds__(kThreads) void means_kernel(const MeansParams p) {
  __shared__ float sums[4][kMeanCols];
  __shared__ int32_t whole[kMeanWindow];
  __shared__ int counts[kMeanWindow / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int window = div_by((int)blockIdx.x, p.by_sharers), own = (int)blockIdx.x - window * p.sharers;
  const int64_t t0 = (int64_t)window * kMeanWindow;
  constexpr int kPer = kMeanWindow / kThreads;
  int32_t block[kPer];
  uint64_t ends[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int64_t t = t0 + k * kThreads + tid;
    const int32_t s = t < p.T ? p.slots[t] : -1;
    const bool end = s >= 0 && s < p.n_slots && s % kBlock == kBlock - 1;
    block[k] = end ? s / kBlock : -1;
    ends[k] = __ballot(end);
    if (lane == 0) counts[4 * k + wave] = (int)__popcll(ends[k]);
  }
  __syncthreads();
  int n = 0, at[kPer] = {};  // of the window, and before the wave's
#pragma unroll
  for (int k = 0; k < kMeanWindow / 64; ++k) {
    if ((k & 3) == wave) at[k >> 2] = n;
    n += counts[k];
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k)
    if (block[k] >= 0) whole[at[k] + (int)__popcll(ends[k] & ((1ull << lane) - 1))] = block[k];
  __syncthreads();
  for (int k = own; k < n; k += p.sharers) {
    const int64_t b = __builtin_amdgcn_readfirstlane(whole[k]);
    block_sums<KV>(p, b, sums);
    __syncthreads();
    float lat = 1.f / kBlock, pe = 1.f / kBlock;
    if constexpr (KV == kKvFp8Shared) {
      lat *= p.ckv_scale[b];
      pe *= p.kpe_scale[b];
    }
    uint32_t* const out = (uint32_t*)(p.means + b * kMeanCols);
    for (int c = tid; c < kMeanCols / 2; c += kThreads) {
      float v[2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        v[i] = ((sums[0][2 * c + i] + sums[1][2 * c + i]) + (sums[2][2 * c + i] + sums[3][2 * c + i])) *
               (c < kDLat / 2 ? lat : pe);
      out[c] = (uint32_t)bf16_bits(v[0]) | (uint32_t)bf16_bits(v[1]) << 16;
    }
    __syncthreads();
  }
}

// ---- scores of blocks.
//
// With k_j the mean key of block j and J the blocks that query row i may choose
// from, its score of j is
//   sum over heads h of exp(s_hj) / sum over j' in J of exp(s_hj'),
//   s_hj = scale (q_lat,h . k_lat,j + q_pe,h . k_pe,j):
// the share of its attention that each head would give the block if its 64 keys
// were their mean, added over the heads, which share one selection.
//
// Two passes over the logits, since a head's weights need its sum over all
// blocks: the first leaves each split's largest logit and sum of a row, the second
// forms the logits again and adds the weights up (the same workgroup where there
// is one split).  Logits kept between the passes would move 8 bytes a head and
// block, the keys again 1152 a block for all heads, mostly out of the caches.
//
// A workgroup of eight waves, two on a SIMD, takes 64 blocks at a time in LDS, the next
// 64's keys on their way (direct-to-LDS loads spread over the products); its waves share
// out 16-row chunks (the heads of one query row, padded) and the columns of 16 blocks.
// bf16 MFMA 16x16x32 with the query rows in registers for the whole kernel, fp32 sums.
//
// What bounds it: for decode rows the keys out of HBM and the chain before the first
// tile, in each of two launches (64 requests of 128 rows over up to 1024 blocks, 72 MB a pass:
// 36 us, of which 18 a pass in one tile's chain and 3.4 tiles at 1.3 to 2); for prompts a
// tile's 2 us, 1.1 of them products, the rest LDS (each wave reads its columns' keys for
// 32 rows only) and exponentials.  From there: the table's entry read under a condition
// was waited for in every tile, and query rows taken from memory as the products need
// them (64 bytes of 16 rows a load) cost 7 us a launch: 49 us with both.  Four waves with
// the exponentials of a tile beside the next one's products took 101 us where eight plain
// ones take 69 (one split).
constexpr int kKeyBytes = 2 * kMeanCols;       // 1152: 72 chunks of 16 bytes
constexpr int kSteps = kMeanCols / 32;         // of a product: 18

// A tile's keys in LDS: latent rows of 1 KiB, 16-byte chunk c of row t in place c ^
// lat_swizzle(t), then RoPE rows of 128 bytes, chunk c in place c ^ rope_swizzle(t).  The
// LDS serves 16 lanes of a 16-byte read at once, rows {0..3, 8..11} of 16 (or the others)
// of two neighbouring chunks: latent rows all begin in one bank, RoPE rows in one of two
// by their lowest bit, and the swizzles put the rest of the row's bits beside the
// chunk's.
__device__ __forceinline__ int lat_swizzle(int t) { return (t & 3) << 2 | ((t >> 3) & 1) << 1; }
__device__ __forceinline__ int rope_swizzle(int t) { return ((t >> 1) & 1) << 1 | ((t >> 3) & 1) << 2; }

// 16 bytes a lane from base + off to dst + 16 * lane; base and dst the same in every lane.
// The wait for it is the code's own: written as asm, since the compiler would wait before
// every LDS read that follows.
__device__ __forceinline__ void to_lds(const uint8_t* base, uint32_t off, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :: "v"(off), "s"(base), "s"(__builtin_amdgcn_readfirstlane(dst)) : "memory", "m0");
}
__device__ __forceinline__ void to_lds(const uint8_t* src, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :: "v"(src), "s"(__builtin_amdgcn_readfirstlane(dst)) : "memory", "m0");
}
__device__ __forceinline__ bf16x8_t lds_read(uint32_t at, int offset) {
  return *(const __attribute__((address_space(3))) bf16x8_t*)(uintptr_t)(at + (uint32_t)offset);
}
constexpr int kWaitLoads = (7 << 4) | (15 << 8);  // s_waitcnt vmcnt(0)

// Sum over lanes l, l ^ 16, l ^ 32, l ^ 48 by the row-swap permutes, which leave the
// other's value beside the own one.
__device__ __forceinline__ float over_rows(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const uint32_t w = __float_as_uint(v);
  const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// op over the 16 lanes of a row of lanes, by rotations within it.
template <class Op>
__device__ __forceinline__ float over_cols(float v, Op op) {
  auto turned = [](float x, auto by) {
    const int u = __float_as_int(x);
    return __int_as_float(__builtin_amdgcn_update_dpp(u, u, 0x120 + decltype(by)::value, 0xF, 0xF, false));
  };
  v = op(v, turned(v, std::integral_constant<int, 1>{}));
  v = op(v, turned(v, std::integral_constant<int, 2>{}));
  v = op(v, turned(v, std::integral_constant<int, 4>{}));
  return op(v, turned(v, std::integral_constant<int, 8>{}));
}

// Statistics (largest logit, sum of exponentials against it) of two sets, joined.
__device__ __forceinline__ f32x2_t join(f32x2_t a, f32x2_t b) {
  const float m = fmaxf(a[0], b[0]), top = fmaxf(m, -3.4e38f);
  return f32x2_t{m, a[1] * __builtin_amdgcn_exp2f(a[0] - top) + b[1] * __builtin_amdgcn_exp2f(b[0] - top)};
}
// What a logit is taken off by so that the exponentials of all are weights.
__device__ __forceinline__ float norm_of(f32x2_t a) { return fmaxf(a[0], -3.4e38f) + __builtin_amdgcn_logf(a[1]); }

// WR waves along the rows, 8 / WR along the columns, NC chunks and COLS columns of 16
// blocks a wave.  PASS 0: both passes; 1: the statistics of a split; 2: the scores,
// given those of all splits.
template <int WR, int NC, int COLS, int PASS>
__global__ __launch_bounds__(kScoreThreads, 2) void scores_kernel(const ScoresParams p) {
  constexpr int kThreads = kScoreThreads, WK = kThreads / 64 / WR;
  constexpr int kTile = kScoreCols;            // blocks of a tile
  static_assert(WK * COLS * 16 == kTile, "a wave's columns");
  constexpr int kSlots = WR * NC;              // chunks of the workgroup
  constexpr int kRope = kTile * 2 * kDLat, kBuffer = kTile * kKeyBytes;
  constexpr int kLoads = 9;                    // of a wave for a tile
  static_assert(kTile == 8 * (kThreads / 64) && kSteps == 2 * kLoads, "a load of the next tile beside two steps' products");
  __shared__ __attribute__((aligned(1024))) uint8_t keys[2 * kBuffer];
  __shared__ float part[2][kSlots][kTile];
  __shared__ f32x2_t stat[WK][kSlots][16];
  __shared__ int32_t is_block[2][kTile];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const int wr = wave / WK, wk = wave % WK;

  // work item: request, group of query rows, split
  // (a request's splits on one XCD, whose L2 then holds its query rows)
  const int w = gridDim.x % 8 ? (int)blockIdx.x : (int)(blockIdx.x % 8) * (int)(gridDim.x / 8) + (int)(blockIdx.x / 8);
  const int a = div_by(w, p.by_splits);
  const int split = w - a * p.n_splits;
  const int b = div_by(a, p.by_groups);
  const int i0 = (a - b * p.n_groups) * p.group_rows;
  const int n_i = min(p.group_rows, p.Mq - i0);
  const int len = max(p.lens[b], 0);
  const int qn = min(max(p.q_lens ? p.q_lens[b] : p.Mq, 0), p.Mq);
  // blocks lo .. end_of(i) - 1 may be chosen by row i
  const int lo = p.first_block;
  auto end_of = [&](int i) {
    const int64_t past = (int64_t)len - qn + i + 1 - p.window;
    return i < qn && past > 0 ? (int)min(past / kBlock, (int64_t)p.NB) : 0;
  };
  const int end = i0 < qn ? end_of(min(i0 + n_i, qn) - 1) : 0;
  const int tile0 = lo / kTile, tiles = end > lo ? (end - 1) / kTile - tile0 + 1 : 0;
  const int t0 = tile0 + (int)((int64_t)tiles * split / p.n_splits);
  const int t1 = tile0 + (int)((int64_t)tiles * (split + 1) / p.n_splits);

  float* const out = p.out + (int64_t)b * p.out_s0;
  if constexpr (PASS != 1) {
    // columns of no tile, shared out over the splits
    const int c0 = tiles > 0 ? tile0 * kTile : 0, c1 = tiles > 0 ? (tile0 + tiles) * kTile : 0;
    for (int i = i0; i < i0 + n_i; ++i) {
      float* const row = out + (int64_t)i * p.out_s1;
      for (int c = split * kThreads + tid; c < p.NB; c += p.n_splits * kThreads)
        if (c < c0 || c >= c1) row[c] = -INFINITY;
    }
  }
  if (t0 == t1 && PASS != 1) return;

  // the keys on their way: wave w loads rows 8 w .. 8 w + 7, a latent row a load, then
  // their RoPE rows in one
  const int32_t* const table = p.table + b * p.table_s0;
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)keys;
  // of row 8 w + (lane & 7): the table's entry of the tile that is loaded next, and its
  // tile (read a tile ahead, whatever it is: a read under a condition would be waited for
  // where the condition ends)
  int id = 0, id_tile = 0, row_of = 0;
  auto ids_of = [&](int t) {
    int l = (int)threadIdx.x & 7;
    asm volatile("" : "+v"(l));
    const int j = t * kTile + 8 * wave + l;
    id = table[min(max(j, lo), end - 1)];
    id_tile = t;
  };
  auto aim_keys = [&](int buffer) {
    const int j = id_tile * kTile + 8 * wave + (lane & 7);
    const bool is = j >= lo && j < end && id >= 0 && id < p.P;
    row_of = is ? id : 0;
    if (lane < 8) is_block[buffer][8 * wave + lane] = is;
  };
  const int half8 = wave & 1;  // the wave's rows are the upper eight of 16
  auto load_key = [&](int buffer, int s) {  // of kLoads
    const uint32_t to = lds + (uint32_t)(buffer * kBuffer);
    // (the lane's offsets are formed here, not held: registers are short)
    int lane = (int)(threadIdx.x & 63);
    asm volatile("" : "+v"(lane));
    if (s < 8) {
      const int64_t row = __builtin_amdgcn_readlane(row_of, s);
      to_lds(p.means + row * kKeyBytes, (uint32_t)((lane ^ lat_swizzle(s) ^ half8 << 1) << 4),
             to + (uint32_t)((8 * wave + s) * 1024));
    } else {
      const int t = lane >> 3;
      const int64_t row = __shfl(row_of, t);
      to_lds(p.means + row * kKeyBytes + 2 * kDLat + (((lane & 7) ^ rope_swizzle(t) ^ half8 << 2) << 4),
             to + (uint32_t)(kRope + 8 * wave * 128));
    }
  };
  // tiles t0 .. t1 - 1, in each pass; the one after t (in the second pass the first
  // again)
  auto after = [&](int t) { return t + 1 < t1 ? t + 1 : t0; };

  // head chunks of the query rows: chunk c of the group is heads 16 (c mod C) .. of
  // row i0 + c / C; more than kSlots of them (one query row of many heads) go in
  // rounds
  const int C = p.row_chunks;
  const int n_chunks = n_i * C;
  const int rounds = (n_chunks + kSlots - 1) / kSlots;
  for (int round = 0; round < rounds; ++round) {
    // The query rows come through the keys' place in LDS, a chunk by each of the first
    // waves: read from memory as the products take them, 16 rows a load by 64 bytes each,
    // they took longer than four tiles.
    constexpr int kQRope = kSlots * 16 * 2 * kDLat;
    static_assert(kQRope + kSlots * 16 * 2 * kDPe <= 2 * kBuffer, "the query rows fit the keys' place");
    if (wave < kSlots) {
      const int c = min(round * kSlots + wave, n_chunks - 1), ci = div_by(c, p.by_chunks), h = 16 * (c - ci * C);
      const uint16_t* const ql = p.q_lat + b * p.ql_s0 + (int64_t)(i0 + ci) * p.ql_s1;
      const uint16_t* const qp = p.q_pe + b * p.qp_s0 + (int64_t)(i0 + ci) * p.qp_s1;
      // (rows past the heads repeat the last one: a key that is infinite is then no NaN
      // that the head does not have)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        to_lds((const uint8_t*)(ql + min(h + r, p.H - 1) * p.ql_s2), (uint32_t)((lane ^ lat_swizzle(r)) << 4),
               lds + (uint32_t)((16 * wave + r) * 1024));
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int t = 8 * r + (lane >> 3);
        to_lds((const uint8_t*)(qp + min(h + t, p.H - 1) * p.qp_s2) + (((lane & 7) ^ rope_swizzle(t)) << 4),
               lds + (uint32_t)(kQRope + (16 * wave + 8 * r) * 128));
      }
    }
    if (t0 < t1) ids_of(t0);
    if constexpr (PASS == 2) {
      // what the rows' weights are taken off by: of all splits, four threads a row
      int e0 = (int)threadIdx.x;
      asm volatile("" : "+v"(e0));
      for (int e = e0; e < kSlots * 64; e += kThreads) {
        const int c = min(round * kSlots + e / 64, n_chunks - 1), r = e / 4 % 16;
        const f32x2_t* const at = (const f32x2_t*)p.stats + (((int64_t)a * p.group_chunks + c) * 16 + r) * p.n_splits;
        f32x2_t y{-INFINITY, 0.f};
        for (int s = e & 3; s < p.n_splits; s += 4) y = join(y, at[s]);
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) y = join(y, f32x2_t{__shfl_xor(y[0], o), __shfl_xor(y[1], o)});
        if ((e & 3) == 0) stat[0][e / 64][r] = f32x2_t{norm_of(y), 0.f};
      }
    }
    __builtin_amdgcn_s_waitcnt(kWaitLoads);
    __syncthreads();
    bf16x8_t q[NC][kSteps];
    int h0[NC], chunk_end[NC];
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = round * kSlots + wr * NC + k;
      const bool is = c < n_chunks;
      const int ci = is ? div_by(c, p.by_chunks) : 0;
      h0[k] = is ? 16 * (c - ci * C) : p.H;
      chunk_end[k] = is ? end_of(i0 + ci) : 0;
      const uint32_t ql = lds + (uint32_t)((16 * (wr * NC + k) + n16) * 1024 + ((g ^ lat_swizzle(n16)) << 4));
      const uint32_t qp = lds + (uint32_t)(kQRope + (16 * (wr * NC + k) + n16) * 128 + ((g ^ rope_swizzle(n16)) << 4));
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
        q[k][s] = s < kDLat / 32 ? lds_read(ql ^ (uint32_t)((s & 3) << 6), (s >> 2) * 256) : lds_read(qp ^ (uint32_t)((s & 1) << 6), 0);
    }
    __syncthreads();  // every wave holds its query rows: their place takes keys
    int buffer = 0;
    if (t0 < t1) {
      aim_keys(buffer);
#pragma unroll
      for (int s = 0; s < kLoads; ++s) load_key(buffer, s);
      ids_of(after(t0));
    }
    // of rows 16 chunk + 4 g + r: the largest logit and sum of this lane's columns
    // (log2 units), in the second pass what norm_of gives of all (of no head: +inf, so
    // that its weights are 0)
    float m[NC][4], l[NC][4];
#pragma unroll
    for (int k = 0; k < NC; ++k)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        m[k][r] = -INFINITY;
        l[k][r] = 0.f;
      }
    auto norms = [&](auto of) {
#pragma unroll
      for (int k = 0; k < NC; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) m[k][r] = h0[k] + 4 * g + r < p.H ? of(wr * NC + k, 4 * g + r) : INFINITY;
    };
    if constexpr (PASS == 2) norms([&](int c, int r) { return stat[0][c][r][0]; });

    // Of the scores that a pass has summed up to a row's chunks in part: a query row's
    // chunks, in order; more than one round's are added up in place (by the same thread)
    auto finish = [&](int t) {
      const int c0 = round * kSlots, c1 = min(n_chunks, c0 + kSlots);
      int e0 = (int)threadIdx.x;
      asm volatile("" : "+v"(e0));
      for (int e = e0; e < n_i * kTile; e += kThreads) {
        const int ii = e / kTile, n = e % kTile, j = t * kTile + n;
        const int from = max(ii * C, c0), to = min((ii + 1) * C, c1);
        if (from >= to || j >= p.NB) continue;
        float* const at = out + (int64_t)(i0 + ii) * p.out_s1 + j;
        float sum = from > ii * C ? *at : 0.f;
        for (int c = from; c < to; ++c) sum += part[t & 1][c - c0][n];
        *at = sum;
      }
    };
    // the lane's places in a tile of its key fragments: chunk 4 s + g of row 16 c + n16;
    // s moves the place by an XOR of the two bits above g's and by whole 256 (128) bytes
    const uint32_t lat_at = lds + (uint32_t)((16 * wk * COLS + n16) * 1024 + ((g ^ lat_swizzle(n16)) << 4));
    const uint32_t rope_at = lds + (uint32_t)(kRope + (16 * wk * COLS + n16) * 128 + ((g ^ rope_swizzle(n16)) << 4));

    auto run = [&](auto second) {
      constexpr bool kScores = decltype(second)::value;  // the second pass
      for (int t = t0; t < t1; ++t) {
        // the tile has landed, and every wave is past the one before it
        __builtin_amdgcn_s_waitcnt(kWaitLoads);
        __syncthreads();
        const uint32_t here = (uint32_t)(buffer * kBuffer);
        bool may[NC][COLS];
#pragma unroll
        for (int c = 0; c < COLS; ++c) {
          const int n = 16 * (wk * COLS + c) + n16;
          const int is = is_block[buffer][n];
#pragma unroll
          for (int k = 0; k < NC; ++k) may[k][c] = (is & (int)(t * kTile + n < chunk_end[k])) != 0;
        }
        buffer ^= 1;
        const bool more = t + 1 < t1 || (PASS == 0 && !kScores);
        if (more) aim_keys(buffer);
        if (kScores && t > t0) finish(t - 1);
        // key fragments are read two steps before their products, into the registers that
        // the last ones' have left (left to itself the compiler waits for each where it is
        // used); the fences keep it so
        constexpr int kAhead = 2;
        bf16x8_t kf[kAhead][COLS];
        const uint32_t la = lat_at + here, ra = rope_at + here;
        auto read_step = [&](int s) {
#pragma unroll
          for (int c = 0; c < COLS; ++c)
            kf[s % kAhead][c] = s < kDLat / 32 ? lds_read(la ^ (uint32_t)((s & 3) << 6), (s >> 2) * 256 + c * 16384)
                                          : lds_read(ra ^ (uint32_t)((s & 1) << 6), c * 2048);
        };
#pragma unroll
        for (int s = 0; s < kAhead; ++s) read_step(s);
        f32x4_t acc[NC][COLS];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          if (more && (s & 1) == 0) load_key(buffer, s >> 1);
#pragma unroll
          for (int c = 0; c < COLS; ++c)
#pragma unroll
            for (int k = 0; k < NC; ++k)
              acc[k][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  q[k][s], kf[s % kAhead][c], s == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : acc[k][c], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
          if (s + kAhead < kSteps) read_step(s + kAhead);
          __builtin_amdgcn_sched_barrier(0);
        }
        if (more) ids_of(after(after(t)));
        if constexpr (!kScores) {
#pragma unroll
          for (int k = 0; k < NC; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              float x[COLS], mx = m[k][r];
#pragma unroll
              for (int c = 0; c < COLS; ++c) {
                x[c] = acc[k][c][r] * p.scale_log2;
                x[c] = may[k][c] ? x[c] : -INFINITY;
                mx = fmaxf(mx, x[c]);
              }
              const float top = fmaxf(mx, -3.4e38f);
              float sum = l[k][r] * __builtin_amdgcn_exp2f(m[k][r] - top);
#pragma unroll
              for (int c = 0; c < COLS; ++c) sum += __builtin_amdgcn_exp2f(x[c] - top);
              l[k][r] = sum;
              m[k][r] = mx;
            }
        } else {
#pragma unroll
          for (int k = 0; k < NC; ++k)
#pragma unroll
            for (int c = 0; c < COLS; ++c) {
              float x[4];
#pragma unroll
              for (int r = 0; r < 4; ++r) x[r] = __builtin_amdgcn_exp2f(acc[k][c][r] * p.scale_log2 - m[k][r]);
              const float sum = over_rows((x[0] + x[1]) + (x[2] + x[3]));
              if (g == 0) part[t & 1][wr * NC + k][16 * (wk * COLS + c) + n16] = may[k][c] ? sum : -INFINITY;
            }
        }
      }
      if constexpr (kScores) {
        __syncthreads();
        if (t0 < t1) finish(t1 - 1);
      }
    };
    if constexpr (PASS != 2) {
      run(std::false_type{});
      // a row's statistics: of the lanes that share it, then of the waves
#pragma unroll
      for (int k = 0; k < NC; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float mm = over_cols(m[k][r], [](float u, float v) { return fmaxf(u, v); });
          const float ll = over_cols(l[k][r] * __builtin_amdgcn_exp2f(m[k][r] - fmaxf(mm, -3.4e38f)),
                                     [](float u, float v) { return u + v; });
          const f32x2_t y{mm, ll};
          if (n16 == 0) stat[wk][wr * NC + k][4 * g + r] = y;
        }
      __syncthreads();
      if constexpr (PASS == 1) {
        for (int e = tid; e < kSlots * 16; e += kThreads) {
          const int c = round * kSlots + e / 16, r = e % 16;
          if (c >= n_chunks) continue;
          f32x2_t y = stat[0][e / 16][r];
#pragma unroll
          for (int k = 1; k < WK; ++k) y = join(y, stat[k][e / 16][r]);
          ((f32x2_t*)p.stats)[(((int64_t)a * p.group_chunks + c) * 16 + r) * p.n_splits + split] = y;
        }
      } else {
        norms([&](int c, int r) {
          f32x2_t y = stat[0][c][r];
#pragma unroll
          for (int v = 1; v < WK; ++v) y = join(y, stat[v][c][r]);
          return norm_of(y);
        });
      }
    }
    if constexpr (PASS != 1) run(std::true_type{});
    __syncthreads();
  }
}

// ---- the K best of each row.
//
// Values are ordered as 32-bit keys that grow with them (NaN above all, -0 as 0).  A
// workgroup holds a row's keys in registers and narrows down the range in which the
// K-th largest lies: a histogram of the keys in the range (the upper bits of where in it
// they lie, so that the bins follow the values there are), then the bin that holds it.  All keys above the range are then taken, and those in it where
// it comes down to one key, the first ones in the order of their places.  -inf is
// never taken.
//
// Read once, written once; bound by the launch and by the dependent steps of the search:
// 64 rows of 1024 values take 4.3 us, one of 8192 8.7, of 16,384 11.7.  A search bit by
// bit over a wave's registers took 10.1 us for 64 rows of 1024, one that reads the row
// again for each byte of the key 111 for 32 of 65,536, which now go in eight pieces of
// 8192 and then in one row of 16,384: 22 us.

__device__ __forceinline__ uint32_t order_key(float v) {
  if (v != v) return 0xFFFFFFFFu;
  const uint32_t u = v == 0.f ? 0u : __float_as_uint(v);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr uint32_t kLowestKey = 0x007FFFFFu;  // of -inf
// op over a wave, in every lane: by rotations within 16 lanes, then by the row swaps.
template <class Op>
__device__ __forceinline__ uint32_t over_wave(uint32_t v, Op op) {
  auto turned = [](uint32_t x, auto by) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x120 + decltype(by)::value, 0xF, 0xF, false);
  };
  v = op(v, turned(v, std::integral_constant<int, 1>{}));
  v = op(v, turned(v, std::integral_constant<int, 2>{}));
  v = op(v, turned(v, std::integral_constant<int, 4>{}));
  v = op(v, turned(v, std::integral_constant<int, 8>{}));
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = op(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return op(b[0], b[1]);
}

// Sum of v over lanes 0 .. the own one.
__device__ __forceinline__ int lanes_up(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true);   // within rows of 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // lane 15 to row 1, 47 to row 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // lane 31 to rows 2 and 3
  return v;
}

// Of a histogram, the bin that holds the `want`-th key from the top, and how many of the
// wanted lie in it (by the first wave; want <= the number of keys).
template <int BINS>
__device__ __forceinline__ void find_bin(const uint32_t* hist, uint32_t want, int lane, int* bin, uint32_t* left,
                                         uint32_t* in_bin) {
  // lane l holds the l-th BINS / 64 bins from the top, the lowest first
  constexpr int kPer = BINS / 64;
  const u32x4_t* const at = (const u32x4_t*)(hist + BINS - kPer * (lane + 1));
  u32x4_t c[kPer / 4];
  uint32_t sum = 0;
#pragma unroll
  for (int j = 0; j < kPer / 4; ++j) {
    c[j] = at[j];
    sum += (c[j][0] + c[j][1]) + (c[j][2] + c[j][3]);
  }
  uint32_t past = (uint32_t)lanes_up((int)sum) - sum;  // in the bins above the lane's
  const uint64_t few = __ballot(past < want);
  if (lane == 63 - __builtin_clzll(few)) {  // the last lane with fewer than `want` above it
    int b = kPer - 1;
    uint32_t here = 0;
#pragma unroll
    for (int j = kPer - 1; j >= 0; --j) {
      const uint32_t n = c[j / 4][j % 4];
      if (j == b) {
        here = n;
        if (j > 0 && past + n < want) {
          past += n;
          b = j - 1;
        }
      }
    }
    *bin = BINS - kPer * (lane + 1) + b;
    *left = want - past;
    *in_bin = here;
  }
}

// A row, or a piece of THREADS E places of it, by THREADS threads, E values each: value e
// of thread t is place e THREADS + t.  A long row goes in pieces first, whose best make
// up a shorter row (with their places beside them, in order): of a piece's values no
// more than K can be among the row's K best.
template <int THREADS, int E>
__global__ __launch_bounds__(THREADS) void topk_kernel(const TopkParams p) {
  // (bins: of a range over both signs and all exponents 1024 still tell eight values of an
  // exponent apart, 32 rows of 16,384 normal values 14.4 us against 17.0 with 256, one of
  // 8192 9.2 against 10.7; few threads clear and search 256 faster, 64 rows of 1024 4.6 us
  // against 4.9, of normal values 4.8 against 6.1)
  constexpr int kWaves = THREADS / 64, kBits = THREADS > 256 ? 10 : 8, kBins = 1 << kBits;
  __shared__ __attribute__((aligned(16))) uint32_t hist[2][kBins];
  __shared__ uint32_t wave_lo[kWaves], wave_hi[kWaves];
  __shared__ int wave_n[kWaves];
  // of 64 neighbours: (above, equal << 16), then the places taken before them; equal ones before them
  __shared__ int counts[E * kWaves], eq_before[E * kWaves];
  __shared__ int n_taken;
  __shared__ int found;
  __shared__ uint32_t left, in_bin;
  const int64_t row = p.first_row + blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t b = div_by((int)row, p.by_Mq), i = row - b * p.Mq;
  const int first = (int)blockIdx.y * (THREADS * E), N = min(p.N - first, THREADS * E);
  const float* const x = p.x + b * p.x_s0 + i * p.x_s1 + first;
  const int32_t* const places = p.places ? p.places + row * p.N + first : nullptr;
  int32_t* const ids = p.ids + b * p.ids_s0 + i * p.ids_s1 + (int64_t)blockIdx.y * p.K;
  float* const best = p.best ? p.best + (row * gridDim.y + blockIdx.y) * p.K : nullptr;
  uint32_t key[E];  // (past the row's places that of -inf, which is never taken)
  {
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = e * THREADS + tid < N ? x[e * THREADS + tid] : -INFINITY;
#pragma unroll
    for (int e = 0; e < E; ++e) key[e] = order_key(v[e]);
  }
  // the range of the keys above -inf, and their number
  uint32_t lo = 0xFFFFFFFFu, hi = 0u;
  int n = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const bool is = key[e] > kLowestKey;
    lo = is ? min(lo, key[e]) : lo;
    hi = is ? max(hi, key[e]) : hi;
    n += is ? 1 : 0;
  }
  lo = over_wave(lo, [](uint32_t u, uint32_t v) { return min(u, v); });
  hi = over_wave(hi, [](uint32_t u, uint32_t v) { return max(u, v); });
  n = (int)over_wave((uint32_t)n, [](uint32_t u, uint32_t v) { return u + v; });
  for (int t = tid; t < 2 * kBins; t += THREADS) ((uint32_t*)hist)[t] = 0;
  if (lane == 0) {
    wave_lo[wave] = lo;
    wave_hi[wave] = hi;
    wave_n[wave] = n;
  }
  __syncthreads();
  n = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    lo = min(lo, wave_lo[w]);
    hi = max(hi, wave_hi[w]);
    n += wave_n[w];
  }
  // keys above hi are taken; of those in lo .. hi `want`
  uint32_t want = (uint32_t)min(p.K, n);
  if (n <= p.K) {
    hi = kLowestKey;
    lo = kLowestKey;
    want = 0;
  }
  for (int turn = 0; lo < hi; turn ^= 1) {
    const int bits = 32 - __builtin_clz(hi - lo), shift = max(bits - kBits, 0);
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (key[e] >= lo && key[e] <= hi) atomicAdd(&hist[turn][(key[e] - lo) >> shift], 1u);
    __syncthreads();
    if (wave == 0) find_bin<kBins>(hist[turn], want, lane, &found, &left, &in_bin);
    for (int t = tid; t < kBins; t += THREADS) hist[turn ^ 1][t] = 0;
    __syncthreads();
    want = left;
    lo += (uint32_t)found << shift;
    hi = lo + min(hi - lo, (1u << shift) - 1);
    if (want == in_bin) {  // all of the bin
      hi = lo - 1;
      want = 0;
    }
  }
  // places before each 64 neighbours'
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const uint64_t gt = __ballot(key[e] > hi), eq = __ballot(want != 0 && key[e] == hi);
    if (lane == 0) counts[e * kWaves + wave] = (int)__popcll(gt) | (int)__popcll(eq) << 16;
  }
  __syncthreads();
  // one wave sums them up, some neighbours a lane
  if (wave == 0) {
    constexpr int kPer = (E * kWaves + 63) / 64;
    int above = 0, equal = 0;
#pragma unroll 4
    for (int k = 0; k < kPer; ++k) {
      const int at = lane * kPer + k;
      const int c = at < E * kWaves ? counts[at] : 0;
      above += c & 0xFFFF;
      equal += c >> 16;
    }
    int a = lanes_up(above) - above, q = lanes_up(equal) - equal;
#pragma unroll 4
    for (int k = 0; k < kPer; ++k) {
      const int at = lane * kPer + k;
      if (at < E * kWaves) {
        const int c = counts[at];
        // (of equal keys, no more count than are wanted)
        counts[at] = a + min(q, (int)want);
        eq_before[at] = q;
        a += c & 0xFFFF;
        q += c >> 16;
      }
    }
    if (lane == 63) n_taken = a + min(q, (int)want);
  }
  __syncthreads();
  const uint64_t before = (1ull << lane) - 1;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const uint64_t gt = __ballot(key[e] > hi), eq = __ballot(want != 0 && key[e] == hi);
    if ((gt | eq) == 0) continue;
    const int base = counts[e * kWaves + wave], q0 = eq_before[e * kWaves + wave];
    const int mine = q0 + (int)__popcll(eq & before);
    const bool take = key[e] > hi || (want != 0 && key[e] == hi && mine < (int)want);
    if (take) {
      const int at = base + (int)__popcll(gt & before) + min(mine, (int)want) - min(q0, (int)want);
      const int place = e * THREADS + tid;
      ids[at] = places ? places[place] : first + place;
      if (best) best[at] = x[place];
    }
  }
  for (int k = n_taken + tid; k < p.K; k += THREADS) {
    ids[k] = -1;
    if (best) best[k] = -INFINITY;
  }
}

// A row of any length by one workgroup, read from memory in each round: eight bits
// of the K-th largest key a round, by a histogram of the values that share the bits
// found before.  Rows that went in pieces come here too, where they are still longer
// than the kernel above holds.  Five reads of the row by one workgroup: 32 rows of
// 262,144 with K 8192 take 461 us, of 139,264 with K 4096 (69,632 left of them) 182.
constexpr int kTopThreads = 1024;
__global__ __launch_bounds__(kTopThreads) void topk_row_kernel(const TopkParams p) {
  constexpr int kBins = 256;
  __shared__ __attribute__((aligned(16))) uint32_t hist[kBins];
  __shared__ int wave_above[kTopThreads / 64], wave_equal[kTopThreads / 64];
  __shared__ int found;
  __shared__ uint32_t left, in_bin;
  const int64_t row = p.first_row + blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t b = div_by((int)row, p.by_Mq), i = row - b * p.Mq;
  const float* const x = p.x + b * p.x_s0 + i * p.x_s1;
  const int32_t* const places = p.places ? p.places + row * p.N : nullptr;
  int32_t* const ids = p.ids + b * p.ids_s0 + i * p.ids_s1;
  uint32_t top = 0;
  int want = min(p.K, p.N);  // of the values that share top's bits so far, so many are taken
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < kBins) hist[tid] = 0;
    __syncthreads();
    for (int e = tid; e < p.N; e += kTopThreads) {
      const uint32_t k = order_key(x[e]);
      if (shift == 24 || k >> (shift + 8) == top >> (shift + 8)) atomicAdd(&hist[k >> shift & 255], 1u);
    }
    __syncthreads();
    if (wave == 0) find_bin<kBins>(hist, (uint32_t)want, lane, &found, &left, &in_bin);
    __syncthreads();
    top |= (uint32_t)found << shift;
    want = (int)left;
    __syncthreads();
  }
  if (top <= kLowestKey) {  // fewer than K above -inf: all of those
    top = kLowestKey;
    want = 0;
  }
  int at = 0;
  const uint64_t before = (1ull << lane) - 1;
  for (int e0 = 0; e0 < p.N; e0 += kTopThreads) {
    const int e = e0 + tid;
    const uint32_t k = e < p.N ? order_key(x[e]) : 0u;
    const uint64_t gt = __ballot(k > top), eq = __ballot(k == top);
    if (lane == 0) {
      wave_above[wave] = (int)__popcll(gt);
      wave_equal[wave] = (int)__popcll(eq);
    }
    __syncthreads();
    int a0 = 0, q0 = 0, an = 0, qn = 0;
#pragma unroll
    for (int w = 0; w < kTopThreads / 64; ++w) {
      if (w == wave) {
        a0 = an;
        q0 = qn;
      }
      an += wave_above[w];
      qn += wave_equal[w];
    }
    // places taken before this one: those above, and of those equal at most `want`
    const int eq_before = q0 + (int)__popcll(eq & before);
    const bool take = k > top || (k == top && eq_before < want);
    if (take) ids[at + a0 + (int)__popcll(gt & before) + min(eq_before, want)] = places ? places[e] : e;
    at += an + min(qn, want);
    want -= min(qn, want);
    __syncthreads();
  }
  for (int k = at + tid; k < p.K; k += kTopThreads) ids[k] = -1;
}

}  // namespace

hipError_t launch_means(const MeansParams& p0, int kv, hipStream_t s) {
  if (p0.T <= 0) return hipSuccess;
  // about 2048 workgroups, one a slot below that
  MeansParams p = p0;
  const int64_t per = (p.T + 2047) / 2048, window = p.T < kMeanWindow ? p.T : kMeanWindow;
  p.sharers = (int32_t)((window + per - 1) / per);
  p.by_sharers = make_div(p.sharers);
  const int64_t grid = (p.T + kMeanWindow - 1) / kMeanWindow * p.sharers;
  const dim3 g((uint32_t)grid), b(kThreads);
  if (kv == kKvMx4) hipLaunchKernelGGL(means_kernel<kKvMx4>, g, b, 0, s, p);
  else if (kv == kKvBf16) hipLaunchKernelGGL(means_kernel<kKvBf16>, g, b, 0, s, p);
  else hipLaunchKernelGGL(means_kernel<kKvFp8Shared>, g, b, 0, s, p);
  return hipGetLastError();
}

template <int WR, int NC, int COLS>
static void launch_scores_rows(const ScoresParams& p, int grid, hipStream_t s) {
  const dim3 g((uint32_t)grid), b(kScoreThreads);
  if (p.n_splits == 1) {
    hipLaunchKernelGGL((scores_kernel<WR, NC, COLS, 0>), g, b, 0, s, p);
    return;
  }
  hipLaunchKernelGGL((scores_kernel<WR, NC, COLS, 1>), g, b, 0, s, p);
  hipLaunchKernelGGL((scores_kernel<WR, NC, COLS, 2>), g, b, 0, s, p);
}

hipError_t launch_scores(const ScoresParams& p, int B, hipStream_t s) {
  const int grid = B * p.n_groups * p.n_splits;
  if (grid <= 0) return hipSuccess;
  if (p.shape == kScores128) launch_scores_rows<4, 2, 2>(p, grid, s);
  else if (p.shape == kScores64) launch_scores_rows<2, 2, 1>(p, grid, s);
  else launch_scores_rows<2, 1, 1>(p, grid, s);
  return hipGetLastError();
}

static hipError_t launch_topk_rows(const TopkParams& p, int64_t rows, int pieces, hipStream_t s) {
  const dim3 g((uint32_t)rows, (uint32_t)pieces);
  if (pieces > 1) {
    static_assert(kTopPiece == 512 * 16, "a piece of the kernel");
    hipLaunchKernelGGL((topk_kernel<512, 16>), g, dim3(512), 0, s, p);
  } else if (p.N <= 256) {
    hipLaunchKernelGGL((topk_kernel<64, 4>), g, dim3(64), 0, s, p);
  } else if (p.N <= 1024) {
    hipLaunchKernelGGL((topk_kernel<256, 4>), g, dim3(256), 0, s, p);
  } else if (p.N <= 4096) {
    hipLaunchKernelGGL((topk_kernel<512, 8>), g, dim3(512), 0, s, p);
  } else if (p.N <= 8192) {
    hipLaunchKernelGGL((topk_kernel<512, 16>), g, dim3(512), 0, s, p);
  } else if (p.N <= 16384) {
    hipLaunchKernelGGL((topk_kernel<1024, 16>), g, dim3(1024), 0, s, p);
  } else if (p.N <= kTopMost) {
    static_assert(kTopMost == 1024 * 64, "the longest row of the kernel");
    hipLaunchKernelGGL((topk_kernel<1024, 64>), g, dim3(1024), 0, s, p);
  } else {
    hipLaunchKernelGGL(topk_row_kernel, g, dim3(kTopThreads), 0, s, p);
  }
  return hipGetLastError();
}

hipError_t launch_topk(const TopkParams& p0, int pieces, hipStream_t s) {
  // one launch holds less than 2^32 threads (past that its size wraps, without an
  // error): 2^31 at a time
  TopkParams p = p0;
  const int64_t most = std::max<int64_t>(1, (1 << 21) / pieces);
  for (p.first_row = 0; p.first_row < p.rows; p.first_row += most) {
    const hipError_t e = launch_topk_rows(p, std::min<int64_t>(most, p.rows - p.first_row), pieces, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace mla
