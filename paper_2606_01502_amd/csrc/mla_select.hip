// What chooses the blocks a query row attends: the mean keys of whole blocks, the
// scores of a request's blocks by them, and the choice of the best.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mla_kernels.h"
#include "mla_mx4.h"

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
// trips where few blocks are whole.
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
// A workgroup takes a tile of blocks at a time in LDS, the next tile's keys on their
// way (direct-to-LDS loads); its waves share out 16-row chunks (the heads of one query row,
// padded) and the tile's columns of 16 blocks.  bf16 MFMA 16x16x32 with the query
// rows in registers for the whole kernel.  128 rows a workgroup where there are as
// many, and two workgroups a compute unit: one's loads and exponentials run beside the
// other's products.
constexpr int kKeyBytes = 2 * kMeanCols;       // 1152: 72 chunks of 16 bytes
constexpr int kSteps = kMeanCols / 32;         // of a product: 18

// A tile's keys in LDS: nine pieces of 128 bytes a row, [piece][row][128], 16-byte
// chunk c of a piece in place c ^ key_swizzle(row).  The LDS serves 16 lanes of a
// 16-byte read at once, rows {0..3, 8..11} (or the others) of two neighbouring chunks;
// rows lie 0 or 128 bytes apart modulo the 64 banks, by their lowest bit, and the key
// puts their other two bits beside the chunk's.
__device__ __forceinline__ int key_swizzle(int n) { return ((n >> 1) & 1) << 1 | ((n >> 3) & 1) << 2; }

// 16 bytes a lane from src to dst + 16 * lane, dst the same in every lane.  The wait for
// it is the code's own: written as asm, since the compiler would wait before every LDS
// read that follows.
__device__ __forceinline__ void to_lds(const uint8_t* src, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :: "v"(src), "s"(__builtin_amdgcn_readfirstlane(dst)) : "memory", "m0");
}
constexpr int kWaitLoads = (7 << 4) | (15 << 8);  // s_waitcnt vmcnt(0)

__device__ __forceinline__ float over_rows(float v) {  // of lanes l, l ^ 16, l ^ 32, l ^ 48
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// Statistics (largest logit, sum of exponentials against it) of two sets, joined.
__device__ __forceinline__ f32x2_t join(f32x2_t a, f32x2_t b) {
  const float m = fmaxf(a[0], b[0]), top = fmaxf(m, -3.4e38f);
  return f32x2_t{m, a[1] * __builtin_amdgcn_exp2f(a[0] - top) + b[1] * __builtin_amdgcn_exp2f(b[0] - top)};
}
// What a logit is taken off by so that the exponentials of all are weights.
__device__ __forceinline__ float norm_of(f32x2_t a) { return fmaxf(a[0], -3.4e38f) + __builtin_amdgcn_logf(a[1]); }

// WR waves along the rows, 4 / WR along the columns, NC chunks and COLS columns of 16
// blocks a wave.  PASS 0: both passes; 1: the statistics of a split; 2: the scores,
// given those of all splits.
template <int WR, int NC, int COLS, int PASS>
__global__ __launch_bounds__(kThreads, 2) void scores_kernel(const ScoresParams p) {
  constexpr int WK = 4 / WR;
  constexpr int kTile = WK * COLS * 16;        // blocks of a tile
  constexpr int kSlots = WR * NC;              // chunks of the workgroup
  constexpr int kRows = kTile / 32;            // keys a lane loads its part of
  constexpr int kPieces = kKeyBytes / 128, kPiece = kTile * 128, kBuffer = kTile * kKeyBytes;
  __shared__ __attribute__((aligned(16))) uint8_t keys[2 * kBuffer];
  __shared__ float part[kSlots][kTile];
  __shared__ f32x2_t stat[WK][kSlots][16];
  __shared__ int32_t is_block[2][kTile];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n16 = lane & 15, g = lane >> 4;
  const int wr = wave / WK, wk = wave % WK;

  // work item: request, group of query rows, split
  const int a = div_by((int)blockIdx.x, p.by_splits);
  const int split = (int)blockIdx.x - a * p.n_splits;
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

  // the keys on their way: wave w loads rows 8 w .. 8 w + 7 (and 32 on), 8 lanes a row
  const int32_t* const table = p.table + b * p.table_s0;
  const int kr = tid >> 3;
  const uint32_t chunk = (uint32_t)(((tid & 7) ^ key_swizzle(kr & 15)) << 4);
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)keys;
  int32_t id[kRows];  // of the tile that is loaded next
  auto ids_of = [&](int t) {
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const int j = t * kTile + kr + 32 * r;
      id[r] = j >= lo && j < end ? table[j] : -1;
    }
  };
  auto load_keys = [&](int buffer) {
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const bool is = id[r] >= 0 && id[r] < p.P;
      const uint8_t* const key = p.means + (int64_t)(is ? id[r] : 0) * kKeyBytes + chunk;
#pragma unroll
      for (int x = 0; x < kPieces; ++x)
        to_lds(key + 128 * x, lds + (uint32_t)(buffer * kBuffer + x * kPiece + (8 * wave + 32 * r) * 128));
      if ((tid & 7) == 0) is_block[buffer][kr + 32 * r] = is;
    }
  };
  constexpr int kFirst = PASS == 2 ? 2 : 1, kLast = PASS == 1 ? 1 : 2;

  // head chunks of the query rows: chunk c of the group is heads 16 (c mod C) .. of
  // row i0 + c / C; more than kSlots of them (one query row of many heads) go in
  // rounds
  const int C = p.row_chunks;
  const int n_chunks = n_i * C;
  const int rounds = (n_chunks + kSlots - 1) / kSlots;
  for (int round = 0; round < rounds; ++round) {
    // tiles t0 .. t1 - 1, in each pass; the one after t (in the second pass the first
    // again)
    auto after = [&](int t) { return t + 1 < t1 ? t + 1 : t0; };
    int buffer = 0;
    if (t0 < t1) {
      ids_of(t0);
      load_keys(buffer);
      ids_of(after(t0));
    }
    bf16x8_t q[NC][kSteps];
    int h0[NC], chunk_end[NC];
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = round * kSlots + wr * NC + k;
      const bool is = c < n_chunks;
      const int ci = is ? div_by(c, p.by_chunks) : 0, i = i0 + ci;
      h0[k] = is ? 16 * (c - ci * C) : p.H;
      chunk_end[k] = is ? end_of(i) : 0;
      const int h = h0[k] + n16;
      if (h < p.H) {
        const uint16_t* const ql = p.q_lat + b * p.ql_s0 + (int64_t)i * p.ql_s1 + h * p.ql_s2 + 8 * g;
        const uint16_t* const qp = p.q_pe + b * p.qp_s0 + (int64_t)i * p.qp_s1 + h * p.qp_s2 + 8 * g;
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
          q[k][s] = s < kDLat / 32 ? *(const bf16x8_t*)(ql + 32 * s) : *(const bf16x8_t*)(qp + 32 * (s - kDLat / 32));
      } else {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) q[k][s] = bf16x8_t{};
      }
    }
    // of rows 16 chunk + 4 g + r: the largest logit and sum of this lane's columns
    // (log2 units), in the second pass what norm_of gives of all
    f32x2_t st[NC][4];
#pragma unroll
    for (int k = 0; k < NC; ++k)
#pragma unroll
      for (int r = 0; r < 4; ++r) st[k][r] = f32x2_t{-INFINITY, 0.f};
    if constexpr (PASS == 2) {
#pragma unroll
      for (int k = 0; k < NC; ++k) {
        const int c = round * kSlots + wr * NC + k;
        if (c >= n_chunks) continue;
        const f32x2_t* const at = (const f32x2_t*)p.stats + (((int64_t)a * p.group_chunks + c) * 16 + 4 * g) * p.n_splits;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          // (lane n16 takes splits n16, n16 + 16, ...)
          f32x2_t x{-INFINITY, 0.f};
          for (int s = n16; s < p.n_splits; s += 16) x = join(x, at[r * p.n_splits + s]);
#pragma unroll
          for (int o = 1; o < 16; o <<= 1) x = join(x, f32x2_t{__shfl_xor(x[0], o), __shfl_xor(x[1], o)});
          st[k][r][0] = norm_of(x);
        }
      }
    }

    for (int pass = kFirst; pass <= kLast; ++pass) {
      for (int t = t0; t < t1; ++t) {
        // the tile has landed, and every wave is past the one before it
        __builtin_amdgcn_s_waitcnt(kWaitLoads);
        __syncthreads();
        const uint8_t* const here = keys + buffer * kBuffer;
        const int32_t* const blocks = is_block[buffer];
        buffer ^= 1;
        if (t + 1 < t1 || pass < kLast) {
          load_keys(buffer);
          ids_of(after(after(t)));
        }
        f32x4_t acc[NC][COLS];
#pragma unroll
        for (int k = 0; k < NC; ++k)
#pragma unroll
          for (int c = 0; c < COLS; ++c) acc[k][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
#pragma unroll
          for (int c = 0; c < COLS; ++c) {
            const int n = 16 * (wk * COLS + c) + n16;
            const bf16x8_t kf = *(const bf16x8_t*)(here + (s >> 1) * kPiece + n * 128 +
                                                   (((4 * (s & 1) + g) ^ key_swizzle(n16)) << 4));
#pragma unroll
            for (int k = 0; k < NC; ++k)
              acc[k][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[k][s], kf, acc[k][c], 0, 0, 0);
          }
        }
        bool block[COLS];
        int col[COLS];
#pragma unroll
        for (int c = 0; c < COLS; ++c) {
          const int n = 16 * (wk * COLS + c) + n16;
          block[c] = blocks[n] != 0;
          col[c] = t * kTile + n;
        }
        if (pass == 1) {
#pragma unroll
          for (int k = 0; k < NC; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              float x[COLS], mx = st[k][r][0];
#pragma unroll
              for (int c = 0; c < COLS; ++c) {
                x[c] = block[c] && col[c] < chunk_end[k] ? acc[k][c][r] * p.scale_log2 : -INFINITY;
                mx = fmaxf(mx, x[c]);
              }
              const float top = fmaxf(mx, -3.4e38f);
              float sum = st[k][r][1] * __builtin_amdgcn_exp2f(st[k][r][0] - top);
#pragma unroll
              for (int c = 0; c < COLS; ++c) sum += __builtin_amdgcn_exp2f(x[c] - top);
              st[k][r] = f32x2_t{mx, sum};
            }
        } else {
#pragma unroll
          for (int k = 0; k < NC; ++k)
#pragma unroll
            for (int c = 0; c < COLS; ++c) {
              float sum = 0.f;
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float e = __builtin_amdgcn_exp2f(acc[k][c][r] * p.scale_log2 - st[k][r][0]);
                sum += h0[k] + 4 * g + r < p.H ? e : 0.f;
              }
              sum = over_rows(sum);
              if (g == 0)
                part[wr * NC + k][16 * (wk * COLS + c) + n16] = block[c] && col[c] < chunk_end[k] ? sum : -INFINITY;
            }
          __syncthreads();
          // a query row's chunks, in order; more than one round's are added up in
          // place (by the same thread)
          const int c0 = round * kSlots, c1 = min(n_chunks, c0 + kSlots);
          for (int e = tid; e < n_i * kTile; e += kThreads) {
            const int ii = e / kTile, n = e % kTile, j = t * kTile + n;
            const int from = max(ii * C, c0), to = min((ii + 1) * C, c1);
            if (from >= to || j >= p.NB) continue;
            float* const at = out + (int64_t)(i0 + ii) * p.out_s1 + j;
            float sum = from > ii * C ? *at : 0.f;
            for (int c = from; c < to; ++c) sum += part[c - c0][n];
            *at = sum;
          }
        }
      }
      if (pass == 1) {
        // a row's statistics: of the lanes that share it, then of the waves
#pragma unroll
        for (int k = 0; k < NC; ++k)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            f32x2_t x = st[k][r];
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) x = join(x, f32x2_t{__shfl_xor(x[0], o), __shfl_xor(x[1], o)});
            if (n16 == 0) stat[wk][wr * NC + k][4 * g + r] = x;
          }
        __syncthreads();
        if constexpr (PASS == 1) {
          for (int e = tid; e < kSlots * 16; e += kThreads) {
            const int c = round * kSlots + e / 16, r = e % 16;
            if (c >= n_chunks) continue;
            f32x2_t x = stat[0][e / 16][r];
#pragma unroll
            for (int w = 1; w < WK; ++w) x = join(x, stat[w][e / 16][r]);
            ((f32x2_t*)p.stats)[(((int64_t)a * p.group_chunks + c) * 16 + r) * p.n_splits + split] = x;
          }
        } else {
#pragma unroll
          for (int k = 0; k < NC; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              f32x2_t x = stat[0][wr * NC + k][4 * g + r];
#pragma unroll
              for (int w = 1; w < WK; ++w) x = join(x, stat[w][wr * NC + k][4 * g + r]);
              st[k][r][0] = norm_of(x);
            }
        }
      }
    }
    __syncthreads();
  }
}

// ---- the K best of each row.
//
// Values are ordered as 32-bit keys that grow with them (NaN above all, -0 as 0).  A
// workgroup holds a row's keys in registers and narrows down the range in which the
// K-th largest lies: a histogram of the keys in the range over 256 bins (an eighth of
// the range's bits at a time, so that the bins follow the values there are), then the
// bin that holds it.  All keys above the range are then taken, and those in it where
// it comes down to one key, the first ones in the order of their places.  -inf is
// never taken.
//
// Read once, written once; few rows are bound by the launch and by the dependent
// steps of the search.

__device__ __forceinline__ uint32_t order_key(float v) {
  if (v != v) return 0xFFFFFFFFu;
  const uint32_t u = v == 0.f ? 0u : __float_as_uint(v);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr uint32_t kLowestKey = 0x007FFFFFu;  // of -inf
constexpr int kBins = 256;

// Of a histogram of `bins`, the bin that holds the `want`-th key from the top, and how
// many of the wanted lie in it (by the first wave; want <= the number of keys).
__device__ __forceinline__ void find_bin(const uint32_t* hist, uint32_t want, int lane, int* bin, uint32_t* left,
                                         uint32_t* in_bin) {
  // lane l holds bins 255 - 4 l .. 252 - 4 l, from the top
  uint32_t c[4], sum = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    c[j] = hist[kBins - 1 - 4 * lane - j];
    sum += c[j];
  }
  uint32_t up = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t v = __shfl_up(up, o);
    if (lane >= o) up += v;
  }
  uint32_t past = up - sum;  // in the bins above the lane's
  const uint64_t few = __ballot(past < want);
  if (lane == 63 - __builtin_clzll(few)) {  // the last lane with fewer than `want` above it
    int j = 0;
    while (j < 3 && past + c[j] < want) past += c[j++];
    *bin = kBins - 1 - 4 * lane - j;
    *left = want - past;
    *in_bin = c[j];
  }
}

// A row by THREADS threads, E values each: value e of thread t is place e THREADS + t.
template <int THREADS, int E>
__global__ __launch_bounds__(THREADS) void topk_kernel(const TopkParams p) {
  constexpr int kWaves = THREADS / 64;
  __shared__ uint32_t hist[2][kBins];
  __shared__ uint32_t wave_lo[kWaves], wave_hi[kWaves];
  __shared__ int wave_n[kWaves];
  // of 64 neighbours: (above, equal << 16), then the places taken before them; equal ones before them
  __shared__ int counts[E * kWaves], eq_before[E * kWaves];
  __shared__ int n_taken;
  __shared__ int found;
  __shared__ uint32_t left, in_bin;
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t b = div_by((int)row, p.by_Mq), i = row - b * p.Mq;
  const float* const x = p.x + b * p.x_s0 + i * p.x_s1;
  int32_t* const ids = p.ids + b * p.ids_s0 + i * p.ids_s1;
  uint32_t key[E];  // (0: no place)
  {
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = e * THREADS + tid < p.N ? x[e * THREADS + tid] : -INFINITY;
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
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    lo = min(lo, (uint32_t)__shfl_xor((int)lo, o));
    hi = max(hi, (uint32_t)__shfl_xor((int)hi, o));
    n += __shfl_xor(n, o);
  }
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
    const int bits = 32 - __builtin_clz(hi - lo), shift = max(bits - 8, 0);
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (key[e] >= lo && key[e] <= hi) atomicAdd(&hist[turn][(key[e] - lo) >> shift], 1u);
    __syncthreads();
    if (wave == 0) find_bin(hist[turn], want, lane, &found, &left, &in_bin);
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
    int a = above, q = equal;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int va = __shfl_up(a, o), vq = __shfl_up(q, o);
      if (lane >= o) {
        a += va;
        q += vq;
      }
    }
    a -= above;
    q -= equal;
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
    if (take)
      ids[base + (int)__popcll(gt & before) + min(mine, (int)want) - min(q0, (int)want)] = e * THREADS + tid;
  }
  for (int k = n_taken + tid; k < p.K; k += THREADS) ids[k] = -1;
}

// A row of any length by one workgroup, read from memory in each round: eight bits
// of the K-th largest key a round, by a histogram of the values that share the bits
// found before.
constexpr int kTopThreads = 1024;
__global__ __launch_bounds__(kTopThreads) void topk_row_kernel(const TopkParams p) {
  __shared__ uint32_t hist[kBins];
  __shared__ int wave_above[kTopThreads / 64], wave_equal[kTopThreads / 64];
  __shared__ int found;
  __shared__ uint32_t left, in_bin;
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t b = div_by((int)row, p.by_Mq), i = row - b * p.Mq;
  const float* const x = p.x + b * p.x_s0 + i * p.x_s1;
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
    if (wave == 0) find_bin(hist, (uint32_t)want, lane, &found, &left, &in_bin);
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
    if (take) ids[at + a0 + (int)__popcll(gt & before) + min(eq_before, want)] = e;
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
  if (p.n_splits == 1) {
    hipLaunchKernelGGL((scores_kernel<WR, NC, COLS, 0>), dim3(grid), dim3(kThreads), 0, s, p);
    return;
  }
  hipLaunchKernelGGL((scores_kernel<WR, NC, COLS, 1>), dim3(grid), dim3(kThreads), 0, s, p);
  hipLaunchKernelGGL((scores_kernel<WR, NC, COLS, 2>), dim3(grid), dim3(kThreads), 0, s, p);
}

hipError_t launch_scores(const ScoresParams& p, int B, hipStream_t s) {
  const int grid = B * p.n_groups * p.n_splits;
  if (grid <= 0) return hipSuccess;
  if (p.shape == kScores128) launch_scores_rows<4, 2, 2>(p, grid, s);
  else if (p.shape == kScores64) launch_scores_rows<2, 2, 2>(p, grid, s);
  else if (p.shape == kScores32) launch_scores_rows<1, 2, 1>(p, grid, s);
  else launch_scores_rows<1, 1, 1>(p, grid, s);
  return hipGetLastError();
}

hipError_t launch_topk(const TopkParams& p, hipStream_t s) {
  if (p.rows <= 0) return hipSuccess;
  const dim3 g((uint32_t)p.rows);
  if (p.N <= 256) hipLaunchKernelGGL((topk_kernel<64, 4>), g, dim3(64), 0, s, p);
  else if (p.N <= 1024) hipLaunchKernelGGL((topk_kernel<256, 4>), g, dim3(256), 0, s, p);
  else if (p.N <= 4096) hipLaunchKernelGGL((topk_kernel<512, 8>), g, dim3(512), 0, s, p);
  else if (p.N <= 16384) hipLaunchKernelGGL((topk_kernel<1024, 16>), g, dim3(1024), 0, s, p);
  else if (p.N <= 65536) hipLaunchKernelGGL((topk_kernel<1024, 64>), g, dim3(1024), 0, s, p);
  else hipLaunchKernelGGL(topk_row_kernel, g, dim3(kTopThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace mla
