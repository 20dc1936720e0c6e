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
// A workgroup takes every n-th of the slots and, of those that are a block's last
// row, that block, all of whose 18 loads a thread are out before the first sum: a
// stream through HBM, bound by the launch and two trips where few blocks are whole.
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
  __shared__ int32_t whole[kThreads];
  __shared__ int n_whole;
  const int tid = threadIdx.x;
  const int64_t step = gridDim.x;
  for (int64_t k0 = 0; blockIdx.x + k0 * step < p.T; k0 += kThreads) {
    const int64_t t = blockIdx.x + (k0 + tid) * step;
    const int32_t s = t < p.T ? p.slots[t] : -1;
    if (tid == 0) n_whole = 0;
    __syncthreads();
    // (their order does not matter)
    if (s >= 0 && s < p.n_slots && s % kBlock == kBlock - 1) whole[atomicAdd(&n_whole, 1)] = s / kBlock;
    __syncthreads();
    const int n = n_whole;
    for (int k = 0; k < n; ++k) {
      const int64_t b = whole[k];
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
// A workgroup takes 64 blocks at a time into LDS; its waves share out 16-row chunks
// (the heads of one query row, padded) and the blocks' four columns of 16.  bf16
// MFMA 16x16x32 with the query rows in registers for the whole kernel.
constexpr int kTileCols = 64;                  // blocks of a tile
constexpr int kKeyBytes = 2 * kMeanCols;       // 1152: 72 chunks of 16 bytes
constexpr int kSteps = kMeanCols / 32;         // of a product: 18
constexpr int kChunks = kScoreChunks;          // 16-row chunks a wave holds

// 16-byte chunk c of a key in LDS row n sits in place c ^ key_swizzle(n): the LDS
// serves 16 lanes of a 16-byte read at once, rows {0..3, 8..11} (or the others) of
// two neighbouring chunks; rows of 1152 bytes lie 0 or 128 bytes apart modulo the 64
// banks, by their lowest bit, and the key puts their other two bits beside the
// chunk's.
__device__ __forceinline__ int key_swizzle(int n) { return ((n >> 1) & 1) << 1 | ((n >> 3) & 1) << 2; }

__device__ __forceinline__ float over_rows(float v) {  // of lanes l, l ^ 16, l ^ 32, l ^ 48
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// WR waves along the rows, 4 / WR along the columns.  PASS 0: both passes; 1: the
// statistics of a split; 2: the scores, given those of all splits.
template <int WR, int PASS>
__global__ __launch_bounds__(kThreads) void scores_kernel(const ScoresParams p) {
  constexpr int WK = 4 / WR, kCols = 4 / WK;  // 16-block columns of a wave
  constexpr int kSlots = WR * kChunks;        // chunks of the workgroup
  __shared__ __attribute__((aligned(16))) uint8_t keys[kTileCols * kKeyBytes];
  __shared__ float part[kSlots][kTileCols];
  __shared__ f32x2_t stat[WK][kSlots][16];
  __shared__ uint64_t live_cols;
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
  const int tile0 = lo / kTileCols, tiles = end > lo ? (end - 1) / kTileCols - tile0 + 1 : 0;
  const int t0 = tile0 + (int)((int64_t)tiles * split / p.n_splits);
  const int t1 = tile0 + (int)((int64_t)tiles * (split + 1) / p.n_splits);

  float* const out = p.out + (int64_t)b * p.out_s0;
  if constexpr (PASS != 1) {
    // columns of no tile
    if (split == p.n_splits - 1) {
      const int c0 = tiles > 0 ? tile0 * kTileCols : 0, c1 = tiles > 0 ? (tile0 + tiles) * kTileCols : 0;
      for (int i = i0; i < i0 + n_i; ++i) {
        float* const row = out + (int64_t)i * p.out_s1;
        for (int c = tid; c < p.NB; c += kThreads)
          if (c < c0 || c >= c1) row[c] = -INFINITY;
      }
    }
  }
  if (t0 == t1 && PASS != 1) return;

  // head chunks of the query rows: chunk c of the group is heads 16 (c mod C) .. of
  // row i0 + c / C; more than kSlots of them (one query row of many heads) go in
  // rounds
  const int C = p.row_chunks;
  const int n_chunks = n_i * C;
  const int rounds = (n_chunks + kSlots - 1) / kSlots;
  for (int round = 0; round < rounds; ++round) {
    bf16x8_t q[kChunks][kSteps];
    int row_i[kChunks], h0[kChunks];
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
      const int c = round * kSlots + wr * kChunks + k;
      const bool is = c < n_chunks;
      const int ci = is ? div_by(c, p.by_chunks) : 0;
      row_i[k] = is ? i0 + ci : -1;
      h0[k] = is ? 16 * (c - ci * C) : p.H;
      const int h = h0[k] + n16;
      if (h < p.H) {
        const uint16_t* const ql = p.q_lat + b * p.ql_s0 + (int64_t)row_i[k] * p.ql_s1 + h * p.ql_s2 + 8 * g;
        const uint16_t* const qp = p.q_pe + b * p.qp_s0 + (int64_t)row_i[k] * p.qp_s1 + h * p.qp_s2 + 8 * g;
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
          q[k][s] = s < kDLat / 32 ? *(const bf16x8_t*)(ql + 32 * s) : *(const bf16x8_t*)(qp + 32 * (s - kDLat / 32));
      } else {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) q[k][s] = bf16x8_t{};
      }
    }
    // of rows 16 chunk + 4 g + r: the largest logit and sum of this lane's columns,
    // then the row's log2 of the sum of all
    float m[kChunks][4], l[kChunks][4];
#pragma unroll
    for (int k = 0; k < kChunks; ++k)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        m[k][r] = -INFINITY;
        l[k][r] = 0.f;
      }

    for (int pass = PASS == 2 ? 2 : 1; pass <= (PASS == 1 ? 1 : 2); ++pass) {
      if (pass == 2) {
        // the rows' statistics: those of all splits, or of this workgroup's waves
        if constexpr (PASS == 0) {
#pragma unroll
          for (int k = 0; k < kChunks; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              float mm = -INFINITY, ll = 0.f;
#pragma unroll
              for (int w = 0; w < WK; ++w) mm = fmaxf(mm, stat[w][wr * kChunks + k][4 * g + r][0]);
              const float top = fmaxf(mm, -3.4e38f);
#pragma unroll
              for (int w = 0; w < WK; ++w) {
                const f32x2_t st = stat[w][wr * kChunks + k][4 * g + r];
                ll += st[1] * __builtin_amdgcn_exp2f(st[0] - top);
              }
              m[k][r] = top + __builtin_amdgcn_logf(ll);
            }
        } else {
#pragma unroll
          for (int k = 0; k < kChunks; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              // (lane n16 takes splits n16, n16 + 16, ...)
              float mm = -INFINITY, ll = 0.f;
              const int c = round * kSlots + wr * kChunks + k;
              const f32x2_t* const st = (const f32x2_t*)p.stats +
                                        (((int64_t)a * p.group_chunks + c) * 16 + 4 * g + r) * p.n_splits;
              if (c < n_chunks) {
                for (int s = n16; s < p.n_splits; s += 16) mm = fmaxf(mm, st[s][0]);
#pragma unroll
                for (int o = 1; o < 16; o <<= 1) mm = fmaxf(mm, __shfl_xor(mm, o));
                const float top = fmaxf(mm, -3.4e38f);
                for (int s = n16; s < p.n_splits; s += 16) ll += st[s][1] * __builtin_amdgcn_exp2f(st[s][0] - top);
#pragma unroll
                for (int o = 1; o < 16; o <<= 1) ll += __shfl_xor(ll, o);
                m[k][r] = top + __builtin_amdgcn_logf(ll);
              }
            }
        }
      }
      for (int t = t0; t < t1; ++t) {
        __syncthreads();  // the last tile's keys and parts are read
        // keys of blocks 64 t .. +63 and which of them there are
        if (tid < kTileCols) {
          const int j = t * kTileCols + tid;
          int32_t blk = -1;
          if (j >= lo && j < end) {
            blk = p.table[b * p.table_s0 + j];
            if (blk >= p.P) blk = -1;
          }
          const uint64_t is = __ballot(blk >= 0);
          if (tid == 0) live_cols = is;
          ((int32_t*)part)[tid] = max(blk, 0);
        }
        __syncthreads();
        u32x4_t v[kTileCols * kKeyBytes / 16 / kThreads];
#pragma unroll
        for (int x = 0; x < kTileCols * kKeyBytes / 16 / kThreads; ++x) {
          const int e = x * kThreads + tid, n = e / (kKeyBytes / 16), c = e - n * (kKeyBytes / 16);
          v[x] = *(const u32x4_t*)(p.means + (int64_t)((const int32_t*)part)[n] * kKeyBytes + 16 * c);
        }
#pragma unroll
        for (int x = 0; x < kTileCols * kKeyBytes / 16 / kThreads; ++x) {
          const int e = x * kThreads + tid, n = e / (kKeyBytes / 16), c = e - n * (kKeyBytes / 16);
          *(u32x4_t*)(keys + n * kKeyBytes + ((c ^ key_swizzle(n & 15)) << 4)) = v[x];
        }
        __syncthreads();
        const uint64_t cols = live_cols;
        f32x4_t acc[kChunks][kCols];
#pragma unroll
        for (int k = 0; k < kChunks; ++k)
#pragma unroll
          for (int c = 0; c < kCols; ++c) acc[k][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
#pragma unroll
          for (int c = 0; c < kCols; ++c) {
            const int n = 16 * (wk * kCols + c) + n16;
            const bf16x8_t kf = *(const bf16x8_t*)(keys + n * kKeyBytes + (((4 * s + g) ^ key_swizzle(n16)) << 4));
#pragma unroll
            for (int k = 0; k < kChunks; ++k)
              acc[k][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[k][s], kf, acc[k][c], 0, 0, 0);
          }
        }
        float w[kChunks][kCols];
#pragma unroll
        for (int k = 0; k < kChunks; ++k) {
          const int ci_end = row_i[k] >= 0 ? end_of(row_i[k]) : 0;
          bool may[kCols];
#pragma unroll
          for (int c = 0; c < kCols; ++c) {
            const int n = 16 * (wk * kCols + c) + n16;
            may[c] = (cols >> n & 1) != 0 && t * kTileCols + n < ci_end;
          }
          if (pass == 1) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              float x[kCols], mx = m[k][r];
#pragma unroll
              for (int c = 0; c < kCols; ++c) {
                x[c] = may[c] ? acc[k][c][r] * p.scale_log2 : -INFINITY;
                mx = fmaxf(mx, x[c]);
              }
              const float top = fmaxf(mx, -3.4e38f);
              float sum = l[k][r] * __builtin_amdgcn_exp2f(m[k][r] - top);
#pragma unroll
              for (int c = 0; c < kCols; ++c) sum += __builtin_amdgcn_exp2f(x[c] - top);
              l[k][r] = sum;
              m[k][r] = mx;
            }
          } else {
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
              float sum = 0.f;
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float e = __builtin_amdgcn_exp2f(acc[k][c][r] * p.scale_log2 - m[k][r]);
                sum += h0[k] + 4 * g + r < p.H ? e : 0.f;
              }
              sum = over_rows(sum);
              w[k][c] = may[c] ? sum : -INFINITY;
            }
          }
        }
        if (pass == 2) {
#pragma unroll
          for (int k = 0; k < kChunks; ++k)
#pragma unroll
            for (int c = 0; c < kCols; ++c)
              if (g == 0) part[wr * kChunks + k][16 * (wk * kCols + c) + n16] = w[k][c];
          __syncthreads();
          // a query row's chunks, in order; more than one round's are added up in
          // place (the same thread's)
          const int c0 = round * kSlots, c1 = min(n_chunks, c0 + kSlots);
          for (int e = tid; e < n_i * kTileCols; e += kThreads) {
            const int ii = e / kTileCols, n = e % kTileCols, j = t * kTileCols + n;
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
        // the lanes' statistics of a row to one
#pragma unroll
        for (int k = 0; k < kChunks; ++k)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float mm = m[k][r];
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) mm = fmaxf(mm, __shfl_xor(mm, o));
            const float top = fmaxf(mm, -3.4e38f);
            float ll = l[k][r] * __builtin_amdgcn_exp2f(m[k][r] - top);
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) ll += __shfl_xor(ll, o);
            if (n16 == 0) stat[wk][wr * kChunks + k][4 * g + r] = f32x2_t{mm, ll};
          }
        __syncthreads();
        if constexpr (PASS == 1) {
          for (int e = tid; e < kSlots * 16; e += kThreads) {
            const int c = round * kSlots + e / 16, r = e % 16;
            if (c >= n_chunks) continue;
            float mm = -INFINITY, ll = 0.f;
#pragma unroll
            for (int w = 0; w < WK; ++w) mm = fmaxf(mm, stat[w][e / 16][r][0]);
            const float top = fmaxf(mm, -3.4e38f);
#pragma unroll
            for (int w = 0; w < WK; ++w) ll += stat[w][e / 16][r][1] * __builtin_amdgcn_exp2f(stat[w][e / 16][r][0] - top);
            ((f32x2_t*)p.stats)[(((int64_t)a * p.group_chunks + c) * 16 + r) * p.n_splits + split] = f32x2_t{mm, ll};
          }
          __syncthreads();
        }
      }
    }
    __syncthreads();
  }
}

// ---- the K best of each row.
//
// Values are ordered as 32-bit keys that grow with them (NaN above all, -0 as 0);
// the K-th largest key T is found a bit at a time from the top, counting the values
// at or above each candidate; then all values above T are taken, and of those equal
// to it the first ones, in the order of their places.  -inf is never taken.

__device__ __forceinline__ uint32_t order_key(float v) {
  if (v != v) return 0xFFFFFFFFu;
  const uint32_t u = v == 0.f ? 0u : __float_as_uint(v);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr uint32_t kLowestKey = 0x007FFFFFu;  // of -inf

// A row by one wave, E values a lane: value e of lane l is place 64 e + l.
template <int E>
__global__ __launch_bounds__(kThreads) void topk_wave_kernel(const TopkParams p) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= p.rows) return;
  const int lane = threadIdx.x & 63;
  const int64_t b = div_by((int)row, p.by_Mq), i = row - b * p.Mq;
  const float* const x = p.x + b * p.x_s0 + i * p.x_s1;
  int32_t* const ids = p.ids + b * p.ids_s0 + i * p.ids_s1;
  uint32_t key[E];
  int n = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    key[e] = 64 * e + lane < p.N ? order_key(x[64 * e + lane]) : 0u;
    n += __popcll(__ballot(key[e] > kLowestKey));
  }
  // the K-th largest key, if there are more than K above -inf
  uint32_t top = kLowestKey + 1;
  if (n > p.K) {
    top = 0;
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t at = top | 1u << bit;
      int c = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) c += __popcll(__ballot(key[e] >= at));
      if (c >= p.K) top = at;
      if (c == p.K) break;
    }
  }
  int above = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) above += __popcll(__ballot(key[e] > top));
  int ties = p.K - above;  // of those equal to it, so many
  int at = 0;
  const uint64_t before = (1ull << lane) - 1;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const uint64_t eq = __ballot(key[e] == top);
    const bool take = key[e] > top || (key[e] == top && (int)__popcll(eq & before) < ties);
    const uint64_t m = __ballot(take);
    if (take) ids[at + __popcll(m & before)] = 64 * e + lane;
    at += __popcll(m);
    ties -= (int)__popcll(eq);  // (below 0 once they are taken)
  }
  for (int k = at + lane; k < p.K; k += 64) ids[k] = -1;
}

// A row of any length by one workgroup, read from memory in each round: eight bits
// of the K-th largest key a round, by a histogram of the values that share the bits
// found before.
constexpr int kTopThreads = 1024;
__global__ __launch_bounds__(kTopThreads) void topk_row_kernel(const TopkParams p) {
  __shared__ uint32_t hist[256];
  __shared__ int wave_above[kTopThreads / 64], wave_equal[kTopThreads / 64];
  __shared__ uint32_t found;
  __shared__ int left;
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t b = div_by((int)row, p.by_Mq), i = row - b * p.Mq;
  const float* const x = p.x + b * p.x_s0 + i * p.x_s1;
  int32_t* const ids = p.ids + b * p.ids_s0 + i * p.ids_s1;
  uint32_t top = 0;
  int want = p.K;  // of the values that share top's bits so far, so many are taken
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int e = tid; e < p.N; e += kTopThreads) {
      const uint32_t k = order_key(x[e]);
      if (shift == 24 || k >> (shift + 8) == top >> (shift + 8)) atomicAdd(&hist[k >> shift & 255], 1u);
    }
    __syncthreads();
    if (tid < 64) {
      // lane l holds bins 255 - 4 l .. 252 - 4 l, from the top
      uint32_t c[4], sum = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        c[j] = hist[255 - 4 * lane - j];
        sum += c[j];
      }
      uint32_t up = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t v = __shfl_up(up, o);
        if (lane >= o) up += v;
      }
      uint32_t past = up - sum;  // in the bins above the lane's
      // (the last lane that has fewer than `want` above it holds the bin, or the
      // lowest bin does where the row has fewer values)
      const uint64_t few = __ballot(past < (uint32_t)want);
      if (lane == 63 - __builtin_clzll(few)) {
        int j = 0;
        while (j < 3 && past + c[j] < (uint32_t)want) past += c[j++];
        found = top | (uint32_t)(255 - 4 * lane - j) << shift;
        left = want - (int)past;
      }
    }
    __syncthreads();
    top = found;
    want = left;
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
      wave_above[wave] = __popcll(gt);
      wave_equal[wave] = __popcll(eq);
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
    const int eq_before = q0 + __popcll(eq & before);
    const bool take = k > top || (k == top && eq_before < want);
    if (take) ids[at + a0 + __popcll(gt & before) + min(eq_before, want)] = e;
    at += an + min(qn, want);
    want -= min(qn, want);
    __syncthreads();
  }
  for (int k = at + tid; k < p.K; k += kTopThreads) ids[k] = -1;
}

}  // namespace

hipError_t launch_means(const MeansParams& p, int kv, hipStream_t s) {
  if (p.T <= 0) return hipSuccess;
  // An odd number of workgroups: of the tokens that follow each other in a request
  // every 64th completes a block, which would all be one workgroup's.
  const int grid = (int)(p.T < 2047 ? p.T : 2047);
  if (kv == kKvMx4) hipLaunchKernelGGL(means_kernel<kKvMx4>, dim3(grid), dim3(kThreads), 0, s, p);
  else if (kv == kKvBf16) hipLaunchKernelGGL(means_kernel<kKvBf16>, dim3(grid), dim3(kThreads), 0, s, p);
  else hipLaunchKernelGGL(means_kernel<kKvFp8Shared>, dim3(grid), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

template <int WR>
static void launch_scores_rows(const ScoresParams& p, int grid, hipStream_t s) {
  if (p.n_splits == 1) {
    hipLaunchKernelGGL((scores_kernel<WR, 0>), dim3(grid), dim3(kThreads), 0, s, p);
    return;
  }
  hipLaunchKernelGGL((scores_kernel<WR, 1>), dim3(grid), dim3(kThreads), 0, s, p);
  hipLaunchKernelGGL((scores_kernel<WR, 2>), dim3(grid), dim3(kThreads), 0, s, p);
}

hipError_t launch_scores(const ScoresParams& p, int B, hipStream_t s) {
  const int grid = B * p.n_groups * p.n_splits;
  if (grid <= 0) return hipSuccess;
  if (p.wave_rows == 4) launch_scores_rows<4>(p, grid, s);
  else if (p.wave_rows == 2) launch_scores_rows<2>(p, grid, s);
  else launch_scores_rows<1>(p, grid, s);
  return hipGetLastError();
}

hipError_t launch_topk(const TopkParams& p, hipStream_t s) {
  if (p.rows <= 0) return hipSuccess;
  const dim3 waves((uint32_t)((p.rows + 3) / 4));
  if (p.N <= 256) hipLaunchKernelGGL(topk_wave_kernel<4>, waves, dim3(kThreads), 0, s, p);
  else if (p.N <= 1024) hipLaunchKernelGGL(topk_wave_kernel<16>, waves, dim3(kThreads), 0, s, p);
  else hipLaunchKernelGGL(topk_row_kernel, dim3((uint32_t)p.rows), dim3(kTopThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace mla
