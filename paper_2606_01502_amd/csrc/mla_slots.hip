// The block tables and slot maps of a batch, from its lengths: what a step needs
// before it can write its new tokens into the paged cache.
//
// With c cached and n new tokens, a request holds ceil(c / 64) blocks and takes
// the next ones off the free list until it holds ceil((c + n) / 64); new token i
// goes to position c + i.  Two exclusive sums over the requests (new tokens, new
// blocks) say where each request's part of the packed tokens and of the free list
// begins; everything else is a search in them.
//
// One launch for two: every workgroup forms both sums itself in LDS (a thread takes
// up to 16 neighbouring requests, 8192 in all, and reads their lengths one by one in
// both of its passes over them) and then takes its share of the tokens and of the
// new blocks.  No workgroup reads a table entry that another writes: a token in a
// new block takes the block from the free list.  Bound by the launch and three
// dependent trips: 64 requests of one token take 4.1 us, 300 of 100,003 tokens (1.2
// MB) 7.6 us; by the lengths' loads where there are many, 8000 of one token 25 us.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mla_kernels.h"

namespace mla {
namespace {

constexpr int kSlotThreads = 512;

// the largest b with off[b] <= v, where off[0] = 0 and v < off[n]: the request
// that element v of the packed order belongs to (requests of no elements are
// passed over)
__device__ __forceinline__ int owner(const int32_t* off, int n, int32_t v) {
  int lo = 0, hi = n;  // off[lo] <= v < off[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (off[mid] <= v) lo = mid;
    else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ int32_t sat(int64_t v) { return (int32_t)min(v, (int64_t)INT32_MAX); }

__global__ __launch_bounds__(kSlotThreads) void slots_kernel(const SlotsParams p) {
  // first packed token and first new block of each request, the totals last
  // (saturated: what lies past 2^31 - 1 is past the outputs as well)
  __shared__ int32_t tok[kMaxSlotRequests + 1], blk[kMaxSlotRequests + 1];
  __shared__ int64_t wave_tok[kSlotThreads / 64], wave_blk[kSlotThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto len = [](int32_t v) { return (int64_t)max(v, 0); };
  auto held = [&](int b) { return (int)min((len(p.cached[b]) + kBlock - 1) / kBlock, (int64_t)p.NB); };
  auto takes = [&](int b) {
    return (int)min((len(p.cached[b]) + len(p.fresh[b]) + kBlock - 1) / kBlock, (int64_t)p.NB) - held(b);
  };
  const int per = (p.B + kSlotThreads - 1) / kSlotThreads;
  const int b0 = min(tid * per, p.B), b1 = min(b0 + per, p.B);
  int64_t st = 0, sb = 0;
  for (int b = b0; b < b1; ++b) {
    st += len(p.fresh[b]);
    sb += takes(b);
  }
  int64_t it = st, ib = sb;  // inclusive over the threads
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t a = __shfl_up(it, o), c = __shfl_up(ib, o);
    if (lane >= o) {
      it += a;
      ib += c;
    }
  }
  if (lane == 63) {
    wave_tok[wave] = it;
    wave_blk[wave] = ib;
  }
  __syncthreads();
  int64_t et = it - st, eb = ib - sb, total_t = 0, total_b = 0;
#pragma unroll
  for (int w = 0; w < kSlotThreads / 64; ++w) {
    if (w < wave) {
      et += wave_tok[w];
      eb += wave_blk[w];
    }
    total_t += wave_tok[w];
    total_b += wave_blk[w];
  }
  for (int b = b0; b < b1; ++b) {
    tok[b] = sat(et);
    blk[b] = sat(eb);
    et += len(p.fresh[b]);
    eb += takes(b);
  }
  if (tid == 0) {
    tok[p.B] = sat(total_t);
    blk[p.B] = sat(total_b);
  }
  __syncthreads();
  const int32_t n_tok = tok[p.B], n_blk = blk[p.B];
  const int64_t step = (int64_t)gridDim.x * kSlotThreads;
  const int64_t first = (int64_t)blockIdx.x * kSlotThreads + tid;
  for (int64_t j = first; j < n_blk; j += step) {
    const int b = owner(blk, p.B, (int32_t)j);
    p.table[b * p.table_s0 + held(b) + ((int32_t)j - blk[b])] = j < p.F ? p.free_blocks[j] : -1;
  }
  for (int64_t t = first; t < p.T; t += step) {
    int32_t slot = -1, pos = -1;
    if (t < n_tok) {
      const int b = owner(tok, p.B, (int32_t)t);
      const int64_t at = len(p.cached[b]) + ((int32_t)t - tok[b]);
      const int64_t col = at / kBlock;
      pos = sat(at);
      if (col < p.NB) {
        int32_t block = -1;
        const int h = held(b);
        if (col < h) {
          block = p.table[b * p.table_s0 + col];
        } else {
          const int64_t j = blk[b] + (col - h);
          if (j < p.F) block = p.free_blocks[j];
        }
        if (block >= 0 && block <= (INT32_MAX >> 6)) slot = block * kBlock + (int32_t)(at % kBlock);
      }
    }
    p.slots[t] = slot;
    p.positions[t] = pos;
  }
  if (blockIdx.x == 0) {
    for (int b = tid; b <= p.B; b += kSlotThreads) {
      p.starts[b] = tok[b];
      if (b < p.B) p.seq_lens[b] = sat(len(p.cached[b]) + len(p.fresh[b]));
    }
    if (tid == 0) {
      p.info[0] = n_tok;
      p.info[1] = (int32_t)min((int64_t)n_blk, p.F);
      p.info[2] = (int32_t)max((int64_t)n_blk - p.F, (int64_t)0);
      p.info[3] = (int32_t)max((int64_t)n_tok - p.T, (int64_t)0);
    }
  }
}

}  // namespace

hipError_t launch_slots(const SlotsParams& p, hipStream_t s) {
  // A workgroup for each 2048 tokens.  Fewer tokens are searched for faster, more
  // workgroups form the sums and share the memory they come from: 300 requests of
  // 100,003 tokens take 7.6 us with 2048, 4.8 with 512 and 11.5 with 4096 tokens a
  // workgroup, 8 of 400,000 4.7, 6.5 and 5.3.
  const int64_t work = p.T > p.B ? p.T : p.B;
  const int64_t grid = (work + 2047) / 2048;
  hipLaunchKernelGGL(slots_kernel, dim3((uint32_t)(grid < 1 ? 1 : grid > 1024 ? 1024 : grid)), dim3(kSlotThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace mla
