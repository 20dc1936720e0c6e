// The latent cache in 4 bits, written and read back, and the write of new tokens
// into a bf16 cache.
//
// A cached token's 512 latent values are 16 groups of 32 neighbours (OCP MX: E2M1
// codes under a shared power of two).  With a the group's largest magnitude, its
// scale is 2^(floor(log2 a) - 2), which puts a between 4 and 8 units (E2M1's
// largest power of two is 4); each code is the nearest E2M1 value, halfway to the
// even code, 6 where a value lies past 6 units.  A row is 272 bytes: 256 of codes,
// the even column in the low half of a byte, then 16 scale exponents plus 127.
// Exponents stay within -125 .. 125, so that every cached value is a normal bf16
// number or 0; a group that holds an infinity or a NaN gets exponent byte 255 and
// reads back as NaN.  The RoPE part stays in bf16: 400 bytes a token for 1152.
//
// Streams through HBM: a wave takes one token, 8 columns a lane (16 bytes read,
// 4 written), so that a group is four lanes.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mla_kernels.h"
#include "mla_mx4.h"

namespace mla {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kRowWords = kMx4Row / 4;
constexpr int kGatherToks = 16;  // tokens a gather workgroup takes

__device__ __forceinline__ int quad_max(int v) {
  v = max(v, __shfl_xor(v, 1));
  return max(v, __shfl_xor(v, 2));
}

// Eight bf16 values (two to a word) -> eight E2M1 codes of v / s, s a power of two:
// to nearest, halfway to the even code, at most 6 (compared for every bf16 value).
// The conversion instruction does two at once: 30,001 tokens are written in 9.2 us
// (46 MB, 5 TB/s), 16.5 with comparisons against the seven borders, which are about
// 130 instructions for these eight values.
__device__ __forceinline__ uint32_t to_codes(u32x4_t v, float s) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  // (a bit cast of a vector's element would take the first one)
  const uint32_t w0 = v[0], w1 = v[1], w2 = v[2], w3 = v[3];
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, w0), s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, w1), s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, w2), s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, w3), s, 3);
}

template <bool MX4>
__global__ __launch_bounds__(kThreads) void append_kernel(const AppendParams p) {
  const int lane = threadIdx.x & 63;
  const int64_t wave = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 6;
  const int64_t t0 = wave * p.wave_toks;
  const int n = (int)min((int64_t)p.wave_toks, p.T - t0);
  constexpr int kAhead = 4;
  for (int k0 = 0; k0 < n; k0 += kAhead) {
    u32x4_t v[kAhead], w[kAhead];
    int64_t row[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int64_t t = t0 + min(k0 + j, n - 1);  // past the end: loaded, not stored
      const int32_t s = p.slots[t];
      row[j] = k0 + j < n && s >= 0 && s < p.n_slots ? s : -1;
      v[j] = *(const u32x4_t*)(p.src_ckv + t * p.ckv_s0 + 8 * lane);
      if (lane < 8) w[j] = *(const u32x4_t*)(p.src_kpe + t * p.kpe_s0 + 8 * lane);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (row[j] < 0) continue;
      if (lane < 8) *(u32x4_t*)(p.kpe + row[j] * (2 * kDPe) + 16 * lane) = w[j];
      if constexpr (!MX4) {
        *(u32x4_t*)(p.ckv + row[j] * (2 * kDLat) + 16 * lane) = v[j];
      } else {
        // magnitudes of bf16 numbers are ordered as their bits
        int mag = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          mag = max(mag, max((int)(v[j][i] & 0x7FFFu), (int)(v[j][i] >> 16 & 0x7FFFu)));
        mag = quad_max(mag);
        // floor(log2 a) + 127 is the exponent field (0 for subnormal numbers, which
        // the lower limit covers)
        const bool bad = mag >= 0x7F80;
        const int byte = min(max((mag >> 7) - 2, 2), 252);
        uint32_t* const dst = (uint32_t*)(p.ckv + row[j] * kMx4Row);
        dst[lane] = to_codes(v[j], __uint_as_float((uint32_t)byte << 23));
        // four groups' bytes to a word: lanes 0, 16, 32, 48 store them
        uint32_t b = (uint32_t)(bad ? 255 : byte) << (lane >> 2 & 3) * 8;
        b |= __shfl_xor(b, 4);
        b |= __shfl_xor(b, 8);
        if ((lane & 15) == 0) dst[kDLat / 8 + (lane >> 4)] = b;
      }
    }
  }
}

// Gather of a selected token set out of a 4-bit pool: out row j of layer l = the
// values of pool token sel[j] in bf16 (exact), a zero row for an empty slot.
// 16 tokens a workgroup: 4096 tokens in 4.2 us, 32,768 in 12.7 (50.7 MB, 4.0 TB/s);
// with 32 of them 4.9 and 15.9, with 8 of them 3.9 and 14.1.  The codes come in by
// ordinary loads: rows end inside cache lines, which their neighbours read too
// (past the caches 13.7 us).
__global__ __launch_bounds__(kThreads) void gather_mx4_kernel(const FetchParams p) {
  constexpr int kTok = kGatherToks;
  const int64_t groups = (p.n + kTok - 1) / kTok;
  const int64_t l = blockIdx.x / groups;
  const int64_t j0 = (blockIdx.x - l * groups) * kTok;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  __shared__ int64_t src_row[kTok];
  if (tid < kTok) {
    int64_t row = -1;
    const int64_t j = j0 + tid;
    if (j < p.n) {
      const int32_t s = p.sel[j];
      if (s >= 0 && s < p.n_ids) {
        const int32_t b = p.table[s / kBlock];
        if (b >= 0 && b < p.P) row = (l * p.P + b) * kBlock + (s % kBlock);
      }
    }
    src_row[tid] = row;
  }
  __syncthreads();
  const uint32_t* const sc = (const uint32_t*)p.src_ckv;
  const u32x4_t* const sk = (const u32x4_t*)p.src_kpe;
  constexpr int kPass = kTok / 4;
  uint32_t c[kPass], e[kPass];
  u32x4_t w{0u, 0u, 0u, 0u};
#pragma unroll
  for (int it = 0; it < kPass; ++it) {
    const int64_t r = src_row[4 * it + wave];
    c[it] = r >= 0 ? sc[r * kRowWords + lane] : 0u;
    e[it] = r >= 0 ? sc[r * kRowWords + kDLat / 8 + (lane >> 4)] : 0u;
  }
  const int64_t row = tid < 8 * kTok ? src_row[tid >> 3] : -1;
  if (row >= 0) w = __builtin_nontemporal_load(&sk[row * 8 + (tid & 7)]);
#pragma unroll
  for (int it = 0; it < kPass; ++it) {
    const int64_t i = j0 + 4 * it + wave;
    if (i >= p.n) continue;
    const float s = mx4_scale(e[it] >> ((lane >> 2 & 3) * 8) & 255u);
    ((u32x4_t*)p.dst_ckv)[(l * p.n + i) * 64 + lane] = mx4x8_bf16(c[it], s);
  }
  const int64_t j = j0 + (tid >> 3);
  if (tid < 8 * kTok && j < p.n) ((u32x4_t*)p.dst_kpe)[(l * p.n + j) * 8 + (tid & 7)] = w;
}

}  // namespace

hipError_t launch_append(const AppendParams& p, hipStream_t s) {
  const int64_t waves = (p.T + p.wave_toks - 1) / p.wave_toks;
  const int64_t grid = (waves + 3) / 4;
  if (grid <= 0) return hipSuccess;
  if (p.mx4) hipLaunchKernelGGL(append_kernel<true>, dim3((uint32_t)grid), dim3(kThreads), 0, s, p);
  else hipLaunchKernelGGL(append_kernel<false>, dim3((uint32_t)grid), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_fetch_gather_mx4(const FetchParams& p, hipStream_t s) {
  // one launch holds 2^24 workgroups of 256: their rows would fill 288 GiB
  const int64_t grid = (int64_t)p.L * ((p.n + kGatherToks - 1) / kGatherToks);
  if (grid <= 0) return hipSuccess;
  hipLaunchKernelGGL(gather_mx4_kernel, dim3((uint32_t)grid), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace mla
