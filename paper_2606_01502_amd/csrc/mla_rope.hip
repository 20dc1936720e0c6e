// Rotary positions: part of each head's dims turned by an angle that grows with
// the row's position, the rest copied.
//
// Pair i of a row at position p becomes m (x cos a - y sin a, x sin a + y cos a),
// a = p w_i; the angular frequencies w_i (long-context scaling included) come
// from the host in turns a position, in double, at most one.  p w_i is formed and
// reduced to one turn in double (a position of 2^31 leaves 2^-22 of a turn, and the
// host's roundings of w_i as much three times), cos and sin of the rest in fp32, the
// products in fp32, one rounding to the output's type.
//
// A stream through HBM: each value read once, written once.  What bounds small
// calls is the launch and the trip; large ones the copy rate.  A workgroup takes
// whole rows (token, head), as many as hold about 2048 16-byte units, forms the
// cosines of the tokens it meets once for all of their heads in LDS, and moves
// units of 16 bytes, four loads before their stores.  4096 tokens of 128 heads x 192
// dims, the last 64 turned (bf16, 403 MB there and back), take 77 us: 5.2 TB/s, a
// copy's rate; 64 tokens of 128 x 64 take 4.6 us, launch and trip.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mla_kernels.h"

namespace mla {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

template <typename T>
__device__ __forceinline__ float widen(T v);
template <>
__device__ __forceinline__ float widen<float>(float v) { return v; }
template <>
__device__ __forceinline__ float widen<__bf16>(__bf16 v) { return (float)v; }

// cos and sin (times m, the sine with the direction's sign) of the pairs of
// tokens t0 .. t0 + n - 1 into cs[n][rot / 2][2]
__device__ __forceinline__ void angles(const RopeParams& p, int64_t t0, int n, float* cs) {
  const int half = p.rot >> 1;
  for (int e = threadIdx.x; e < n * half; e += kThreads) {
    const int k = e / half, i = e - k * half;
    double turns = (double)p.pos[t0 + k] * p.turns[i];
    turns -= rint(turns);
    float s, c;
    sincospif(2.0f * (float)turns, &s, &c);
    cs[2 * e] = c * p.mscale;
    cs[2 * e + 1] = s * p.sin_scale;
  }
}

// VEC: 16-byte units, E values each; else units of one pair or one copied value.
template <typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void rope_kernel(const RopeParams p) {
  extern __shared__ float cs[];
  constexpr int E = VEC ? 16 / (int)sizeof(T) : 1;
  const int64_t row0 = (int64_t)blockIdx.x * p.wg_rows;
  const int n_rows = (int)min((int64_t)p.wg_rows, p.rows - row0);
  const int64_t t0 = row0 / p.H;
  const int h0 = (int)(row0 - t0 * p.H);
  const int n_tok = (h0 + n_rows - 1) / p.H + 1;
  angles(p, t0, n_tok, cs);
  __syncthreads();
  const int half = p.rot >> 1;
  // units of a row: the rotated part, then what is copied.  Pairs of
  // neighbours: a unit is E / 2 pairs (scalar: one pair); pairs half the part
  // apart: a unit and its partner.
  const int n_rot = VEC ? (p.pairing == 0 ? p.rot / E : half / E) : half;
  const int units = p.row_units;
  const T* const x = (const T*)p.x;
  T* const out = (T*)p.out;
  const int total = n_rows * units;
  auto place = [&](int u, int64_t& xi, int64_t& oi, int& k, int& v) {
    const int r = div_by(u, p.by_units);
    v = u - r * units;
    k = div_by(h0 + r, p.by_H);
    const int h = h0 + r - k * p.H;
    xi = (t0 + k) * p.x_s0 + h * p.x_s1;
    oi = (t0 + k) * p.out_s0 + h * p.out_s1;
  };
  // the first column of unit v, and its partner's where it has one
  auto col_of = [&](int v, int& c0, int& c1) {
    c1 = -1;
    if (v < n_rot) {
      if (VEC && p.pairing == 0) {
        c0 = p.at + v * E;
      } else if (p.pairing == 0) {
        c0 = p.at + 2 * v;
        c1 = c0 + 1;
      } else {
        c0 = p.at + v * E;
        c1 = c0 + half;
      }
    } else {
      c0 = (v - n_rot) * E;
      if (c0 >= p.at) c0 += p.rot;
    }
  };
  if constexpr (VEC) {
    constexpr int kAhead = 4;
    for (int base = threadIdx.x; base < total; base += kAhead * kThreads) {
      u32x4_t a[kAhead], b[kAhead];
      int64_t oi[kAhead];
      int k[kAhead], v[kAhead], c0[kAhead], c1[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int u = min(base + j * kThreads, total - 1);  // past the end: loaded, not stored
        int64_t xi;
        place(u, xi, oi[j], k[j], v[j]);
        col_of(v[j], c0[j], c1[j]);
        a[j] = __builtin_nontemporal_load((const u32x4_t*)(x + xi + c0[j]));
        if (c1[j] >= 0) b[j] = __builtin_nontemporal_load((const u32x4_t*)(x + xi + c1[j]));
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (base + j * kThreads >= total) break;
        union {
          u32x4_t w;
          T e[E];
        } ua, ub;
        ua.w = a[j];
        ub.w = b[j];
        if (v[j] < n_rot) {
          const float* t = cs + 2 * (k[j] * half);
          if (p.pairing == 0) {
#pragma unroll
            for (int e = 0; e < E / 2; ++e) {
              const int i = v[j] * (E / 2) + e;
              const float c = t[2 * i], s = t[2 * i + 1];
              const float xe = widen(ua.e[2 * e]), ye = widen(ua.e[2 * e + 1]);
              ua.e[2 * e] = (T)(xe * c - ye * s);
              ua.e[2 * e + 1] = (T)(xe * s + ye * c);
            }
          } else {
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const int i = v[j] * E + e;
              const float c = t[2 * i], s = t[2 * i + 1];
              const float xe = widen(ua.e[e]), ye = widen(ub.e[e]);
              ua.e[e] = (T)(xe * c - ye * s);
              ub.e[e] = (T)(xe * s + ye * c);
            }
          }
        }
        *(u32x4_t*)(out + oi[j] + c0[j]) = ua.w;
        if (c1[j] >= 0) *(u32x4_t*)(out + oi[j] + c1[j]) = ub.w;
      }
    }
  } else {
    for (int u = threadIdx.x; u < total; u += kThreads) {
      int64_t xi, oi;
      int k, v, c0, c1;
      place(u, xi, oi, k, v);
      col_of(v, c0, c1);
      if (c1 >= 0) {
        const float* t = cs + 2 * (k * half + v);
        const float xe = widen(x[xi + c0]), ye = widen(x[xi + c1]);
        out[oi + c0] = (T)(xe * t[0] - ye * t[1]);
        out[oi + c1] = (T)(xe * t[1] + ye * t[0]);
      } else {
        out[oi + c0] = x[xi + c0];
      }
    }
  }
}

}  // namespace

hipError_t launch_rope(const RopeParams& p, hipStream_t s) {
  const int64_t grid = (p.rows + p.wg_rows - 1) / p.wg_rows;
  if (grid <= 0) return hipSuccess;
  const size_t lds = (size_t)p.wg_toks * p.rot * sizeof(float);
  const dim3 g((uint32_t)grid), b(kThreads);
  if (p.fp32 && p.vec) hipLaunchKernelGGL((rope_kernel<float, true>), g, b, lds, s, p);
  else if (p.fp32) hipLaunchKernelGGL((rope_kernel<float, false>), g, b, lds, s, p);
  else if (p.vec) hipLaunchKernelGGL((rope_kernel<__bf16, true>), g, b, lds, s, p);
  else hipLaunchKernelGGL((rope_kernel<__bf16, false>), g, b, lds, s, p);
  return hipGetLastError();
}

}  // namespace mla
