// Reading a 4-bit latent cache: E2M1 codes under a power of two per 32 columns.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mla {

// The scale of exponent byte b: 2^(b - 127); 255 is NaN.  (The conversions take the
// exponent field alone, whose 0 is 2^-127: byte 0 is no zero.)
__device__ __forceinline__ float mx4_scale(uint32_t b) {
  return __uint_as_float(b == 255u ? 0x7FC00000u : b << 23);
}

// Two codes (byte N of w) times s -> two bf16, exact unless past bf16's largest.
template <int N>
__device__ __forceinline__ uint32_t mx4x2_bf16(uint32_t w, float s) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, N));
}

// Eight codes (a dword, low half of a byte first) times s -> eight bf16.
__device__ __forceinline__ uint32_t __attribute__((ext_vector_type(4))) mx4x8_bf16(uint32_t w, float s) {
  typedef uint32_t v4 __attribute__((ext_vector_type(4)));
  return v4{mx4x2_bf16<0>(w, s), mx4x2_bf16<1>(w, s), mx4x2_bf16<2>(w, s), mx4x2_bf16<3>(w, s)};
}

}  // namespace mla
