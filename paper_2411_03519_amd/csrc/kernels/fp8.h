// Device helpers of the 8-bit feed-forward kernels (gfx950, wave64).
//
// An 8-bit row holds e4m3 codes (4 exponent bits, 3 mantissa bits, largest
// finite value 448) and, for each 128 consecutive values, one byte E: the power
// of two 2^(E - 127) that the codes are multiples of (E8M0).  A group's power
// is the smallest that brings its largest magnitude within 448, at least
// 2^-126; codes round to nearest, ties to even.  A power of two and not the
// exact maximum / 448, because the matrix cores then apply it themselves
// (v_mfma_scale_*) and a value code * 2^(E - 127) is exact in bf16 and fp32.  An
// infinity or a NaN makes a NaN code (a NaN does not count for the power, an
// infinity makes it 2^120).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"

namespace metro {

constexpr int kGroup = 128;  // values that share a power of two

typedef int i32x8 __attribute__((ext_vector_type(8)));

// E8M0 byte of a group whose largest magnitude is amax: 448 = 1.75 * 2^8, so the
// exponent of amax less 8, one more where its mantissa is above 1.75.
__device__ __forceinline__ int e8m0_of(float amax) {
  return max(static_cast<int>((__float_as_uint(amax) + 0x1fffffu) >> 23) - 8, 1);
}

// 2^(127 - e), 1 <= e <= 253
__device__ __forceinline__ float e8m0_inverse(int e) { return __uint_as_float(static_cast<uint32_t>(254 - e) << 23); }

// e4m3 codes of four values scaled into range
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}

__device__ __forceinline__ int padded_groups(int k) { return (k / kGroup + 3) / 4 * 4; }

// Weights W [N][Kp] of 8 bits in the operand order of the 16 x 16 x 128 matrix
// instruction: tiles of 16 rows x 128 columns, row-major over (n / 16, k / 128),
// each two halves of 64 columns, a half 64 chunks of 16 bytes in lane order: lane
// l = 16 g + r has W[16 tn + r][128 tk + 64 h + 16 g .. + 15].  (Which columns of
// the 128 a lane feeds does not matter to the sum as long as X's lanes take the
// same ones.)
__host__ __device__ __forceinline__ int64_t packed8_offset(int64_t n, int64_t k, int64_t Kp) {
  return ((n >> 4) * (Kp >> 7) + (k >> 7)) * 2048 + ((k >> 6) & 1) * 1024 + ((n & 15) + 16 * ((k >> 4) & 3)) * 16 +
         (k & 15);
}
// Their E8M0 bytes, groups of four 128-column blocks together: byte of row n,
// block kb (groups = Kp / 128 rounded up to a multiple of 4)
__host__ __device__ __forceinline__ int64_t packed8_scale_offset(int64_t n, int64_t kb, int64_t groups) {
  return (((n >> 4) * (groups >> 2) + (kb >> 2)) * 16 + (n & 15)) * 4 + (kb & 3);
}

// Two 16-row blocks of W rows, each 8 gate rows then the 8 matching up rows:
// lanes 0-31 get gate and up of block x, lanes 32-63 of block y.
__device__ __forceinline__ void gate_and_up(f32x4 x, f32x4 y, f32x4& gate, f32x4& up) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[i]), __float_as_uint(y[i]), false, false);
    gate[i] = __uint_as_float(p[0]);
    up[i] = __uint_as_float(p[1]);
  }
}

}  // namespace metro
