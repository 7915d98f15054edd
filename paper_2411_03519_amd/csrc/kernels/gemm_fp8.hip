// 8-bit products on the matrix cores of gfx950 (v_mfma_scale_f32_16x16x128_f8f6f4,
// fp32 accumulation):  acc[m, n] = sum over blocks kb of 128 columns of
// 2^(sx[m, kb] + sw[n, kb] - 254) * sum_k X[m, k] W[n, k], dense or with the rows of
// each expert against its own W, then bf16 rows or SwiGLU and 8-bit rows.
//
// One instruction takes 16 rows of W (A), 16 rows of X (B) and 128 columns, and
// applies both rows' powers of two itself.  Lane l = 16 g + r supplies 32
// columns of W row r and X row r and one byte of power for each, and receives
// D[4 g + i][r]: four consecutive W rows of X row r.
//
// Precision: accumulators are fp32.  Within one instruction the products of
// each run of eight columns are aligned to the largest of them and cut below
// 2^-13 of it: 1.5e-5 of the result's 2-norm on normal data (2.6e-5 where X is
// a product of normals), against 1.7e-3 that the rounding to bf16 adds behind it.
#include <algorithm>
#include <type_traits>

#include "fp8.h"
#include "kernels_fp8.h"

namespace metro {

namespace {

__device__ __forceinline__ f32x4 mfma8(uint4 a0, uint4 a1, uint4 b0, uint4 b1, f32x4 c, int sa, int sb) {
  const i32x8 a = {static_cast<int>(a0.x), static_cast<int>(a0.y), static_cast<int>(a0.z), static_cast<int>(a0.w),
                   static_cast<int>(a1.x), static_cast<int>(a1.y), static_cast<int>(a1.z), static_cast<int>(a1.w)};
  const i32x8 b = {static_cast<int>(b0.x), static_cast<int>(b0.y), static_cast<int>(b0.z), static_cast<int>(b0.w),
                   static_cast<int>(b1.x), static_cast<int>(b1.y), static_cast<int>(b1.z), static_cast<int>(b1.w)};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb);
}

__device__ __forceinline__ float silu_f32(float z) { return z / (1.0f + expf(-z)); }

// Rows m0 .. m1 - 1 of row block b of BM rows, and their expert.  By experts,
// every expert's rows are cut into blocks of their own; offsets are held within
// 0 .. M, so that whatever they say, rows lie in range.  False: no such block.
__device__ __forceinline__ bool row_block(const GemmFp8Args& a, int b, int BM, int& e, int& m0, int& m1) {
  if (!a.offsets) {
    e = 0;
    m0 = b * BM;
    m1 = min(m0 + BM, a.M);
    return m0 < a.M;
  }
  const int lane = threadIdx.x & 63;
  int carry = 0;
  for (int c = 0; c < a.E; c += 64) {
    const int i = c + lane;
    const int lo = i < a.E ? min(max(a.offsets[i], 0), a.M) : 0;
    const int hi = i < a.E ? min(max(a.offsets[i + 1], 0), a.M) : 0;
    const int nb = (max(hi - lo, 0) + BM - 1) / BM;
    int incl = nb;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int y = __shfl_up(incl, o);
      if (lane >= o) incl += y;
    }
    const int first = carry + incl - nb;
    const uint64_t here = __ballot(b >= first && b < first + nb);
    if (here) {
      const int l = __builtin_ctzll(here);
      e = c + l;
      m0 = __builtin_amdgcn_readlane(lo, l) + (b - __builtin_amdgcn_readlane(first, l)) * BM;
      m1 = min(m0 + BM, __builtin_amdgcn_readlane(hi, l));
      return true;
    }
    carry += __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

// row of X that slot m reads (indexes are held within x_rows)
__device__ __forceinline__ int64_t source_row(const GemmFp8Args& a, int m) {
  return a.src ? min(max(a.src[m], 0), a.x_rows - 1) : m;
}

// ---------------------------------------------------------------------------
// 256 rows of W x 16 MT rows of X per workgroup, operands straight from global
// memory, K whole.  A wave has 64 rows of W; the 128 features of a workgroup's
// SwiGLU output are one group, whose maximum the four waves find through LDS.
// ---------------------------------------------------------------------------
template <int MT, int EPI>
__global__ __launch_bounds__(256) void gemm_fp8_kernel(GemmFp8Args a) {
  int e, m0, m1;
  if (!row_block(a, blockIdx.y, 16 * MT, e, m0, m1)) return;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int groups = padded_groups(a.Kp), nkb = a.Kp / kGroup;
  const uint8_t* W = a.W + static_cast<int64_t>(e) * a.N * a.Kp;
  const uint8_t* ws = a.w_scale + static_cast<int64_t>(e) * a.N * groups;
  const int n0 = blockIdx.x * 256 + wave * 64;
  const uint8_t *wp[4], *wsp[4], *xp[MT], *xsp[MT];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int tn = min(n0 / 16 + i, a.N / 16 - 1);
    wp[i] = W + static_cast<int64_t>(tn) * a.Kp * 16 + lane * 16;
    wsp[i] = ws + static_cast<int64_t>(tn) * groups * 16 + r * 4;
  }
#pragma unroll
  for (int j = 0; j < MT; ++j) {
    const int64_t row = source_row(a, min(m0 + 16 * j + r, m1 - 1));
    xp[j] = a.X + row * a.ldx + 16 * g;
    xsp[j] = a.x_scale + row * a.ldxs;
  }
  f32x4 acc[4][MT];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int kb = 0; kb < nkb; ++kb) {
    uint4 x0[MT], x1[MT];
    int sx[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      x0[j] = *reinterpret_cast<const uint4*>(xp[j] + kb * kGroup);
      x1[j] = *reinterpret_cast<const uint4*>(xp[j] + kb * kGroup + 64);
      sx[j] = xsp[j][kb];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 w0 = *reinterpret_cast<const uint4*>(wp[i] + static_cast<int64_t>(kb) * 2048);
      const uint4 w1 = *reinterpret_cast<const uint4*>(wp[i] + static_cast<int64_t>(kb) * 2048 + 1024);
      const int sw = wsp[i][(kb >> 2) * 64 + (kb & 3)];
#pragma unroll
      for (int j = 0; j < MT; ++j) acc[i][j] = mfma8(w0, w1, x0[j], x1[j], acc[i][j], sw, sx[j]);
    }
  }
  if constexpr (EPI == kEpi8Bf16) {
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      const int m = m0 + 16 * j + r;
      if (m >= m1) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int n = n0 + 16 * i + 4 * g;
        if (n < a.N)
          *reinterpret_cast<uint2*>(a.out16 + static_cast<int64_t>(m) * a.ldo + n) =
              make_uint2(pack_bf16x2(acc[i][j][0], acc[i][j][1]), pack_bf16x2(acc[i][j][2], acc[i][j][3]));
      }
    }
  } else {
    __shared__ float top[4][MT][16];
    const int F = a.N / 2;
    f32x4 y[2][MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      float best = 0.f;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        f32x4 gate, up;
        gate_and_up(acc[2 * p][j], acc[2 * p + 1][j], gate, up);
        const bool in = n0 + 32 * p < a.N;  // (N % 32 == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[p][j][i] = in ? silu_f32(gate[i]) * up[i] : 0.f;
          best = fmaxf(best, fabsf(y[p][j][i]));
        }
      }
      best = max_xor32(max_xor16(best));
      if (g == 0) top[wave][j][r] = best;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      const int m = m0 + 16 * j + r;
      if (m >= m1) continue;
      const int ex = e8m0_of(fmaxf(fmaxf(top[0][j][r], top[1][j][r]), fmaxf(top[2][j][r], top[3][j][r])));
      const float s = e8m0_inverse(ex);
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int f = n0 / 2 + 16 * p + 8 * (g >> 1) + 4 * (g & 1);
        if (f < (F + kGroup - 1) / kGroup * kGroup)  // (columns that fill the last group: zero codes)
          *reinterpret_cast<uint32_t*>(a.out8 + static_cast<int64_t>(m) * a.ldo + f) =
              pack_e4m3(y[p][j][0] * s, y[p][j][1] * s, y[p][j][2] * s, y[p][j][3] * s);
      }
      if (wave == 0 && g == 0) a.out_scale[static_cast<int64_t>(m) * a.ldos + blockIdx.x] = static_cast<uint8_t>(ex);
    }
  }
}

// Row blocks of BM rows that M rows can make: by experts, each may leave one
// partly filled.
int row_blocks(const GemmFp8Args& a, int BM) {
  if (!a.offsets) return (a.M + BM - 1) / BM;
  return static_cast<int>(std::min<int64_t>(a.M, (a.M + static_cast<int64_t>(a.E) * (BM - 1)) / BM));
}

}  // namespace

hipError_t launch_gemm_fp8(const GemmFp8Args& a, int epilogue, hipStream_t s) {
  if (a.M <= 0) return hipSuccess;
  auto go = [&](auto mt) {
    constexpr int MT = decltype(mt)::value;
    const dim3 grid((a.N + 255) / 256, row_blocks(a, 16 * MT));
    if (epilogue == kEpi8SwiGLU)
      gemm_fp8_kernel<MT, kEpi8SwiGLU><<<grid, dim3(256), 0, s>>>(a);
    else
      gemm_fp8_kernel<MT, kEpi8Bf16><<<grid, dim3(256), 0, s>>>(a);
  };
  if (a.M <= 16 * a.E)
    go(std::integral_constant<int, 1>{});
  else
    go(std::integral_constant<int, 4>{});
  return hipGetLastError();
}

}  // namespace metro
