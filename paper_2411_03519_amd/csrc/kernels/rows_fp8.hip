// Row kernels of the 8-bit feed-forward block (gfx950, wave64): RMSNorm with the
// residual's addition and 8-bit output, weight packing, and the weighted sum of
// the experts' rows.
#include <algorithm>
#include <type_traits>

#include "fp8.h"
#include "kernels_fp8.h"

namespace metro {

// ---------------------------------------------------------------------------
// x' = x + delta;  h = x' * rsqrt(mean(x'^2) + eps) * g;  h to 8-bit rows.
// One block per row (more rows than blocks: every gridDim-th); a thread holds VPT
// float4 of it, 32 neighbouring lanes one group of 128.  The norm is fp32 and the
// codes are rounded from its fp32 values (not from the optional bf16 ones).
//
// Bound by HBM: a value costs 5 to 13 bytes, and the row stays in registers between
// its sum and its codes (31527 rows of 4096 with everything written: 1.68 GB in 291
// us, 5.8 TB/s, where a copy reaches 5.2; one row 3.6).  Threads without a value only cost
// (rows of 2048 on 512 / 1024 threads, 134 M values with delta and bf16 rows: 212 /
// 353 us; of 512 on 128 / 256: 202 / 295), two float4 a thread pay where blocks
// share a CU (rows of 4096 on 512 x 2 / 1024 x 1 / 256 x 4: 212 / 231 / 217; one
// row 3.5 / 3.3 / 4.6; rows of 8192 on 1024 x 2 / 512 x 4: 226 / 232).
// ---------------------------------------------------------------------------
template <int NTH, int VPT>
__global__ __launch_bounds__(NTH) void rmsnorm_fp8_kernel(NormFp8Args a) {
  constexpr int NWV = NTH / 64;
  __shared__ float red[NWV];
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const int n4 = a.d / 4, pad4 = (a.d + kGroup - 1) / kGroup * (kGroup / 4);
    const float4* xr = reinterpret_cast<const float4*>(a.x + r * a.ldx);
    const uint2* dr = reinterpret_cast<const uint2*>(a.delta + r * a.ldd);
    const uint2* gr = reinterpret_cast<const uint2*>(a.gain);
    float4 v[VPT];
    uint2 gw[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int i = threadIdx.x + j * NTH;
      v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
      gw[j] = make_uint2(0, 0);
      if (i < n4) {
        v[j] = xr[i];
        gw[j] = gr[i];
      }
    }
    if (a.delta) {
      float4* xo = reinterpret_cast<float4*>(a.x_out + r * a.ldx);
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int i = threadIdx.x + j * NTH;
        if (i >= n4) continue;
        const uint2 dw = dr[i];
        v[j].x += lo_bf16(dw.x);
        v[j].y += hi_bf16(dw.x);
        v[j].z += lo_bf16(dw.y);
        v[j].w += hi_bf16(dw.y);
        if (a.x_out) xo[i] = v[j];
      }
    }
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < VPT; ++j) ss += v[j].x * v[j].x + v[j].y * v[j].y + v[j].z * v[j].z + v[j].w * v[j].w;
    ss = wave_sum(ss);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = ss;
    __syncthreads();
    float tot = 0.f;
#pragma unroll
    for (int w = 0; w < NWV; ++w) tot += red[w];
    const float inv = rsqrtf(tot / static_cast<float>(a.d) + a.eps);
    uint32_t* hr = reinterpret_cast<uint32_t*>(a.h + r * a.ldh);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int i = threadIdx.x + j * NTH;
      if (i >= pad4) continue;  // (whole groups of 32 lanes)
      const float4 h = make_float4(v[j].x * inv * lo_bf16(gw[j].x), v[j].y * inv * hi_bf16(gw[j].x),
                                   v[j].z * inv * lo_bf16(gw[j].y), v[j].w * inv * hi_bf16(gw[j].y));
      if (a.h16 && i < n4)
        reinterpret_cast<uint2*>(a.h16 + r * a.ldh16)[i] = make_uint2(pack_bf16x2(h.x, h.y), pack_bf16x2(h.z, h.w));
      // (from 0 on: a group of nothing but NaNs has the least power)
      float m = fmaxf(fmaxf(fmaxf(fabsf(h.x), fabsf(h.y)), fmaxf(fabsf(h.z), fabsf(h.w))), 0.f);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 32));
      const int e = e8m0_of(m);
      const float s = e8m0_inverse(e);
      // columns d .. of the last group: zero codes, whatever 0 * inv * 0 is there
      hr[i] = i < n4 ? pack_e4m3(h.x * s, h.y * s, h.z * s, h.w * s) : 0u;
      if (threadIdx.x % 32 == 0) a.h_scale[r * a.lds + i / 32] = static_cast<uint8_t>(e);
    }
    if (r + gridDim.x < a.rows) __syncthreads();  // (red is read)
  }
}

hipError_t launch_rmsnorm_fp8(const NormFp8Args& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  const int pad4 = (a.d + kGroup - 1) / kGroup * (kGroup / 4);
  auto go = [&](auto nth, auto vpt) {
    constexpr int NTH = decltype(nth)::value, VPT = decltype(vpt)::value;
    rmsnorm_fp8_kernel<NTH, VPT><<<dim3(std::min(a.rows, 1 << 21)), dim3(NTH), 0, s>>>(a);
  };
  using std::integral_constant;
  if (pad4 <= 64)
    go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  else if (pad4 <= 128)
    go(integral_constant<int, 128>{}, integral_constant<int, 1>{});
  else if (pad4 <= 256)
    go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  else if (pad4 <= 512)
    go(integral_constant<int, 512>{}, integral_constant<int, 1>{});
  else if (pad4 <= 1024)
    go(integral_constant<int, 512>{}, integral_constant<int, 2>{});
  else if (pad4 <= kNormFp8MaxDim / 4)
    go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Weights, once at loading: a wave quantises one group (row n, 128 columns), two
// values a lane.  Columns K .. Kp - 1 are zero codes.  Bound by its accesses of two
// bytes a lane: 28672 x 4096 222 us, 1.6 TB/s of bytes that 61 us would move.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(256) void pack_weight_fp8_kernel(const uint16_t* __restrict__ src, int64_t ld, int N, int K,
                                                              int Kp, uint8_t* __restrict__ dst,
                                                              uint8_t* __restrict__ scale) {
  const int lane = threadIdx.x & 63, groups = Kp / kGroup, padded = padded_groups(Kp);
  const int64_t n = static_cast<int64_t>(N) * padded;
  for (int64_t u = blockIdx.x * 4ll + (threadIdx.x >> 6); u < n; u += 4ll * gridDim.x) {
    const int64_t row = u / padded;
    const int kb = static_cast<int>(u % padded);
    if (kb >= groups) {  // bytes that fill the last four
      if (lane == 0) scale[packed8_scale_offset(row, kb, padded)] = 127;
      continue;
    }
    const int k = kb * kGroup + 2 * lane;
    const float a = k < K ? bf16_to_f32(src[row * ld + k]) : 0.f, b = k + 1 < K ? bf16_to_f32(src[row * ld + k + 1]) : 0.f;
    const int e = e8m0_of(wave_max(fmaxf(fmaxf(fabsf(a), fabsf(b)), 0.f)));
    const float s = e8m0_inverse(e);
    const uint32_t c = __builtin_amdgcn_cvt_pk_fp8_f32(a * s, b * s, 0, false);
    *reinterpret_cast<uint16_t*>(dst + packed8_offset(row, k, Kp)) = static_cast<uint16_t>(c);
    if (lane == 0) scale[packed8_scale_offset(row, kb, padded)] = static_cast<uint8_t>(e);
  }
}

hipError_t launch_pack_weight_fp8(const uint16_t* src, int64_t ld, int N, int K, int Kp, uint8_t* dst, uint8_t* scale,
                                  hipStream_t s) {
  const int64_t waves = static_cast<int64_t>(N) * ((Kp / kGroup + 3) / 4 * 4);
  const int64_t blocks = std::min<int64_t>((waves + 3) / 4, 65536);
  pack_weight_fp8_kernel<<<dim3(static_cast<uint32_t>(blocks)), dim3(256), 0, s>>>(src, ld, N, K, Kp, dst, scale);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// out[t] = resid[t] + sum_j weights[t, j] * y[slot[t, j]], j in order, fp32.  A
// thread owns 8 columns of a token; a slot outside the rows of y adds nothing.
// Bound by HBM: 16001 tokens of 4096 with 2 rows each 786 MB in 143 us, 5.5 TB/s, with 8
// rows of 2048 5.0; 25 tokens 3.1 us.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(256) void combine_kernel(CombineArgs a) {
  const int n8 = a.d / 8;
  const int64_t n = static_cast<int64_t>(a.T) * n8;
  for (int64_t u = blockIdx.x * 256ll + threadIdx.x; u < n; u += 256ll * gridDim.x) {
    const int64_t t = u / n8;
    const int c = static_cast<int>(u % n8) * 8;
    float acc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = 0.f;
    if (a.resid) {
      const float4* p = reinterpret_cast<const float4*>(a.resid + t * a.ldo + c);
      const float4 lo = p[0], hi = p[1];
      acc[0] = lo.x, acc[1] = lo.y, acc[2] = lo.z, acc[3] = lo.w;
      acc[4] = hi.x, acc[5] = hi.y, acc[6] = hi.z, acc[7] = hi.w;
    }
    for (int j = 0; j < a.k; ++j) {
      const int sl = a.slot[t * a.k + j];
      if (sl < 0 || sl >= a.y_rows) continue;
      const float w = a.weights[t * a.k + j];
      const uint4 v = *reinterpret_cast<const uint4*>(a.y + static_cast<int64_t>(sl) * a.ldy + c);
      const uint32_t q[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        acc[2 * i] = fmaf(w, lo_bf16(q[i]), acc[2 * i]);
        acc[2 * i + 1] = fmaf(w, hi_bf16(q[i]), acc[2 * i + 1]);
      }
    }
    float4* o = reinterpret_cast<float4*>(a.out + t * a.ldo + c);
    o[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    o[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
  }
}

hipError_t launch_combine(const CombineArgs& a, hipStream_t s) {
  if (a.T <= 0) return hipSuccess;
  const int64_t blocks = std::min<int64_t>((static_cast<int64_t>(a.T) * (a.d / 8) + 255) / 256, 65536);
  combine_kernel<<<dim3(static_cast<uint32_t>(blocks)), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace metro
