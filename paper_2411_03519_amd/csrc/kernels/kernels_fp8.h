// Host-side launchers of the 8-bit feed-forward kernels.  Shapes are checked by
// the entry points before any launch; the launchers assume them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace metro {

// --- rows (rows_fp8.hip) -----------------------------------------------------

constexpr int kNormFp8MaxDim = 8192;

struct NormFp8Args {
  const float* x;         // [rows][ldx]
  const uint16_t* delta;  // [rows][ldd] bf16, or null
  const uint16_t* gain;   // [d] bf16
  float eps;
  float* x_out;           // [rows][ldx] or null
  uint16_t* h16;          // [rows][ldh16] bf16, or null
  uint8_t* h;             // [rows][ldh] e4m3
  uint8_t* h_scale;       // [rows][lds] E8M0
  int ldx, ldd, ldh16, ldh, lds, rows, d;
};
hipError_t launch_rmsnorm_fp8(const NormFp8Args& a, hipStream_t s);

// Row-major bf16 [N, ld] (first K columns) -> packed 8-bit weights and bytes
hipError_t launch_pack_weight_fp8(const uint16_t* src, int64_t ld, int N, int K, int Kp, uint8_t* dst, uint8_t* scale,
                                  hipStream_t s);

// out[t] = resid[t] + sum_j weights[t, j] * y[slot[t, j]]
struct CombineArgs {
  const uint16_t* y;     // [y_rows][ldy] bf16
  const float* weights;  // [T][k]
  const int32_t* slot;   // [T][k]
  const float* resid;    // [T][ldo] or null
  float* out;            // [T][ldo]
  int ldy, y_rows, ldo, T, k, d;
};
hipError_t launch_combine(const CombineArgs& a, hipStream_t s);

// --- routing (route.hip) -----------------------------------------------------

constexpr int kRouteMaxExperts = 512;
constexpr int kRouteMaxTopK = 32;
constexpr int kRouteMaxGroups = 64;
constexpr int kRouteMaxTokens = 1 << 24;  // (times kRouteMaxTopK within 31 bits)
constexpr int kRouteBlock = 64;  // tokens whose places in the experts' rows one workgroup finds

struct RouteArgs {
  const float* logits;  // [T][ldl]
  const float* bias;    // [E] or null
  int ldl, T, E, k, sigmoid, groups, top_groups, renormalise;
  float scale;
  int32_t* experts;  // [T][k]
  float* weights;    // [T][k]
  int32_t* offsets;  // [E + 1]
  int32_t* src;      // [T * k]
  int32_t* slot;     // [T][k]
  int32_t* ws;       // [E][ceil(T / kRouteBlock)], unused for one block
};
hipError_t launch_route(const RouteArgs& a, hipStream_t s);

// --- products (gemm_fp8.hip) ---------------------------------------------------

enum GemmFp8Epilogue {
  kEpi8Bf16 = 0,    // out[m, n] = bf16(acc)
  kEpi8SwiGLU = 2,  // silu(gate) * up of W rows in blocks of 8 gate, 8 up -> 8-bit rows
};

// Dense (offsets null): rows m = 0 .. M-1 of X with one W.  By experts: slots
// offsets[e] .. offsets[e + 1] - 1 (within 0 .. M) take W + e * N * Kp, slot m
// row src[m] of X (row m where src is null).
constexpr int kGemmFp8MaxRows = 1 << 26, kGemmFp8MaxCols = 1 << 30, kGemmFp8MaxExperts = 1024;
constexpr int64_t kGemmFp8MaxOut = int64_t{1} << 36;  // results: workgroups of any plan that is chosen fit a grid
struct GemmFp8Args {
  const uint8_t* X;        // [x_rows][ldx] e4m3
  const uint8_t* x_scale;  // [x_rows][ldxs]
  const uint8_t* W;        // packed
  const uint8_t* w_scale;  // packed
  const int32_t* src;
  const int32_t* offsets;
  uint16_t* out16;     // [M][ldo]
  uint8_t* out8;       // [M][ldo]
  uint8_t* out_scale;  // [M][ldos]
  float* ws;
  int64_t ws_floats;
  int ldx, ldxs, ldo, ldos, Kp, M, N, E, x_rows;
};

enum class GemmFp8Kind { kDirect, kStream, kTiled };
struct GemmFp8Plan {
  GemmFp8Kind kind;
  int nt, mt;  // 16-row tiles of W and of X: of a workgroup, kTiled: of each of its 2 x 2 waves
  int ks;      // k slices through the workspace and a finishing launch; 0: none
  bool nt_hint;  // kTiled: W passes the caches by
};
GemmFp8Plan plan_gemm_fp8(const GemmFp8Args& a, int epilogue);
hipError_t launch_gemm_fp8(const GemmFp8Args& a, int epilogue, hipStream_t s);

}  // namespace metro
