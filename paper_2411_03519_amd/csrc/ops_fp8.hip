// extern "C" entry points of the 8-bit feed-forward operators (include/metro_ops.h):
// argument checks, then one launcher.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "../../include/metro_ops.h"
#include "errors.h"
#include "kernels/kernels_fp8.h"

using metro::clear_error;
using metro::report;

namespace {

bool misaligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }
int32_t groups_of(int32_t k) { return (k + 127) / 128; }
bool too_large(int32_t M, int32_t N, int32_t experts) {
  return M > metro::kGemmFp8MaxRows || N > metro::kGemmFp8MaxCols || static_cast<int64_t>(M) * N > metro::kGemmFp8MaxOut ||
         experts > metro::kGemmFp8MaxExperts;
}

metro_status launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return METRO_OK;
  return report(METRO_E_HIP, "HIP error %d (%s) in %s", static_cast<int>(e), hipGetErrorString(e), what);
}

// the parts that the dense and the experts' product share
metro_status gemm_fp8(const char* who, metro::GemmFp8Args& a, int32_t epilogue, float* workspace,
                      int64_t workspace_bytes, void* stream) {
  if (epilogue != metro::kEpi8Bf16 && epilogue != metro::kEpi8SwiGLU)
    return report(METRO_E_INVAL, "%s: epilogue %d (0 or 2)", who, epilogue);
  const bool swiglu = epilogue == metro::kEpi8SwiGLU;
  if (!a.W || !a.w_scale || (a.M > 0 && (!a.X || !a.x_scale || (swiglu ? !a.out8 || !a.out_scale : !a.out16))))
    return report(METRO_E_INVAL, "%s: NULL operand or output", who);
  if (a.M < 0 || a.N <= 0 || a.N % 32 || a.Kp <= 0 || a.Kp % 128)
    return report(METRO_E_INVAL, "%s: bad shape (rows >= 0, N %% 32, Kp %% 128 required)", who);
  if (too_large(a.M, a.N, a.E))
    return report(METRO_E_INVAL, "%s: more than 2^26 rows, N 2^30, 2^36 results or %d experts", who, metro::kGemmFp8MaxExperts);
  if (a.ldx < a.Kp || a.ldx % 16 || a.ldxs < (groups_of(a.Kp) + 3) / 4 * 4 || a.ldxs % 4)
    return report(METRO_E_INVAL, "%s: ldx must be a multiple of 16 from Kp on, ldxs one of 4 from Kp / 128 on", who);
  if (swiglu ? a.ldo < groups_of(a.N / 2) * 128 || a.ldo % 16 || a.ldos < groups_of(a.N / 2) : a.ldo < a.N || a.ldo % 4)
    return report(METRO_E_INVAL, "%s: bad ldo or ldos", who);
  if (misaligned(a.X, 16) || misaligned(a.x_scale, 4) || misaligned(a.W, 16) || misaligned(a.w_scale, 16) ||
      misaligned(a.out16, 8) || misaligned(a.out8, 16) || misaligned(workspace, 16))
    return report(METRO_E_INVAL, "%s: X, W, w_scale, out_fp8 and workspace must be 16-byte, out_bf16 8-byte and x_scale "
                                 "4-byte aligned", who);
  if (workspace_bytes < 0) return report(METRO_E_INVAL, "%s: workspace_bytes < 0", who);
  a.ws = workspace;
  a.ws_floats = workspace ? workspace_bytes / 4 : 0;
  return launched(metro::launch_gemm_fp8(a, epilogue, static_cast<hipStream_t>(stream)), who);
}

// the plan of a product that is described by its sizes alone
metro_status plan_of(const char* who, int32_t M, int32_t N, int32_t Kp, int32_t epilogue, int32_t n_experts,
                     int64_t workspace_bytes, bool outputs, metro::GemmFp8Plan& p) {
  if (!outputs || M <= 0 || N <= 0 || N % 32 || Kp <= 0 || Kp % 128 || n_experts < 0 || workspace_bytes < 0 ||
      (epilogue != metro::kEpi8Bf16 && epilogue != metro::kEpi8SwiGLU))
    return report(METRO_E_INVAL, "%s: bad shape (N %% 32, Kp %% 128), epilogue or NULL output", who);
  if (too_large(M, N, n_experts))
    return report(METRO_E_INVAL, "%s: more than 2^26 rows, N 2^30, 2^36 results or %d experts", who, metro::kGemmFp8MaxExperts);
  static const int32_t some = 0;
  metro::GemmFp8Args a{};
  a.offsets = n_experts ? &some : nullptr;  // (not read)
  a.E = n_experts ? n_experts : 1;
  a.M = M, a.N = N, a.Kp = a.ldx = Kp;
  a.ws_floats = workspace_bytes / 4;
  p = metro::plan_gemm_fp8(a, epilogue);
  return METRO_OK;
}

}  // namespace

extern "C" {

metro_status metro_op_pack_weight_fp8(const uint16_t* W_rowmajor, int32_t ld, int32_t N, int32_t K, int32_t Kp,
                                      uint8_t* W_packed, uint8_t* W_scale, void* stream) {
  clear_error();
  if (!W_rowmajor || !W_packed || !W_scale || N <= 0 || N % 16 || Kp <= 0 || Kp % 128 || K <= 0 || K > Kp || ld < K)
    return report(METRO_E_INVAL, "pack_weight_fp8: bad shape (N %% 16, Kp %% 128, 0 < K <= Kp, ld >= K required) or NULL");
  if (misaligned(W_rowmajor, 2) || misaligned(W_packed, 16) || misaligned(W_scale, 16))
    return report(METRO_E_INVAL, "pack_weight_fp8: W_packed and W_scale must be 16-byte aligned");
  return launched(metro::launch_pack_weight_fp8(W_rowmajor, ld, N, K, Kp, W_packed, W_scale,
                                                static_cast<hipStream_t>(stream)),
                  "pack_weight_fp8");
}

metro_status metro_op_rmsnorm_fp8(const float* x, int32_t ldx, const uint16_t* delta, int32_t ldd, const uint16_t* g,
                                  float eps, float* x_out, uint16_t* h_bf16, int32_t ldh_bf16, uint8_t* h, int32_t ldh,
                                  uint8_t* h_scale, int32_t lds, int32_t rows, int32_t d, void* stream) {
  clear_error();
  if (!g || rows < 0 || (rows > 0 && (!x || !h || !h_scale)) || d <= 0 || d % 4 || d > metro::kNormFp8MaxDim)
    return report(METRO_E_INVAL, "rmsnorm_fp8: bad arguments (d %% 4, d <= %d required)", metro::kNormFp8MaxDim);
  if (rows > 0 && x_out && !delta) return report(METRO_E_INVAL, "rmsnorm_fp8: x_out without delta");
  if (ldx < d || ldx % 4 || (delta && (ldd < d || ldd % 4)) || (h_bf16 && (ldh_bf16 < d || ldh_bf16 % 4)) ||
      ldh < groups_of(d) * 128 || ldh % 4 || lds < groups_of(d))
    return report(METRO_E_INVAL, "rmsnorm_fp8: row strides must reach d (ldh: d rounded up to 128, lds: its groups) and be "
                                 "multiples of 4");
  if (misaligned(x, 16) || misaligned(x_out, 16) || misaligned(delta, 8) || misaligned(g, 8) || misaligned(h_bf16, 8) ||
      misaligned(h, 4))
    return report(METRO_E_INVAL, "rmsnorm_fp8: x and x_out must be 16-byte, delta, g and h_bf16 8-byte, h 4-byte aligned");
  const metro::NormFp8Args a{x, delta, g, eps, x_out, h_bf16, h, h_scale, ldx, ldd, ldh_bf16, ldh, lds, rows, d};
  return launched(metro::launch_rmsnorm_fp8(a, static_cast<hipStream_t>(stream)), "rmsnorm_fp8");
}

metro_status metro_op_gemm_fp8(const uint8_t* X, int32_t ldx, const uint8_t* x_scale, int32_t ldxs, const uint8_t* W,
                               const uint8_t* w_scale, int32_t Kp, int32_t M, int32_t N, int32_t epilogue,
                               uint16_t* out_bf16, uint8_t* out_fp8, int32_t ldo, uint8_t* out_scale, int32_t ldos,
                               float* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  metro::GemmFp8Args a{X, x_scale, W, w_scale, nullptr, nullptr, out_bf16, out_fp8, out_scale, nullptr, 0,
                       ldx, ldxs, ldo, ldos, Kp, M, N, 1, M};
  return gemm_fp8("gemm_fp8", a, epilogue, workspace, workspace_bytes, stream);
}

metro_status metro_op_gemm_fp8_plan(int32_t M, int32_t N, int32_t Kp, int32_t epilogue, int32_t n_experts,
                                    int64_t workspace_bytes, int32_t* kind, int32_t* w_rows, int32_t* x_rows,
                                    int32_t* k_slices) {
  clear_error();
  metro::GemmFp8Plan p;
  const metro_status st = plan_of("gemm_fp8_plan", M, N, Kp, epilogue, n_experts, workspace_bytes,
                                  kind && w_rows && x_rows && k_slices, p);
  if (st != METRO_OK) return st;
  const int waves = p.kind == metro::GemmFp8Kind::kTiled ? 2 : 1;
  *kind = static_cast<int32_t>(p.kind);
  *w_rows = 16 * p.nt * waves;
  *x_rows = 16 * p.mt * waves;
  *k_slices = p.ks;
  return METRO_OK;
}

metro_status metro_op_gemm_fp8_plan_bypass(int32_t M, int32_t N, int32_t Kp, int32_t epilogue, int32_t n_experts,
                                           int64_t workspace_bytes, int32_t* w_bypass) {
  clear_error();
  metro::GemmFp8Plan p;
  const metro_status st =
      plan_of("gemm_fp8_plan_bypass", M, N, Kp, epilogue, n_experts, workspace_bytes, w_bypass != nullptr, p);
  if (st == METRO_OK) *w_bypass = p.nt_hint;
  return st;
}

metro_status metro_op_route(const float* logits, int32_t ldl, const float* bias, int32_t T, int32_t n_experts,
                            int32_t scoring, int32_t n_groups, int32_t top_groups, int32_t top_k, int32_t renormalise,
                            float scale, int32_t* experts, float* weights, int32_t* offsets, int32_t* src, int32_t* slot,
                            int32_t* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  if (!offsets || T < 0 || (T > 0 && (!logits || !experts || !weights || !src || !slot)))
    return report(METRO_E_INVAL, "route: NULL argument or T < 0");
  if (n_experts <= 0 || n_experts > metro::kRouteMaxExperts || ldl < n_experts)
    return report(METRO_E_INVAL, "route: 1 to %d experts, ldl >= n_experts required", metro::kRouteMaxExperts);
  if (scoring != 0 && scoring != 1) return report(METRO_E_INVAL, "route: scoring %d (0 softmax, 1 sigmoid)", scoring);
  if (n_groups <= 0 || n_groups > metro::kRouteMaxGroups || n_experts % n_groups || top_groups <= 0 || top_groups > n_groups)
    return report(METRO_E_INVAL, "route: n_groups must divide n_experts (at most %d), 1 <= top_groups <= n_groups",
                  metro::kRouteMaxGroups);
  if (top_k <= 0 || top_k > metro::kRouteMaxTopK || top_k > n_experts / n_groups * top_groups)
    return report(METRO_E_INVAL, "route: top_k must be 1 .. %d and at most the experts of top_groups groups",
                  metro::kRouteMaxTopK);
  if (T > metro::kRouteMaxTokens) return report(METRO_E_INVAL, "route: more than %d tokens", metro::kRouteMaxTokens);
  if (misaligned(logits, 4) || misaligned(bias, 4) || misaligned(experts, 4) || misaligned(weights, 4) ||
      misaligned(offsets, 4) || misaligned(src, 4) || misaligned(slot, 4) || misaligned(workspace, 4))
    return report(METRO_E_INVAL, "route: misaligned buffer");
  if (T > metro::kRouteBlock) {
    const int64_t need = 4ll * n_experts * ((T + metro::kRouteBlock - 1) / metro::kRouteBlock);
    if (!workspace || workspace_bytes < need)
      return report(METRO_E_INVAL, "route: a workspace of %lld bytes is needed", static_cast<long long>(need));
  }
  const metro::RouteArgs a{logits, bias, ldl, T, n_experts, top_k, scoring, n_groups, top_groups, renormalise, scale,
                           experts, weights, offsets, src, slot, workspace};
  return launched(metro::launch_route(a, static_cast<hipStream_t>(stream)), "route");
}

metro_status metro_op_gemm_fp8_experts(const uint8_t* X, int32_t ldx, const uint8_t* x_scale, int32_t ldxs,
                                       int32_t x_rows, const int32_t* src, const int32_t* offsets, int32_t n_experts,
                                       int32_t R, const uint8_t* W, const uint8_t* w_scale, int32_t Kp, int32_t N,
                                       int32_t epilogue, uint16_t* out_bf16, uint8_t* out_fp8, int32_t ldo,
                                       uint8_t* out_scale, int32_t ldos, float* workspace, int64_t workspace_bytes,
                                       void* stream) {
  clear_error();
  if (!offsets || n_experts <= 0) return report(METRO_E_INVAL, "gemm_fp8_experts: NULL offsets or n_experts <= 0");
  if (misaligned(src, 4) || misaligned(offsets, 4))
    return report(METRO_E_INVAL, "gemm_fp8_experts: src and offsets must be 4-byte aligned");
  if (x_rows < 0 || (src ? R > 0 && x_rows < 1 : x_rows < R))
    return report(METRO_E_INVAL, "gemm_fp8_experts: x_rows must cover the slots (without src) or be at least 1");
  metro::GemmFp8Args a{X, x_scale, W, w_scale, src, offsets, out_bf16, out_fp8, out_scale, nullptr, 0,
                       ldx, ldxs, ldo, ldos, Kp, R, N, n_experts, x_rows};
  return gemm_fp8("gemm_fp8_experts", a, epilogue, workspace, workspace_bytes, stream);
}

metro_status metro_op_combine_experts(const uint16_t* y, int32_t ldy, int32_t y_rows, const float* weights,
                                      const int32_t* slot, int32_t T, int32_t top_k, int32_t d, const float* resid,
                                      float* out, int32_t ldo, void* stream) {
  clear_error();
  if (T < 0 || y_rows < 0 || (T > 0 && (!weights || !slot || !out || (y_rows > 0 && !y))) || top_k <= 0 || d <= 0 || d % 8)
    return report(METRO_E_INVAL, "combine_experts: bad arguments (d %% 8, top_k >= 1 required)");
  if (ldy < d || ldy % 8 || ldo < d || ldo % 4)
    return report(METRO_E_INVAL, "combine_experts: ldy must be a multiple of 8 and ldo one of 4, both from d on");
  if (misaligned(y, 16) || misaligned(resid, 16) || misaligned(out, 16) || misaligned(weights, 4) || misaligned(slot, 4))
    return report(METRO_E_INVAL, "combine_experts: y, resid and out must be 16-byte aligned");
  const metro::CombineArgs a{y, weights, slot, resid, out, ldy, y_rows, ldo, T, top_k, d};
  return launched(metro::launch_combine(a, static_cast<hipStream_t>(stream)), "combine_experts");
}

}  // extern "C"
