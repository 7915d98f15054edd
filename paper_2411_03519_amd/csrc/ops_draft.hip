// extern "C" entry points of a speculative decoding step's operators
// (include/metro_ops.h): argument checks, then one launcher.
#include <hip/hip_runtime.h>

#include <cmath>
#include <stdint.h>

#include "../../include/metro_ops.h"
#include "errors.h"
#include "kernels/kernels_draft.h"

using metro::clear_error;
using metro::report;

namespace {

constexpr int32_t kMaxPages = (INT32_MAX - 15) / 16;  // (slots are int32)
constexpr int64_t kMaxBlocks = 1 << 22;

bool misaligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

metro_status launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return METRO_OK;
  return report(METRO_E_HIP, "HIP error %d (%s) in %s", static_cast<int>(e), hipGetErrorString(e), what);
}

// the cache's shape, which three of the operators share
metro_status check_cache(const char* who, const void* kv, int32_t n_pages, int32_t nkv, int32_t hd) {
  if (hd != 64 && hd != 128) return report(METRO_E_INVAL, "%s: head_dim must be 64 or 128", who);
  if (nkv <= 0 || nkv > 256) return report(METRO_E_INVAL, "%s: 1 to 256 kv heads required", who);
  if (n_pages <= 0 || n_pages > kMaxPages) return report(METRO_E_INVAL, "%s: 1 to %d pages required", who, kMaxPages);
  if (misaligned(kv, 16)) return report(METRO_E_INVAL, "%s: kv must be 16-byte aligned", who);
  return METRO_OK;
}

metro_status check_tree(const char* who, int32_t nq, int32_t nkv, int32_t items, int32_t rows, int32_t max_q,
                        int32_t max_keys) {
  if (nq <= 0 || nkv <= 0 || nq % nkv) return report(METRO_E_INVAL, "%s: nq must be a multiple of nkv", who);
  const int g = nq / nkv;
  if (g != 1 && g != 2 && g != 4 && g != 8) return report(METRO_E_INVAL, "%s: group size must be 1, 2, 4 or 8", who);
  if (items < 0 || rows < 0) return report(METRO_E_INVAL, "%s: items or rows < 0", who);
  if (max_q <= 0 || max_q > metro::kTreeMaxQ)
    return report(METRO_E_INVAL, "%s: max_q must be 1 .. %d", who, metro::kTreeMaxQ);
  if (max_keys <= 0 || max_keys > metro::kTreeMaxKeys)
    return report(METRO_E_INVAL, "%s: max_keys must be 1 .. %d", who, metro::kTreeMaxKeys);
  if (static_cast<int64_t>(items) * nkv * ((max_q * g + 15) / 16) > kMaxBlocks || static_cast<int64_t>(items) * max_q > kMaxBlocks)
    return report(METRO_E_INVAL, "%s: more than 2^22 items by queries or by tiles of 16 columns", who);
  return METRO_OK;
}

}  // namespace

extern "C" {

metro_status metro_op_rope_append(const float* qkv_f32, const uint16_t* qkv_bf16, int32_t ld, int32_t T, int32_t nq,
                                  int32_t nkv, int32_t hd, const uint16_t* q_gain, const uint16_t* k_gain, float eps,
                                  const float* rope, int32_t n_pos, const int32_t* pos, const int32_t* slot, uint16_t* q,
                                  uint16_t* kv, int32_t n_pages, void* stream) {
  clear_error();
  const metro_status st = check_cache("rope_append", kv, n_pages, nkv, hd);
  if (st != METRO_OK) return st;
  if (qkv_f32 && qkv_bf16) return report(METRO_E_INVAL, "rope_append: rows in fp32 or in bf16, not both");
  if (T < 0 || (T > 0 && ((!qkv_f32 && !qkv_bf16) || !rope || !pos || !slot || !q || !kv)))
    return report(METRO_E_INVAL, "rope_append: NULL argument or T < 0");
  if (nq <= 0 || nq > 1024 || n_pos <= 0) return report(METRO_E_INVAL, "rope_append: nq must be 1 .. 1024, n_pos positive");
  const int32_t width = (nq + 2 * nkv) * hd;
  if (ld < width || ld % 8) return report(METRO_E_INVAL, "rope_append: ld must be a multiple of 8 from (nq + 2 nkv) hd on");
  if (static_cast<int64_t>(T) * (nq + 2 * nkv) > 1 << 25)
    return report(METRO_E_INVAL, "rope_append: more than 2^25 rows by heads");
  if (misaligned(qkv_f32, 16) || misaligned(qkv_bf16, 16) || misaligned(q, 16) || misaligned(rope, 16) ||
      misaligned(q_gain, 16) || misaligned(k_gain, 16) || misaligned(pos, 4) || misaligned(slot, 4))
    return report(METRO_E_INVAL, "rope_append: qkv, q, rope and the gains must be 16-byte, pos and slot 4-byte aligned");
  const metro::AppendArgs a{qkv_f32, qkv_bf16, q_gain, k_gain, reinterpret_cast<const float2*>(rope), pos, slot, q, kv, eps,
                            ld, T, nq, nkv, hd, n_pos, n_pages};
  return launched(metro::launch_rope_append(a, static_cast<hipStream_t>(stream)), "rope_append");
}

metro_status metro_op_kv_move(uint16_t* kv, int64_t layer_stride, int32_t n_layers, int32_t n_pages, int32_t nkv, int32_t hd,
                              const int32_t* src, const int32_t* dst, const int32_t* offsets, int32_t n_groups,
                              int32_t n_moves, void* stream) {
  clear_error();
  const metro_status st = check_cache("kv_move", kv, n_pages, nkv, hd);
  if (st != METRO_OK) return st;
  if (n_layers < 0 || n_layers > metro::kMoveMaxLayers || n_groups < 0 || n_groups > metro::kMoveMaxGroups || n_moves < 0)
    return report(METRO_E_INVAL, "kv_move: 0 to %d layers, 0 to %d groups, n_moves >= 0 required", metro::kMoveMaxLayers,
                  metro::kMoveMaxGroups);
  if (n_layers > 0 && n_groups > 0 && n_moves > 0 && (!kv || !src || !dst || !offsets))
    return report(METRO_E_INVAL, "kv_move: NULL argument");
  if (n_layers > 1 && (layer_stride < static_cast<int64_t>(n_pages) * 2 * nkv * 16 * hd || layer_stride % 8))
    return report(METRO_E_INVAL, "kv_move: layer_stride must be a multiple of 8 that covers a layer's pages");
  if (misaligned(src, 4) || misaligned(dst, 4) || misaligned(offsets, 4))
    return report(METRO_E_INVAL, "kv_move: src, dst and offsets must be 4-byte aligned");
  const metro::MoveArgs a{kv, layer_stride, src, dst, offsets, n_layers, n_pages, nkv, hd, n_groups, n_moves};
  return launched(metro::launch_kv_move(a, static_cast<hipStream_t>(stream)), "kv_move");
}

metro_status metro_op_attn_tree_workspace(int32_t nq, int32_t nkv, int32_t hd, int32_t n_items, int32_t rows, int32_t max_q,
                                          int32_t max_keys, int64_t* bytes) {
  clear_error();
  metro_status st = check_cache("attn_tree_workspace", nullptr, 1, nkv, hd);
  if (st == METRO_OK) st = check_tree("attn_tree_workspace", nq, nkv, n_items, rows, max_q, max_keys);
  if (st != METRO_OK) return st;
  if (!bytes) return report(METRO_E_INVAL, "attn_tree_workspace: NULL output");
  *bytes = 0;
  if (n_items == 0 || rows == 0) return METRO_OK;
  const metro::TreePlan p = metro::plan_attn_tree(nq, nkv, hd, n_items, rows, max_q, max_keys, INT64_MAX / 8);
  if (p.splits > 1) *bytes = static_cast<int64_t>(p.splits) * rows * nq * (hd + 2) * 4;
  return METRO_OK;
}

metro_status metro_op_attn_tree(const uint16_t* q, const uint16_t* kv, int32_t n_pages, int32_t nq, int32_t nkv, int32_t hd,
                                int32_t n_items, const int32_t* cu_q, int32_t rows, const int32_t* ctx, int32_t max_q,
                                int32_t max_keys, const uint32_t* mask, int32_t ldm, const int32_t* block_tables,
                                int32_t ldb, uint16_t* out, float* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  metro_status st = check_cache("attn_tree", kv, n_pages, nkv, hd);
  if (st == METRO_OK) st = check_tree("attn_tree", nq, nkv, n_items, rows, max_q, max_keys);
  if (st != METRO_OK) return st;
  if (n_items > 0 && rows > 0 && (!q || !kv || !cu_q || !ctx || !block_tables || !out))
    return report(METRO_E_INVAL, "attn_tree: NULL argument");
  if (mask && static_cast<int64_t>(ldm) * 32 < max_q) return report(METRO_E_INVAL, "attn_tree: ldm words hold fewer than max_q bits");
  if (static_cast<int64_t>(ldb) * 16 < max_keys) return report(METRO_E_INVAL, "attn_tree: ldb pages hold fewer than max_keys keys");
  if (workspace_bytes < 0) return report(METRO_E_INVAL, "attn_tree: workspace_bytes < 0");
  if (misaligned(q, 16) || misaligned(out, 16) || misaligned(workspace, 16) || misaligned(cu_q, 4) || misaligned(ctx, 4) ||
      misaligned(mask, 4) || misaligned(block_tables, 4))
    return report(METRO_E_INVAL, "attn_tree: q, out and workspace must be 16-byte, the index arrays and mask 4-byte aligned");
  const metro::TreeArgs a{q, kv, cu_q, ctx, mask, block_tables, out, workspace, workspace ? workspace_bytes / 4 : 0,
                          1.0f / std::sqrt(static_cast<float>(hd)), n_items, rows, nq, nkv, hd, n_pages, max_q, max_keys, ldm, ldb};
  return launched(metro::launch_attn_tree(a, static_cast<hipStream_t>(stream)), "attn_tree");
}

metro_status metro_op_sample_workspace(int32_t rows, int32_t vocab, int64_t* bytes) {
  clear_error();
  if (rows < 0 || vocab <= 0 || vocab > metro::kSampleMaxVocab || !bytes)
    return report(METRO_E_INVAL, "sample_workspace: rows >= 0, vocab 1 .. %d and an output required", metro::kSampleMaxVocab);
  *bytes = rows > 0 ? metro::sample_workspace(rows, vocab) : 0;
  return METRO_OK;
}

metro_status metro_op_sample(const float* logits, int32_t ldl, int32_t rows, int32_t vocab, const float* temperature,
                             const int32_t* top_k, const float* top_p, const float* min_p, const float* u, int32_t* out,
                             float* prob, void* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  if (rows < 0 || (rows > 0 && (!logits || !u || !out))) return report(METRO_E_INVAL, "sample: NULL argument or rows < 0");
  if (vocab <= 0 || vocab > metro::kSampleMaxVocab || ldl < vocab)
    return report(METRO_E_INVAL, "sample: vocab must be 1 .. %d, ldl at least vocab", metro::kSampleMaxVocab);
  if (rows > metro::kSampleMaxRows) return report(METRO_E_INVAL, "sample: more than %d rows", metro::kSampleMaxRows);
  if (misaligned(logits, 4) || misaligned(temperature, 4) || misaligned(top_k, 4) || misaligned(top_p, 4) ||
      misaligned(min_p, 4) || misaligned(u, 4) || misaligned(out, 4) || misaligned(prob, 4) || misaligned(workspace, 16))
    return report(METRO_E_INVAL, "sample: buffers must be 4-byte, workspace 16-byte aligned");
  if (rows > 0) {
    const int64_t need = metro::sample_workspace(rows, vocab);
    if (workspace_bytes < need || (need > 0 && !workspace))
      return report(METRO_E_INVAL, "sample: a workspace of %lld bytes is needed", static_cast<long long>(need));
  }
  const metro::SampleArgs a{logits, temperature, top_k, top_p, min_p, u, out, prob, static_cast<char*>(workspace), workspace_bytes,
                            ldl, rows, vocab};
  return launched(metro::launch_sample(a, static_cast<hipStream_t>(stream)), "sample");
}

}  // extern "C"
