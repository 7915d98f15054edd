// Host-side launchers of the kernels of a speculative decoding step.  Shapes are
// checked by the entry points before any launch; the launchers assume them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace metro {

// --- the paged cache (append.hip) --------------------------------------------

struct AppendArgs {
  const float* y32;        // [T][ld] fp32 rows of a QKV product, or null
  const uint16_t* y16;     // [T][ld] the same in bf16, or null
  const uint16_t* q_gain;  // [hd] bf16, or null
  const uint16_t* k_gain;  // [hd] bf16, or null
  const float2* rope;      // [n_pos][hd / 2] (cos, sin)
  const int32_t* pos;      // [T]
  const int32_t* slot;     // [T] page * 16 + offset, or outside the cache
  uint16_t* q;             // [T][nq][hd] bf16
  uint16_t* kv;            // n_pages pages of one layer
  float eps;
  int ld, T, nq, nkv, hd, n_pos, n_pages;
};
hipError_t launch_rope_append(const AppendArgs& a, hipStream_t s);

struct MoveArgs {
  uint16_t* kv;            // [layers] of n_pages pages, layer_stride elements apart
  int64_t layer_stride;
  const int32_t* src;      // [moves]
  const int32_t* dst;      // [moves]
  const int32_t* offsets;  // [groups + 1]
  int layers, n_pages, nkv, hd, groups, moves;
};
constexpr int kMoveMaxGroups = 65535, kMoveMaxLayers = 65535;
constexpr int kMoveRun = 8;  // moves of a group that are read before any of them is written
hipError_t launch_kv_move(const MoveArgs& a, hipStream_t s);

// --- attention of drafted trees (attn_tree.hip) -------------------------------

struct TreeArgs {
  const uint16_t* q;      // [rows][nq][hd] bf16
  const uint16_t* kv;     // n_pages pages of one layer
  const int32_t* cu;      // [items + 1] first query row of each item
  const int32_t* ctx;     // [items] keys before the item's queries
  const uint32_t* mask;   // [rows][ldm] drafted keys that a query sees, or null: those up to its own
  const int32_t* tables;  // [items][ldb] page ids
  uint16_t* out;          // [rows][nq][hd] bf16
  float* part;            // split states
  int64_t part_floats;
  float scale;            // 1 / sqrt(hd)
  int items, rows, nq, nkv, hd, n_pages, max_q, max_keys, ldm, ldb;
};
constexpr int kTreeMaxQ = 4096;       // queries of an item
constexpr int kTreeMaxKeys = 1 << 30;  // keys of an item
// How a call is cut: `tiles` tiles of `wide` columns (query, head of a group) for each item and kv head, and the keys
// into `splits` parts of `pairs` page pairs.
struct TreePlan {
  int wide, tiles;
  int splits, pairs;
};
TreePlan plan_attn_tree(int nq, int nkv, int hd, int items, int rows, int max_q, int max_keys, int64_t part_floats);
hipError_t launch_attn_tree(const TreeArgs& a, hipStream_t s);

// --- sampling (sample.hip) -----------------------------------------------------

struct SampleArgs {
  const float* logits;       // [rows][ldl]
  const float* temperature;  // [rows] or null: 1
  const int32_t* top_k;      // [rows] or null: all
  const float* top_p;        // [rows] or null: 1
  const float* min_p;        // [rows] or null: 0
  const float* u;            // [rows]
  int32_t* out;              // [rows]
  float* prob;               // [rows] or null
  char* ws;
  int64_t ws_bytes;
  int ldl, rows, vocab;
};
constexpr int kSampleMaxVocab = 1 << 18;
constexpr int kSampleMaxRows = 65535;
int64_t sample_workspace(int rows, int vocab);
hipError_t launch_sample(const SampleArgs& a, hipStream_t s);

}  // namespace metro
