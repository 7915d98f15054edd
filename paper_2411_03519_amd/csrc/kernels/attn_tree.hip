// Attention of drafted trees over the paged cache (gfx950, MFMA, wave64).
//
// An item's queries see the ctx keys before them and, of the item's own drafted
// keys, those that their mask names: with z = q.k / sqrt(hd) over the keys a
// query sees,  out = sum_t exp(z_t - max z) v_t / sum_t exp(z_t - max z).
//
// The matrix products are those of the decode and prefill kernels: scores S^T =
// K Q^T and outputs O^T += V^T P^T on 16 keys x 16 columns, a column being a
// (query, head) pair of one kv head's group, so that a key is read once for all
// queries of a tree.  A wave takes pairs of pages (32 keys) straight from memory
// into operand registers and holds up to CT tiles of 16 columns against each;
// the waves of a workgroup share a split's pairs in turn and merge their (max,
// sum, output) states through LDS in wave order, and a second launch merges the
// splits in order.  Scores, softmax and sums are fp32; the weights enter the
// bf16 matrix cores as hi + lo, about 16 significant bits.
#include "common.h"
#include "kernels.h"
#include "kernels_draft.h"

namespace metro {

constexpr float kTreeLog2e = 1.4426950408889634f;
// the running maximum before any key: every finite score of use lies above it, and differences from it are finite
constexpr float kTreeNone = -1.7e38f;
constexpr int kTreeWaves = 4;

__device__ __forceinline__ f32x4 mfma32(uint4 a, uint4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
}

// Keep the values of a V^T operand word (keys k, k + 1) below key n that are finite; *odd tells of others.
__device__ __forceinline__ uint32_t keep_finite(uint32_t w, int k, int n, bool* odd) {
  if (k + 1 >= n) w = k < n ? w & 0xffffu : 0u;
  if ((w & 0x7f80u) == 0x7f80u) {
    w &= 0xffff0000u;
    *odd = true;
  }
  if ((w & 0x7f800000u) == 0x7f800000u) {
    w &= 0xffffu;
    *odd = true;
  }
  return w;
}

struct TreeItem {
  int row0, n, ctx, keys, pairs;
};

__device__ __forceinline__ TreeItem tree_item(const TreeArgs& a, int item) {
  TreeItem t;
  t.row0 = min(max(a.cu[item], 0), a.rows);
  t.n = min(min(max(a.cu[item + 1], t.row0), a.rows) - t.row0, a.max_q);
  t.ctx = min(max(a.ctx[item], 0), a.max_keys);
  t.keys = min(t.ctx + t.n, a.max_keys);
  t.pairs = (t.keys + 2 * kPage - 1) / (2 * kPage);
  return t;
}

template <int HD, int G, int CT>
__global__ __launch_bounds__(kTreeWaves * 64) void attn_tree_kernel(TreeArgs a, int q_tiles, int splits, int pairs_per_split) {
  constexpr int NW = kTreeWaves;
  constexpr int KQ = HD / 32, NT = HD / 16;
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int b = blockIdx.x;
  const int h = b % a.nkv;
  b /= a.nkv;
  const int qt = b % q_tiles;
  b /= q_tiles;
  const int split = b % splits, item = b / splits;
  const TreeItem it = tree_item(a, item);
  const int col0 = qt * CT * 16, cols = it.n * G;
  if (col0 >= cols) return;
  const int p0 = split * pairs_per_split, p1 = min(p0 + pairs_per_split, it.pairs);
  if (p0 >= p1 && split > 0) return;
  const float qscale = a.scale * kTreeLog2e;
  const int32_t* bt = a.tables + static_cast<size_t>(item) * a.ldb;
  const int last_page = (it.keys - 1) / kPage;

  uint4 qf[CT][KQ];
  f32x4 o[CT][NT];
  float m[CT], l[CT];
  int tok[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int c = col0 + 16 * ct + col;
    tok[ct] = c / G;
    const bool on = c < cols;
    const uint16_t* qp = a.q + (static_cast<size_t>(it.row0 + (on ? tok[ct] : 0)) * a.nq + h * G + c % G) * HD + 8 * grp;
#pragma unroll
    for (int i = 0; i < KQ; ++i) qf[ct][i] = on ? *reinterpret_cast<const uint4*>(qp + 32 * i) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int t = 0; t < NT; ++t) o[ct][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    m[ct] = kTreeNone;
    l[ct] = 0.f;
  }
  const size_t pstride = static_cast<size_t>(2) * a.nkv * kPage * HD;

  for (int p = p0 + wave; p < p1; p += NW) {
    const uint16_t* page[2];
#pragma unroll
    for (int pg = 0; pg < 2; ++pg) {
      const int id = min(max(bt[min(2 * p + pg, last_page)], 0), a.n_pages - 1);
      page[pg] = a.kv + static_cast<size_t>(id) * pstride + static_cast<size_t>(h) * kPage * HD;
    }
    uint4 kf[2][KQ], vf[2][NT / 2];
#pragma unroll
    for (int pg = 0; pg < 2; ++pg) {
#pragma unroll
      for (int i = 0; i < KQ; ++i) kf[pg][i] = *reinterpret_cast<const uint4*>(page[pg] + 512 * i + 8 * lane);
#pragma unroll
      for (int c = 0; c < NT / 2; ++c)
        vf[pg][c] = *reinterpret_cast<const uint4*>(page[pg] + static_cast<size_t>(a.nkv) * kPage * HD + 512 * c + 8 * lane);
    }
    const bool masked = (2 * p + 2) * kPage > it.ctx;
    bool odd = false;
    if (masked) {
#pragma unroll
      for (int pg = 0; pg < 2; ++pg) {
        const int k0 = (2 * p + pg) * kPage + 4 * grp;
#pragma unroll
        for (int c = 0; c < NT / 2; ++c) {
          uint4& v = vf[pg][c];
          v.x = keep_finite(v.x, k0, it.keys, &odd);
          v.y = keep_finite(v.y, k0 + 2, it.keys, &odd);
          v.z = keep_finite(v.z, k0, it.keys, &odd);
          v.w = keep_finite(v.w, k0 + 2, it.keys, &odd);
        }
      }
      odd = __any(odd);
    }
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      float s[2][4];
#pragma unroll
      for (int pg = 0; pg < 2; ++pg) {
        f32x4 sc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KQ; ++i) sc = mfma32(kf[pg][i], qf[ct][i], sc);
#pragma unroll
        for (int r = 0; r < 4; ++r) s[pg][r] = sc[r] * qscale;
      }
      if (masked) {
        const uint32_t* words = a.mask && tok[ct] < it.n ? a.mask + static_cast<size_t>(it.row0 + tok[ct]) * a.ldm : nullptr;
#pragma unroll
        for (int pg = 0; pg < 2; ++pg)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int k = (2 * p + pg) * kPage + 4 * grp + r, j = k - it.ctx;
            const bool see = k < it.keys && (j < 0 || (words ? ((words[j >> 5] >> (j & 31)) & 1u) != 0 : !a.mask && j <= tok[ct]));
            if (!see) s[pg][r] = -INFINITY;
          }
      }
      float mp = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                       fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
      mp = max_xor32(max_xor16(mp));
      const float mn = fmaxf(m[ct], mp);
      const float corr = exp2f(m[ct] - mn);
      m[ct] = mn;
      l[ct] *= corr;
#pragma unroll
      for (int t = 0; t < NT; ++t) o[ct][t] *= corr;
      float pv[2][4];
#pragma unroll
      for (int pg = 0; pg < 2; ++pg)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          pv[pg][r] = __builtin_amdgcn_exp2f(s[pg][r] - mn);
          l[ct] += pv[pg][r];
        }
      // k slot 8 grp + i of the products is key 4 grp + i % 4 of page i / 4
      uint4 hi, lo;
      hi.x = pack_bf16x2(pv[0][0], pv[0][1]);
      hi.y = pack_bf16x2(pv[0][2], pv[0][3]);
      hi.z = pack_bf16x2(pv[1][0], pv[1][1]);
      hi.w = pack_bf16x2(pv[1][2], pv[1][3]);
      lo.x = pack_bf16x2(pv[0][0] - lo_bf16(hi.x), pv[0][1] - hi_bf16(hi.x));
      lo.y = pack_bf16x2(pv[0][2] - lo_bf16(hi.y), pv[0][3] - hi_bf16(hi.y));
      lo.z = pack_bf16x2(pv[1][0] - lo_bf16(hi.z), pv[1][1] - hi_bf16(hi.z));
      lo.w = pack_bf16x2(pv[1][2] - lo_bf16(hi.w), pv[1][3] - hi_bf16(hi.w));
#pragma unroll
      for (int c = 0; c < NT / 2; ++c) {
        const uint4 v0 = make_uint4(vf[0][c].x, vf[0][c].y, vf[1][c].x, vf[1][c].y);
        const uint4 v1 = make_uint4(vf[0][c].z, vf[0][c].w, vf[1][c].z, vf[1][c].w);
        o[ct][2 * c] = mfma32(v0, hi, o[ct][2 * c]);
        o[ct][2 * c] = mfma32(v0, lo, o[ct][2 * c]);
        o[ct][2 * c + 1] = mfma32(v1, hi, o[ct][2 * c + 1]);
        o[ct][2 * c + 1] = mfma32(v1, lo, o[ct][2 * c + 1]);
      }
      // An infinity or a NaN among the drafted values counts for the queries that see its key alone: it is taken
      // out of the operand, where 0 times it would reach all columns, and added by hand.
      if (odd) {
#pragma unroll
        for (int pg = 0; pg < 2; ++pg)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll 1
            for (int g = 0; g < 4; ++g) {
              const float w = __shfl(pv[pg][r], g * 16 + col, kWave);
              const int key = 4 * g + r;
              if ((2 * p + pg) * kPage + key >= it.keys) continue;
              const uint16_t* vt = page[pg] + static_cast<size_t>(a.nkv) * kPage * HD;
#pragma unroll
              for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const uint16_t v = vt[vt_tile_offset(16 * t + 4 * grp + i, key)];
                  if ((v & 0x7f80u) == 0x7f80u && w != 0.f) o[ct][t][i] += w * bf16_to_f32(v);
                }
            }
      }
    }
  }

  // merge the waves in order, one tile at a time
  __shared__ float so[NW][HD][16 + 1];
  __shared__ float sm[NW][16], sl[NW][16];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    if (col0 + 16 * ct >= cols) break;
    float L = l[ct];
    L = sum_xor32(sum_xor16(L));
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) so[wave][16 * t + 4 * grp + i][col] = o[ct][t][i];
    if (grp == 0) {
      sm[wave][col] = m[ct];
      sl[wave][col] = L;
    }
    __syncthreads();
    for (int idx = threadIdx.x; idx < 16 * HD; idx += NW * 64) {
      const int c = idx / HD, d = idx % HD;
      const int gc = col0 + 16 * ct + c;
      if (gc >= cols) break;
      float M = sm[0][c];
#pragma unroll
      for (int w = 1; w < NW; ++w) M = fmaxf(M, sm[w][c]);
      float sum = 0.f, O = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float f = exp2f(sm[w][c] - M);
        sum += sl[w][c] * f;
        O += so[w][d][c] * f;
      }
      const size_t head = static_cast<size_t>(it.row0 + gc / G) * a.nq + h * G + gc % G;
      if (splits == 1) {
        a.out[head * HD + d] = sum == 0.f ? 0 : f32_to_bf16(O / sum);
      } else {
        float* pp = a.part + (static_cast<size_t>(split) * a.rows * a.nq + head) * (HD + 2);
        pp[d] = O;
        if (d == 0) {
          pp[HD] = M;
          pp[HD + 1] = sum;
        }
      }
    }
    __syncthreads();
  }
}

// The splits of each (query, head) in split order.  Grid: (items * max_q, nq); hd threads.
__global__ __launch_bounds__(128) void attn_tree_combine_kernel(TreeArgs a, int splits, int pairs_per_split) {
  const int item = blockIdx.x / a.max_q, tok = blockIdx.x % a.max_q, d = threadIdx.x;
  const TreeItem it = tree_item(a, item);
  if (tok >= it.n) return;
  const int ns = max((it.pairs + pairs_per_split - 1) / pairs_per_split, 1);
  const size_t head = static_cast<size_t>(it.row0 + tok) * a.nq + blockIdx.y;
  const size_t stride = static_cast<size_t>(a.rows) * a.nq * (a.hd + 2);
  const float* pp = a.part + head * (a.hd + 2);
  float M = kTreeNone;
  for (int s = 0; s < ns; ++s) M = fmaxf(M, pp[s * stride + a.hd]);
  float sum = 0.f, O = 0.f;
  for (int s = 0; s < ns; ++s) {
    const float f = exp2f(pp[s * stride + a.hd] - M);
    sum += pp[s * stride + a.hd + 1] * f;
    O += pp[s * stride + d] * f;
  }
  a.out[head * a.hd + d] = sum == 0.f ? 0 : f32_to_bf16(O / sum);
}

TreePlan plan_attn_tree(int nq, int nkv, int hd, int items, int rows, int max_q, int max_keys, int64_t part_floats) {
  const int cols = max_q * (nq / nkv);
  TreePlan p;
  p.ct = cols <= 16 ? 1 : cols <= 32 ? 2 : 4;
  const int64_t tiles = static_cast<int64_t>(items) * nkv * ((cols + 16 * p.ct - 1) / (16 * p.ct));
  const int pairs = (max_keys + 2 * kPage - 1) / (2 * kPage);
  int64_t want = (512 + tiles - 1) / tiles;
  const int64_t state = static_cast<int64_t>(rows) * nq * (hd + 2);
  if (want > part_floats / state) want = part_floats / state;
  if (want > (pairs + kTreeWaves - 1) / kTreeWaves) want = (pairs + kTreeWaves - 1) / kTreeWaves;
  if (want < 1) want = 1;
  p.pairs = static_cast<int>((pairs + want - 1) / want);
  if (p.pairs < 1) p.pairs = 1;
  p.splits = pairs > 0 ? (pairs + p.pairs - 1) / p.pairs : 1;
  return p;
}

template <int HD, int G>
static hipError_t launch_tree_g(const TreeArgs& a, const TreePlan& p, hipStream_t s) {
  const int q_tiles = (a.max_q * G + 16 * p.ct - 1) / (16 * p.ct);
  const dim3 grid(a.items * p.splits * q_tiles * a.nkv), block(kTreeWaves * 64);
  switch (p.ct) {
    case 1: launch_kernel((attn_tree_kernel<HD, G, 1>), grid, block, 0, s, a, q_tiles, p.splits, p.pairs); break;
    case 2: launch_kernel((attn_tree_kernel<HD, G, 2>), grid, block, 0, s, a, q_tiles, p.splits, p.pairs); break;
    default: launch_kernel((attn_tree_kernel<HD, G, 4>), grid, block, 0, s, a, q_tiles, p.splits, p.pairs); break;
  }
  if (p.splits > 1) launch_kernel(attn_tree_combine_kernel, dim3(a.items * a.max_q, a.nq), dim3(HD), 0, s, a, p.splits, p.pairs);
  return hipGetLastError();
}

template <int HD>
static hipError_t launch_tree_hd(const TreeArgs& a, const TreePlan& p, hipStream_t s) {
  switch (a.nq / a.nkv) {
    case 1: return launch_tree_g<HD, 1>(a, p, s);
    case 2: return launch_tree_g<HD, 2>(a, p, s);
    case 4: return launch_tree_g<HD, 4>(a, p, s);
    case 8: return launch_tree_g<HD, 8>(a, p, s);
    default: return hipErrorInvalidValue;
  }
}

hipError_t launch_attn_tree(const TreeArgs& a, hipStream_t s) {
  if (a.items <= 0 || a.rows <= 0) return hipSuccess;
  const TreePlan p = plan_attn_tree(a.nq, a.nkv, a.hd, a.items, a.rows, a.max_q, a.max_keys, a.part_floats);
  return a.hd == 128 ? launch_tree_hd<128>(a, p, s) : launch_tree_hd<64>(a, p, s);
}

}  // namespace metro
