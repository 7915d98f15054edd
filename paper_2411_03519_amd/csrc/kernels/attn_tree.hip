// Attention of drafted trees over the paged cache (gfx950, MFMA, wave64).
//
// An item's queries see the ctx keys before them and, of the item's own drafted
// keys, those that their mask names: with z = q.k / sqrt(hd) over the keys a
// query sees,  out = sum_t exp(z_t - max z) v_t / sum_t exp(z_t - max z).
//
// The matrix products are those of the decode and prefill kernels: scores S^T =
// K Q^T and outputs O^T += V^T P^T on 16 keys x 16 columns, a column being a
// (query, head) pair of one kv head's group, so that a key is read once for all
// queries of a tree.  Pages go in pairs (32 keys).  Up to 32 columns they pass from
// memory straight into operand registers, each wave with pairs of its own; more
// columns are eight waves of 16 against the same pairs, which go through LDS.  The
// keys of an item are cut into splits where that fills the chip, and a second
// launch merges their (max, sum, output) states in order.  Scores, softmax and
// sums are fp32; the weights enter the bf16 matrix cores as hi + lo, about 16
// significant bits, which costs a third of the matrix instructions.
//
// What bounds it.  One token a sequence: K and V, streamed at 5.0 TB/s (123
// contexts of 256 .. 4096 keys, 142 us, and 25 of them 27, 33 where the caches hold none
// of it; the model's decode kernel takes 139 and 29 on the same inputs).  Trees of 8 to
// 32 tokens read the same and are held up besides by the scores' way through the vector
// ALU (exponentials, the split into hi + lo), which overlaps the matrix cores' only
// between waves, and by the waits that the ring's kernel notes: 123 trees 209 to 240 us,
// 25 of 9 to 17 tokens 43 us.  512 columns after 20000 to 30000 keys: matrix cores busy
// 40% of the time, the vector ALU issuing 65% (matrix instructions among them), 206 to
// 238 us, 490 to 425 TFLOP/s of the products asked for and half as many again for lo (a
// large library product reaches 1211 on this card).  A chain's tiles of columns go
// through all pairs of its item, those behind the tile's last query too, where every
// weight is 0: 512 queries 43 us, 4096 of them 1018, 16 items of 512 271, for which
// the model's prefill kernel takes 19, 211 and 92; after a context of 4096 keys 512
// queries 114 against 127.  Two and four tiles a
// wave against LDS or registers, scores of the next pair formed beside this one's
// weights, and tiles of up to 64 columns with the pairs shared by two halves of the
// workgroup gave nothing over this.
#include "common.h"
#include "kernels.h"
#include "kernels_draft.h"

namespace metro {

constexpr float kTreeLog2e = 1.4426950408889634f;
// the running maximum before any key: every finite score of use lies above it, and differences from it are finite
constexpr float kTreeNone = -1.7e38f;
constexpr int kTreeMaxSplits = 64;  // (a lane each in the merge)

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

// Bit b: the item's query tok sees key k0 + b, for a pair of pages from k0 on that reaches into the drafted keys.
__device__ __forceinline__ uint32_t seen_window(const TreeArgs& a, const TreeItem& it, int tok, int k0) {
  auto below = [](int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; };  // bits 0 .. n - 1
  if (tok >= it.n) return 0;
  const int j0 = k0 - it.ctx;  // the drafted key at bit 0; -31 or more
  uint32_t w;
  if (a.mask) {
    const uint32_t* words = a.mask + static_cast<size_t>(it.row0 + tok) * a.ldm;
    const int at = j0 >> 5;  // -1 or more
    const uint32_t lo = at >= 0 && at < a.ldm ? words[at] : 0u, hi = at + 1 < a.ldm ? words[at + 1] : 0u;
    w = static_cast<uint32_t>(((static_cast<uint64_t>(hi) << 32) | lo) >> (j0 & 31));
  } else {
    w = below(tok + 1 - j0);
  }
  return (w | below(-j0)) & below(it.keys - k0);
}

// One wave's CT tiles of 16 columns: queries, running maxima and sums, outputs.
template <int HD, int CT>
struct TreeTiles {
  static constexpr int KQ = HD / 32, NT = HD / 16, NC = NT / 2;
  uint4 q[CT][KQ];
  f32x4 o[CT][NT];
  float m[CT], l[CT];
  int tok[CT];

  __device__ __forceinline__ void start(const TreeArgs& a, const TreeItem& it, int h, int gl, int col0, int cols, int lane) {
    const int col = lane & 15, grp = lane >> 4;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      const int c = col0 + 16 * ct + col;
      tok[ct] = c >> gl;
      const bool on = c < cols;
      const uint16_t* p = a.q + (static_cast<size_t>(it.row0 + (on ? tok[ct] : 0)) * a.nq + (h << gl) + (c & ((1 << gl) - 1))) * HD +
                          8 * grp;
#pragma unroll
      for (int i = 0; i < KQ; ++i) q[ct][i] = on ? *reinterpret_cast<const uint4*>(p + 32 * i) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int t = 0; t < NT; ++t) o[ct][t] = f32x4{0.f, 0.f, 0.f, 0.f};
      m[ct] = kTreeNone;
      l[ct] = 0.f;
    }
  }

  // Scores of a pair of pages; k(pg, i): K operand of page pg, dims 32 i .. 32 i + 31.
  template <typename K>
  __device__ __forceinline__ void scores(K k, float (&s)[CT][8]) {
    f32x4 sc[2][CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) sc[0][ct] = sc[1][ct] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < KQ; ++i)
#pragma unroll
      for (int pg = 0; pg < 2; ++pg) {
        const uint4 kf = k(pg, i);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) sc[pg][ct] = mfma32(kf, q[ct][i], sc[pg][ct]);
      }
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[ct][i] = sc[i >> 2][ct][i & 3];
  }

  // Exponents of the softmax weights, e = z - m in powers of two, of the scores s (value 4 pg + r of lane (col, grp): key
  // 4 grp + r of page pg).
  __device__ __forceinline__ float exponents(const float (&s)[CT][8], float qscale, float (&e)[CT][8]) {
    float top = kTreeNone;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        e[ct][i] = fmaf(s[ct][i], qscale, -m[ct]);
        top = fmaxf(top, e[ct][i]);
      }
    return top;
  }

  // The reference m moves only when an exponent passes 8 (a factor of 2^8 in o and l, which their quotient does not
  // see), so the columns' maxima are formed, and o is scaled, hardly ever.
  __device__ __forceinline__ void refer(const float (&s)[CT][8], float qscale, float top, float (&e)[CT][8]) {
    if (!__any(top > 8.f)) return;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      const float(&v)[8] = s[ct];
      float mp = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
      mp = max_xor32(max_xor16(mp)) * qscale;
      const float mn = fmaxf(m[ct], mp);
      const float corr = exp2f(m[ct] - mn);
      m[ct] = mn;
      l[ct] *= corr;
#pragma unroll
      for (int t = 0; t < NT; ++t) o[ct][t] *= corr;
#pragma unroll
      for (int i = 0; i < 8; ++i) e[ct][i] = fmaf(v[i], qscale, -mn);
    }
  }

  // Weights 2^e as the pair hi + lo of bf16 values, and their sum.  (k slot 8 grp + i of the products with V is key
  // 4 grp + i % 4 of page i / 4.)
  struct Weights {
    uint4 hi[CT], lo[CT];
  };
  __device__ __forceinline__ void weigh(float (&e)[CT][8], Weights& w) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      float(&p)[8] = e[ct];
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = __builtin_amdgcn_exp2f(p[i]);
        sum += p[i];
      }
      l[ct] += sum;
      uint4 &hi = w.hi[ct], &lo = w.lo[ct];
      hi.x = pack_bf16x2(p[0], p[1]);
      hi.y = pack_bf16x2(p[2], p[3]);
      hi.z = pack_bf16x2(p[4], p[5]);
      hi.w = pack_bf16x2(p[6], p[7]);
      lo.x = pack_bf16x2(p[0] - lo_bf16(hi.x), p[1] - hi_bf16(hi.x));
      lo.y = pack_bf16x2(p[2] - lo_bf16(hi.y), p[3] - hi_bf16(hi.y));
      lo.z = pack_bf16x2(p[4] - lo_bf16(hi.z), p[5] - hi_bf16(hi.z));
      lo.w = pack_bf16x2(p[6] - lo_bf16(hi.w), p[7] - hi_bf16(hi.w));
    }
  }

  // o += V^T P^T of a pair; v(c, a, b) fills a, b with the two pages' chunks c of V^T: a page's 16 bytes hold output
  // tiles 2c and 2c + 1, so their inner halves trade places.
  template <typename V>
  __device__ __forceinline__ void add_values(V v, const Weights& w) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      uint4 x, y;
      v(c, x, y);
      swap_halves<2>(x, y);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        o[ct][2 * c] = mfma32(x, w.hi[ct], o[ct][2 * c]);
        o[ct][2 * c + 1] = mfma32(y, w.hi[ct], o[ct][2 * c + 1]);
      }
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        o[ct][2 * c] = mfma32(x, w.lo[ct], o[ct][2 * c]);
        o[ct][2 * c + 1] = mfma32(y, w.lo[ct], o[ct][2 * c + 1]);
      }
    }
  }

  // Scores of the keys that a query does not see, in the pair of pages from key k0 on, become -inf.
  __device__ __forceinline__ void mask(const TreeArgs& a, const TreeItem& it, int k0, int grp, float (&s)[CT][8]) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      const uint32_t see = seen_window(a, it, tok[ct], k0) >> (4 * grp);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (!((see >> (16 * (i >> 2) + (i & 3))) & 1u)) s[ct][i] = -INFINITY;
    }
  }

  // Infinities and NaN among the drafted values count for the queries that see their keys alone.  They were taken out
  // of the operands (keep_finite), where 0 times them would reach all columns; the products of where they are and of
  // which weights are not 0 say which outputs get them.  v0, v1: the pages' V^T tiles in memory.
  __device__ __forceinline__ void add_odd(const TreeItem& it, const uint16_t* v0, const uint16_t* v1, int k0, int lane,
                                          const float (&p)[CT][8]) {
#pragma unroll 1
    for (int kind = 0; kind < 3; ++kind) {
      // +inf, -inf, NaN: bits & mask in base .. base + span
      const uint32_t mask = kind == 2 ? 0x7fffu : 0xffffu, span = kind == 2 ? 0x7eu : 0u;
      const uint32_t base = kind == 0 ? 0x7f80u : kind == 1 ? 0xff80u : 0x7f81u;
      auto mark = [&](uint32_t w, int k) {
        w = k + 1 < it.keys ? w : k < it.keys ? w & 0xffffu : 0u;
        return ((w & mask) - base <= span ? 0x3f80u : 0u) | (((w >> 16) & mask) - base <= span ? 0x3f800000u : 0u);
      };
      const float add = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : __builtin_nanf("");
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const uint4 x = *reinterpret_cast<const uint4*>(v0 + 512 * c + 8 * lane);
        const uint4 y = *reinterpret_cast<const uint4*>(v1 + 512 * c + 8 * lane);
        const uint4 at[2] = {make_uint4(mark(x.x, k0), mark(x.y, k0 + 2), mark(y.x, k0 + kPage), mark(y.y, k0 + kPage + 2)),
                             make_uint4(mark(x.z, k0), mark(x.w, k0 + 2), mark(y.z, k0 + kPage), mark(y.w, k0 + kPage + 2))};
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          auto one = [&](int i) { return (p[ct][i] != 0.f ? 0x3f80u : 0u) | (p[ct][i + 1] != 0.f ? 0x3f800000u : 0u); };
          const uint4 weighs = make_uint4(one(0), one(2), one(4), one(6));
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const f32x4 n = mfma32(at[u], weighs, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int i = 0; i < 4; ++i) o[ct][2 * c + u][i] += n[i] > 0.f ? add : 0.f;
          }
        }
      }
    }
  }
};

// Takes what is not finite, and keys past the item's, out of a chunk of V^T of a page from key k0 (of this lane) on.
__device__ __forceinline__ void keep_finite(uint4& v, int k0, int keys, bool* odd) {
  v.x = keep_finite(v.x, k0, keys, odd);
  v.y = keep_finite(v.y, k0 + 2, keys, odd);
  v.z = keep_finite(v.z, k0, keys, odd);
  v.w = keep_finite(v.w, k0 + 2, keys, odd);
}

// Where a workgroup's part of the call lies.
struct TreePlace {
  TreeItem it;
  int item, h, tile, split, cols, p0, p1;  // pairs p0 .. p1 - 1
  bool none;
  bool whole;  // the item's keys are one split: results are final
};

// Workgroups go by split, item, tile of columns, head (the fastest).  Those of a head and item are close in time and, with
// eight heads, on one XCD, whose L2 then serves the second reading of a page; splits that a short item does not have
// come last: between the others they left half of the chip idle (123 items, two splits that one of them has: 325 us, in
// this order 204).
__device__ __forceinline__ TreePlace tree_place(const TreeArgs& a, int q_tiles, int pairs_per_split, int gl, int wide) {
  TreePlace w;
  int b = blockIdx.x;
  w.h = b % a.nkv;
  b /= a.nkv;
  w.tile = b % q_tiles;
  b /= q_tiles;
  w.item = b % a.items;
  w.split = b / a.items;
  w.it = tree_item(a, w.item);
  w.cols = w.it.n << gl;
  w.p0 = w.split * pairs_per_split;
  w.p1 = min(w.p0 + pairs_per_split, w.it.pairs);
  w.whole = w.it.pairs <= pairs_per_split;
  w.none = w.tile * wide >= w.cols || (w.p0 >= w.p1 && w.split > 0);
  return w;
}

// ---------------------------------------------------------------------------
// Few columns: K and V pass from memory straight into operand registers, up to two
// tiles a wave, and the waves of a workgroup take the pairs of its split in turn.
// ---------------------------------------------------------------------------
constexpr int kTreeWaves = 4;

template <int HD, int CT>
__global__ __launch_bounds__(kTreeWaves * 64) __attribute__((amdgpu_waves_per_eu(CT == 1 ? 3 : 2))) void attn_tree_kernel(
    TreeArgs a, int q_tiles, int splits, int pairs_per_split, int gl) {
  using Tiles = TreeTiles<HD, CT>;
  constexpr int KQ = Tiles::KQ, NT = Tiles::NT, NC = Tiles::NC, WP = kTreeWaves;
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const TreePlace w = tree_place(a, q_tiles, pairs_per_split, gl, 16 * CT);
  if (w.none) return;
  const TreeItem it = w.it;
  const float qscale = a.scale * kTreeLog2e;
  const int32_t* bt = a.tables + static_cast<size_t>(w.item) * a.ldb;
  const int last_page = (it.keys - 1) / kPage;
  Tiles x;
  x.start(a, it, w.h, gl, w.tile * 16 * CT, w.cols, lane);
  const size_t pstride = static_cast<size_t>(2) * a.nkv * kPage * HD;
  const uint16_t* kbase = a.kv + static_cast<size_t>(w.h) * kPage * HD;
  const uint16_t* vbase = kbase + static_cast<size_t>(a.nkv) * kPage * HD;
  uint4 kf[2][KQ], vf[2][NC];
  auto load = [&](uint4* f, const uint16_t* base, int id, int n) __attribute__((always_inline)) {
    const uint16_t* p = base + static_cast<size_t>(id) * pstride;
#pragma unroll
    for (int i = 0; i < n; ++i) f[i] = *reinterpret_cast<const uint4*>(p + 512 * i + 8 * lane);
  };
  // K of the next pair is on its way from the moment the scores are done, V of this one while they are formed: loads
  // and waits go in one order, with no branch around a load, so that each wait is for its own loads alone.
  const int np = w.p0 + wave < w.p1 ? (w.p1 - w.p0 - wave + WP - 1) / WP : 0;
  int ida = 0, idb = 0;  // lane l: page ids of the wave's pair 64 k + l
  auto page_ids = [&](int j) __attribute__((always_inline)) {
    const int p = 2 * (w.p0 + wave + WP * min(j + lane, np - 1));
    ida = min(max(bt[min(p, last_page)], 0), a.n_pages - 1);
    idb = min(max(bt[min(p + 1, last_page)], 0), a.n_pages - 1);
    asm volatile("" : "+v"(ida), "+v"(idb));
  };
  if (np > 0) {
    page_ids(0);
    load(kf[0], kbase, __builtin_amdgcn_readlane(ida, 0), KQ);
    load(kf[1], kbase, __builtin_amdgcn_readlane(idb, 0), KQ);
  }
  for (int j = 0; j < np; ++j) {
    const int k0 = 2 * kPage * (w.p0 + wave + WP * j);
    const int id0 = __builtin_amdgcn_readlane(ida, j & 63), id1 = __builtin_amdgcn_readlane(idb, j & 63);
    load(vf[0], vbase, id0, NC);
    load(vf[1], vbase, id1, NC);
    __builtin_amdgcn_sched_barrier(0);
    float s[CT][8];
    x.scores([&](int pg, int i) { return kf[pg][i]; }, s);
    if (((j + 1) & 63) == 0 && j + 1 < np) page_ids(j + 1);
    const int jn = min(j + 1, np - 1) & 63;
    load(kf[0], kbase, __builtin_amdgcn_readlane(ida, jn), KQ);
    load(kf[1], kbase, __builtin_amdgcn_readlane(idb, jn), KQ);
    __builtin_amdgcn_sched_barrier(0);
    bool odd = false;
    if (k0 + 2 * kPage > it.ctx) {  // drafted keys
      x.mask(a, it, k0, grp, s);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        keep_finite(vf[0][c], k0 + 4 * grp, it.keys, &odd);
        keep_finite(vf[1][c], k0 + kPage + 4 * grp, it.keys, &odd);
      }
      odd = __any(odd);
    }
    float e[CT][8];
    const float top = x.exponents(s, qscale, e);
    x.refer(s, qscale, top, e);
    typename Tiles::Weights weights;
    x.weigh(e, weights);
    x.add_values([&](int c, uint4& p, uint4& q) { p = vf[0][c], q = vf[1][c]; }, weights);
    if (odd)
      x.add_odd(it, vbase + static_cast<size_t>(id0) * pstride, vbase + static_cast<size_t>(id1) * pstride, k0 + 4 * grp, lane, e);
  }

  // Merge the waves in order, one tile at a time.
  __shared__ float so[WP][HD][16 + 1];
  __shared__ float sm[WP][16], sl[WP][16];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const float sum = sum_xor32(sum_xor16(x.l[ct]));
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) so[wave][16 * t + 4 * grp + i][col] = x.o[ct][t][i];
    if (grp == 0) {
      sm[wave][col] = x.m[ct];
      sl[wave][col] = sum;
    }
    __syncthreads();
    for (int idx = threadIdx.x; idx < 16 * HD; idx += WP * 64) {
      const int c = idx / HD, d = idx % HD;
      const int gc = (w.tile * CT + ct) * 16 + c;
      if (gc >= w.cols) break;
      float M = sm[0][c];
#pragma unroll
      for (int v = 1; v < WP; ++v) M = fmaxf(M, sm[v][c]);
      float L = 0.f, O = 0.f;
#pragma unroll
      for (int v = 0; v < WP; ++v) {
        const float f = exp2f(sm[v][c] - M);
        L += sl[v][c] * f;
        O += so[v][d][c] * f;
      }
      const size_t head = static_cast<size_t>(it.row0 + (gc >> gl)) * a.nq + (w.h << gl) + (gc & ((1 << gl) - 1));
      if (w.whole) {
        a.out[head * HD + d] = L == 0.f ? 0 : f32_to_bf16(O / L);
      } else {
        const size_t heads = static_cast<size_t>(a.rows) * a.nq, at = w.split * heads + head;
        a.part[at * HD + d] = O;
        if (d == 0) reinterpret_cast<float2*>(a.part + splits * heads * HD)[at] = make_float2(M, L);
      }
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Many columns: eight waves of one tile each against the same pairs, whose pages
// go through LDS in a ring of four stages by direct loads, issued three pairs ahead.
// As compiled, each turn waits before its first products until at most two or three of
// a wave's six loads under way are outstanding (the queries' loads count as pending
// through the loop), so little more than the last pair issued is on its way while one is
// used: waves wait 39 to 64% of the time.  Two such workgroups fit a CU.
// ---------------------------------------------------------------------------
constexpr int kTreeSharedWaves = 8, kTreeStages = 4;

template <int HD>
struct TreeRing {
  static constexpr int PCH = kPage * HD / 8;  // 16-byte chunks of a K (or V^T) tile
  uint4 at[kTreeStages][4][PCH];              // stage: K page 0, K page 1, V^T page 0, V^T page 1
};

// The part of a wave with a tile, or (ON false) of one that only brings its share of the pages.
template <int HD, bool ON>
__device__ __forceinline__ void tree_shared_wave(const TreeArgs& a, const TreePlace& w, TreeRing<HD>& ring, int wave, int lane,
                                                 int splits, int gl) {
  using Tiles = TreeTiles<HD, 1>;
  constexpr int NT = Tiles::NT, NC = Tiles::NC, NS = kTreeStages, NW = kTreeSharedWaves;
  constexpr int PCH = TreeRing<HD>::PCH, LPW = PCH * 4 / NW / 64;  // direct loads of a wave for a stage
  const int col = lane & 15, grp = lane >> 4;
  const TreeItem it = w.it;
  const float qscale = a.scale * kTreeLog2e;
  const int32_t* bt = a.tables + static_cast<size_t>(w.item) * a.ldb;
  const int last_page = (it.keys - 1) / kPage;
  const int col0 = (w.tile * NW + wave) * 16;
  Tiles x;
  if constexpr (ON) x.start(a, it, w.h, gl, col0, w.cols, lane);
  const size_t pstride = static_cast<size_t>(2) * a.nkv * kPage * HD;
  // NW / 4 waves bring a tile of every stage; lane l holds the page ids of pairs 64 k + l
  const int tile = wave / (NW / 4), piece = wave % (NW / 4) * LPW;
  const uint16_t* mine = a.kv + static_cast<size_t>((tile >> 1) * a.nkv + w.h) * kPage * HD + 512 * piece;
  const int n = max(w.p1 - w.p0, 0);
  int pid = 0;
  auto issue = [&](int j) __attribute__((always_inline)) {
    if ((j & 63) == 0) {
      pid = min(max(bt[min(2 * (w.p0 + j + lane) + (tile & 1), last_page)], 0), a.n_pages - 1);
      asm volatile("" : "+v"(pid));
    }
    const uint16_t* src = mine + static_cast<size_t>(__builtin_amdgcn_readlane(pid, j & 63)) * pstride;
    const uint32_t dst = lds_address(&ring.at[j % NS][tile][64 * piece]);
#pragma unroll
    for (int c = 0; c < LPW; ++c) lds_load16s(src + 512 * c, 16 * lane, dst + 1024 * c);
  };
#pragma unroll
  for (int j = 0; j < NS - 1; ++j)
    if (j < n) issue(j);
  for (int j = 0; j < n; ++j) {
    // this wave's part of pair j has landed once at most the later pairs' loads are outstanding; behind the barrier all
    // have, and the stage that was read last is free
    const int later = min(n - 1 - j, NS - 2);
    if (later >= 2) wait_vmcnt<2 * LPW>();
    else if (later == 1) wait_vmcnt<LPW>();
    else wait_vmcnt<0>();
    lds_barrier();
    if (j + NS - 1 < n) issue(j + NS - 1);
    if constexpr (ON) {
      const uint4(*st)[PCH] = ring.at[j % NS];
      const int k0 = 2 * kPage * (w.p0 + j);
      float s[1][8], e[1][8];
      typename Tiles::Weights weights;
      x.scores([&](int pg, int i) { return st[pg][64 * i + lane]; }, s);
      if (k0 + 2 * kPage > it.ctx) x.mask(a, it, k0, grp, s);  // drafted keys
      const float top = x.exponents(s, qscale, e);
      x.refer(s, qscale, top, e);
      x.weigh(e, weights);
      if (k0 + 2 * kPage > it.ctx) {
        bool odd = false;
        x.add_values(
            [&](int c, uint4& p, uint4& q) {
              p = st[2][64 * c + lane], q = st[3][64 * c + lane];
              keep_finite(p, k0 + 4 * grp, it.keys, &odd);
              keep_finite(q, k0 + kPage + 4 * grp, it.keys, &odd);
            },
            weights);
        if (__any(odd)) {
          const uint16_t* vbase = a.kv + static_cast<size_t>(a.nkv + w.h) * kPage * HD;
          const int i0 = min(max(bt[min(k0 / kPage, last_page)], 0), a.n_pages - 1);
          const int i1 = min(max(bt[min(k0 / kPage + 1, last_page)], 0), a.n_pages - 1);
          x.add_odd(it, vbase + static_cast<size_t>(i0) * pstride, vbase + static_cast<size_t>(i1) * pstride, k0 + 4 * grp, lane, e);
        }
      } else {
        x.add_values([&](int c, uint4& p, uint4& q) { p = st[2][64 * c + lane], q = st[3][64 * c + lane]; }, weights);
      }
    }
  }
  if constexpr (ON) {
    const float L = sum_xor32(sum_xor16(x.l[0]));
    const int c = col0 + col;
    if (c >= w.cols) return;
    const size_t head = static_cast<size_t>(it.row0 + x.tok[0]) * a.nq + (w.h << gl) + (c & ((1 << gl) - 1));
    if (w.whole) {
      const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        uint2 v;
        v.x = pack_bf16x2(x.o[0][t][0] * inv, x.o[0][t][1] * inv);
        v.y = pack_bf16x2(x.o[0][t][2] * inv, x.o[0][t][3] * inv);
        *reinterpret_cast<uint2*>(a.out + head * HD + 16 * t + 4 * grp) = v;
      }
    } else {
      const size_t heads = static_cast<size_t>(a.rows) * a.nq, at = w.split * heads + head;
#pragma unroll
      for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4*>(a.part + at * HD + 16 * t + 4 * grp) = x.o[0][t];
      if (grp == 0) reinterpret_cast<float2*>(a.part + splits * heads * HD)[at] = make_float2(x.m[0], L);
    }
  }
}

template <int HD>
__global__ __launch_bounds__(kTreeSharedWaves * 64, 4) void attn_tree_shared_kernel(TreeArgs a, int q_tiles, int splits,
                                                                                    int pairs_per_split, int gl) {
  __shared__ TreeRing<HD> ring;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const TreePlace w = tree_place(a, q_tiles, pairs_per_split, gl, 16 * kTreeSharedWaves);
  if (w.none) return;
  if ((w.tile * kTreeSharedWaves + wave) * 16 < w.cols)
    tree_shared_wave<HD, true>(a, w, ring, wave, lane, splits, gl);
  else
    tree_shared_wave<HD, false>(a, w, ring, wave, lane, splits, gl);
}

// The splits of the items that have several, a workgroup for four heads of a query, a wave for each: lane l brings split l's
// maximum and sum, then each HD / 4 lanes add up the outputs of every PER-th split (four values a lane), and those
// sums are added in order.
template <int HD>
__global__ __launch_bounds__(256) void attn_tree_combine_kernel(TreeArgs a, int splits, int pairs_per_split) {
  constexpr int LN = HD / 4, PER = 64 / LN;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int item = blockIdx.x % a.items, tok = blockIdx.x / a.items;
  const TreeItem it = tree_item(a, item);
  const int ns = (it.pairs + pairs_per_split - 1) / pairs_per_split;
  if (tok >= it.n || ns <= 1) return;
  const size_t heads = static_cast<size_t>(a.rows) * a.nq;
  if (const int j = blockIdx.y * 4 + wave; j < a.nq) {
    const size_t head = static_cast<size_t>(it.row0 + tok) * a.nq + j;
    const float2 mine = reinterpret_cast<const float2*>(a.part + splits * heads * HD)[min(lane, ns - 1) * heads + head];
    const float M = wave_max(mine.x);
    const float f = exp2f(mine.x - M);
    const float L = wave_sum(lane < ns ? mine.y * f : 0.f);
    const float4* po = reinterpret_cast<const float4*>(a.part + head * HD) + lane % LN;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int s0 = 0; s0 < ns; s0 += PER) {  // (all lanes go through it: each reads another's f)
      const int s = min(s0 + lane / LN, ns - 1);
      const float4 v = po[s * heads * LN];
      const float w = __shfl(f, s, kWave);
      if (s0 + lane / LN >= ns) continue;
      o.x += v.x * w;
      o.y += v.y * w;
      o.z += v.z * w;
      o.w += v.w * w;
    }
#pragma unroll
    for (int x = LN; x < 64; x <<= 1) {
      o.x += __shfl_xor(o.x, x, kWave);
      o.y += __shfl_xor(o.y, x, kWave);
      o.z += __shfl_xor(o.z, x, kWave);
      o.w += __shfl_xor(o.w, x, kWave);
    }
    if (lane >= LN) return;
    const float inv = L == 0.f ? 0.f : 1.f / L;
    uint2 w;
    w.x = pack_bf16x2(o.x * inv, o.y * inv);
    w.y = pack_bf16x2(o.z * inv, o.w * inv);
    *reinterpret_cast<uint2*>(a.out + head * HD + 4 * lane) = w;
  }
}

// The same for many queries of few splits: a workgroup for each query, a thread for 16 values of a head, so that one
// round of loads serves all heads.
template <int HD>
__global__ __launch_bounds__(256) void attn_tree_combine_many_kernel(TreeArgs a, int splits, int pairs_per_split) {
  constexpr int PH = HD / 16;  // threads of a head
  const int item = blockIdx.x % a.items, tok = blockIdx.x / a.items;
  const TreeItem it = tree_item(a, item);
  const int ns = (it.pairs + pairs_per_split - 1) / pairs_per_split;
  if (tok >= it.n || ns <= 1) return;
  const size_t heads = static_cast<size_t>(a.rows) * a.nq;
  for (int unit = threadIdx.x; unit < a.nq * PH; unit += 256) {
    const size_t head = static_cast<size_t>(it.row0 + tok) * a.nq + unit / PH;
    const float2* ml = reinterpret_cast<const float2*>(a.part + splits * heads * HD) + head;
    const float4* po = reinterpret_cast<const float4*>(a.part + head * HD) + unit % PH * 4;
    float M = kTreeNone;
#pragma unroll 4
    for (int s = 0; s < ns; ++s) M = fmaxf(M, ml[s * heads].x);
    float L = 0.f;
    float4 o[4] = {};
#pragma unroll 2
    for (int s = 0; s < ns; ++s) {
      const float2 v = ml[s * heads];
      const float f = exp2f(v.x - M);
      L += v.y * f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 w = po[s * heads * (HD / 4) + i];
        o[i].x += w.x * f;
        o[i].y += w.y * f;
        o[i].z += w.z * f;
        o[i].w += w.w * f;
      }
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    uint4* out = reinterpret_cast<uint4*>(a.out + head * HD + unit % PH * 16);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      out[i] = make_uint4(pack_bf16x2(o[2 * i].x * inv, o[2 * i].y * inv), pack_bf16x2(o[2 * i].z * inv, o[2 * i].w * inv),
                          pack_bf16x2(o[2 * i + 1].x * inv, o[2 * i + 1].y * inv), pack_bf16x2(o[2 * i + 1].z * inv, o[2 * i + 1].w * inv));
  }
}

// Up to 32 columns an item: the kernel through registers, one or two tiles a wave; more: the shared one.  A split has
// to be worth its states (a column's is 520 bytes written and read again, a pair of pages 16 KiB): at least an eighth
// of its columns in pairs, and four.  More splits are made while max_keys would leave fewer than `full` workgroups; the
// items are often shorter than it, hence some times the 256 CUs, and where the items alone are more than fit the chip at
// once, the longest of them must not outlast the others.  Measured (us; heads 32 over 8 of 128 but for the 64 tokens'):
// 25 single tokens after 256 .. 4096 keys, full 1024 / 2048 / 4096: 36.0 / 33.1 / 36.7; 123 of them 152 / 142 / 140; 25
// trees of 9 .. 17 tokens 43 / 50 / 54; 123 of 8 .. 32 224 / 204 / 202; two of 57 .. 64 after 20000 .. 30000 keys, 64 heads
// over 8, 194 .. 207 / 202 .. 207 / 227 .. 234.
TreePlan plan_attn_tree(int nq, int nkv, int hd, int items, int rows, int max_q, int max_keys, int64_t part_floats) {
  const int cols = max_q * (nq / nkv);
  TreePlan p;
  p.wide = cols <= 16 ? 16 : cols <= 32 ? 32 : 16 * kTreeSharedWaves;
  p.tiles = (cols + p.wide - 1) / p.wide;
  const int64_t groups = static_cast<int64_t>(items) * nkv * p.tiles;
  const int full = cols <= 16 || (cols > 32 && groups > 512) ? 2048 : 1024;
  const int pairs = max_keys / (2 * kPage) + (max_keys % (2 * kPage) ? 1 : 0);
  int64_t most = part_floats / (static_cast<int64_t>(rows) * nq * (hd + 2));  // splits whose states fit
  if (most > kTreeMaxSplits) most = kTreeMaxSplits;
  if (most < 1) most = 1;
  int64_t per = (pairs * groups + full - 1) / full;
  const int least = (cols < p.wide ? cols : p.wide) / 8;
  if (per < least) per = least;
  if (per < 4) per = 4;
  if (per * most < pairs) per = (pairs + most - 1) / most;
  p.pairs = static_cast<int>(per < pairs ? per : pairs);
  p.splits = (pairs + p.pairs - 1) / p.pairs;
  return p;
}

template <int HD>
static hipError_t launch_tree_hd(const TreeArgs& a, const TreePlan& p, hipStream_t s) {
  const int gl = __builtin_ctz(a.nq / a.nkv);
  const dim3 grid(a.items * p.splits * p.tiles * a.nkv);
  if (p.wide == 16)
    launch_kernel((attn_tree_kernel<HD, 1>), grid, dim3(kTreeWaves * 64), 0, s, a, p.tiles, p.splits, p.pairs, gl);
  else if (p.wide == 32)
    launch_kernel((attn_tree_kernel<HD, 2>), grid, dim3(kTreeWaves * 64), 0, s, a, p.tiles, p.splits, p.pairs, gl);
  else
    launch_kernel((attn_tree_shared_kernel<HD>), grid, dim3(kTreeSharedWaves * 64), 0, s, a, p.tiles, p.splits, p.pairs, gl);
  if (p.splits > 1) {
    // a head a wave while that leaves at most 4096 workgroups
    const int64_t queries = static_cast<int64_t>(a.items) * a.max_q;
    const int nb = (a.nq + 3) / 4;
    if (queries * nb <= 4096)
      launch_kernel((attn_tree_combine_kernel<HD>), dim3(queries, nb), dim3(256), 0, s, a, p.splits, p.pairs);
    else
      launch_kernel((attn_tree_combine_many_kernel<HD>), dim3(queries), dim3(256), 0, s, a, p.splits, p.pairs);
  }
  return hipGetLastError();
}

hipError_t launch_attn_tree(const TreeArgs& a, hipStream_t s) {
  if (a.items <= 0 || a.rows <= 0) return hipSuccess;
  const TreePlan p = plan_attn_tree(a.nq, a.nkv, a.hd, a.items, a.rows, a.max_q, a.max_keys, a.part_floats);
  return a.hd == 128 ? launch_tree_hd<128>(a, p, s) : launch_tree_hd<64>(a, p, s);
}

}  // namespace metro
