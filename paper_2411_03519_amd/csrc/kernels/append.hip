// Rows into the paged KV cache (gfx950, wave64): the per-head norm, the rotation
// and the write of a QKV product's rows, and the move of keys and values between
// slots of the cache.
#include "common.h"
#include "kernels.h"
#include "kernels_draft.h"

namespace metro {

// ---------------------------------------------------------------------------
// Append.  y = one head of a row; q and k heads with a gain are normalised,
//   y <- y / sqrt(mean(y^2) + eps) * g,
// then turned by pairs (i, i + hd/2) with the position's (cos, sin):
//   (a, b) -> (a c - b s, a s + b c),
// all in fp32, and rounded to bf16 once.  v is rounded as it is.
//
// A wave takes RW = 8 (16 for head dim 64) rows; a lane has 8 pairs of one row,
// with their cosines and sines in registers for all heads that the wave goes
// through, the next head's values on their way.  Queries and keys leave as 16-byte
// stores (a K tile's chunk is 8 dims of one key, those of consecutive keys lie side
// by side).  A V^T tile holds 4 keys of a dim together, so values are taken four
// rows at a time where the rows' slots are four such keys, whatever row they begin
// at, and one by one elsewhere.
//
// Bound by memory: 8180 rows of 48 heads of 128 in fp32, with norms, 306 MB in 71 us
// (4.3 TB/s, a third of it writes), a wave a (row, head) with 2-byte stores 124; 336
// drafts' rows in bf16 5.9 us, one row 2.9, which is a launch.
// ---------------------------------------------------------------------------
template <bool F32>
__device__ __forceinline__ void load8(const AppendArgs& a, size_t at, float (&x)[8]) {
  if constexpr (F32) {
    const float4 u = *reinterpret_cast<const float4*>(a.y32 + at), v = *reinterpret_cast<const float4*>(a.y32 + at + 4);
    x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
  } else {
    const uint4 u = *reinterpret_cast<const uint4*>(a.y16 + at);
    x[0] = lo_bf16(u.x), x[1] = hi_bf16(u.x), x[2] = lo_bf16(u.y), x[3] = hi_bf16(u.y);
    x[4] = lo_bf16(u.z), x[5] = hi_bf16(u.z), x[6] = lo_bf16(u.w), x[7] = hi_bf16(u.w);
  }
}

template <bool F32>
__device__ __forceinline__ float4 load4(const AppendArgs& a, size_t at) {
  if constexpr (F32) return *reinterpret_cast<const float4*>(a.y32 + at);
  const uint2 u = *reinterpret_cast<const uint2*>(a.y16 + at);
  return make_float4(lo_bf16(u.x), hi_bf16(u.x), lo_bf16(u.y), hi_bf16(u.y));
}

__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

__device__ __forceinline__ void times8(float (&x)[8], float s, uint4 g) {
  x[0] *= s * lo_bf16(g.x), x[1] *= s * hi_bf16(g.x), x[2] *= s * lo_bf16(g.y), x[3] *= s * hi_bf16(g.y);
  x[4] *= s * lo_bf16(g.z), x[5] *= s * hi_bf16(g.z), x[6] *= s * lo_bf16(g.w), x[7] *= s * hi_bf16(g.w);
}

template <int HD, bool F32>
__global__ __launch_bounds__(256) void rope_append_kernel(AppendArgs a, int slices) {
  constexpr int HALF = HD / 2, LPR = HALF / 8, RW = 64 / LPR;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t0 = blockIdx.x / slices * RW, first = blockIdx.x % slices * 4 + wave, step = 4 * slices;
  const int n_slots = a.n_pages * kPage, turned = a.nq + a.nkv, heads = turned + a.nkv;

  int h = first;
  if (h < turned) {
    const int t = t0 + lane / LPR, d = lane % LPR * 8;
    const bool on = t < a.T;
    const int row = on ? t : a.T - 1;
    const size_t at = static_cast<size_t>(row) * a.ld + d;
    float x[8], y[8];
    load8<F32>(a, at + static_cast<size_t>(h) * HD, x);
    load8<F32>(a, at + static_cast<size_t>(h) * HD + HALF, y);
    const int p = a.pos[row], slot = a.slot[row];
    const bool cached = on && slot >= 0 && slot < n_slots;
    float c[8], s[8];
    const float4* cs = reinterpret_cast<const float4*>(a.rope + static_cast<size_t>(min(max(p, 0), a.n_pos - 1)) * HALF + d);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 v = cs[i];
      c[2 * i] = v.x, s[2 * i] = v.y, c[2 * i + 1] = v.z, s[2 * i + 1] = v.w;
    }
    if (p < 0 || p >= a.n_pos)
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] = s[i] = __builtin_nanf("");
    const uint4 none = make_uint4(0, 0, 0, 0);
    const uint4 qg0 = a.q_gain ? *reinterpret_cast<const uint4*>(a.q_gain + d) : none;
    const uint4 qg1 = a.q_gain ? *reinterpret_cast<const uint4*>(a.q_gain + d + HALF) : none;
    const uint4 kg0 = a.k_gain ? *reinterpret_cast<const uint4*>(a.k_gain + d) : none;
    const uint4 kg1 = a.k_gain ? *reinterpret_cast<const uint4*>(a.k_gain + d + HALF) : none;
    uint16_t* ktile = a.kv + kv_offset(cached ? slot / kPage : 0, 0, a.nkv, 0, 0, HD, 0) + (d / 8 * kPage + (cached ? slot % kPage : 0)) * 8;
    uint16_t* qrow = a.q + static_cast<size_t>(row) * a.nq * HD + d;
    for (; h < turned; h += step) {
      float nx[8], ny[8];
      const int hn = min(h + step, turned - 1);
      load8<F32>(a, at + static_cast<size_t>(hn) * HD, nx);
      load8<F32>(a, at + static_cast<size_t>(hn) * HD + HALF, ny);
      const bool is_q = h < a.nq;
      if (is_q ? a.q_gain != nullptr : a.k_gain != nullptr) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss += x[i] * x[i] + y[i] * y[i];
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) ss += __shfl_xor(ss, o, kWave);
        const float inv = rsqrtf(ss * (1.f / HD) + a.eps);
        times8(x, inv, is_q ? qg0 : kg0);
        times8(y, inv, is_q ? qg1 : kg1);
      }
      float u[8], v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        u[i] = x[i] * c[i] - y[i] * s[i];
        v[i] = x[i] * s[i] + y[i] * c[i];
      }
      if (is_q) {
        if (on) {
          *reinterpret_cast<uint4*>(qrow + h * HD) = pack8(u);
          *reinterpret_cast<uint4*>(qrow + h * HD + HALF) = pack8(v);
        }
      } else if (cached) {
        uint16_t* k = ktile + static_cast<size_t>(h - a.nq) * kPage * HD;
        *reinterpret_cast<uint4*>(k) = pack8(u);
        *reinterpret_cast<uint4*>(k + HALF / 8 * kPage * 8) = pack8(v);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = nx[i], y[i] = ny[i];
    }
  }
  if (h >= heads) return;

  // Which rows begin four keys of a tile that follow one another (lane i: row t0 - 3 + i; the first three rows may be
  // taken along by such a one before them).
  bool leads = false;
  bool stored = false;
  if (const int t = t0 - 3 + lane; lane < RW + 3 && t >= 0 && t < a.T) {
    const int s0 = a.slot[t];
    stored = s0 >= 0 && s0 < n_slots;
    if (stored && s0 % 4 == 0 && t + 3 < a.T) leads = a.slot[t + 1] == s0 + 1 && a.slot[t + 2] == s0 + 2 && a.slot[t + 3] == s0 + 3;
  }
  const uint64_t lead = __ballot(leads);
  const uint64_t own = lead >> 3, taken = (lead | lead << 1 | lead << 2 | lead << 3) >> 3;
  const uint32_t alone = static_cast<uint32_t>((__ballot(stored) >> 3) & ~taken) & ((1u << RW) - 1);
  constexpr int LPV = HD / 4;  // lanes of a row of values, four dims each
  const int d = lane % LPV * 4;
  // this lane's quad: the (lane / LPV)-th of the wave's (at most RW / 4 begin within RW rows)
  uint32_t bits = static_cast<uint32_t>(own) & ((1u << RW) - 1);
  for (int k = 0; k < lane / LPV; ++k) bits &= bits - 1;
  const bool quad = bits != 0;
  const int tq = t0 + (quad ? __ffs(static_cast<int>(bits)) - 1 : 0);
  for (; h < heads; h += step) {
    const int head = h - turned;
    if (quad) {
      const size_t at = static_cast<size_t>(tq) * a.ld + static_cast<size_t>(h) * HD + d;
      const float4 r0 = load4<F32>(a, at), r1 = load4<F32>(a, at + a.ld), r2 = load4<F32>(a, at + 2 * static_cast<size_t>(a.ld)),
                   r3 = load4<F32>(a, at + 3 * static_cast<size_t>(a.ld));
      const int slot = a.slot[tq];
      uint16_t* vt = a.kv + kv_offset(slot / kPage, 1, a.nkv, head, 0, HD, 0) + vt_tile_offset(d, slot % kPage);
      *reinterpret_cast<uint2*>(vt) = make_uint2(pack_bf16x2(r0.x, r1.x), pack_bf16x2(r2.x, r3.x));
      *reinterpret_cast<uint2*>(vt + 8) = make_uint2(pack_bf16x2(r0.y, r1.y), pack_bf16x2(r2.y, r3.y));
      *reinterpret_cast<uint2*>(vt + 16) = make_uint2(pack_bf16x2(r0.z, r1.z), pack_bf16x2(r2.z, r3.z));
      *reinterpret_cast<uint2*>(vt + 24) = make_uint2(pack_bf16x2(r0.w, r1.w), pack_bf16x2(r2.w, r3.w));
    }
    // one by one: each LPV lanes take another of these rows
    uint32_t rest = alone;
    for (int k = 0; k < lane / LPV; ++k) rest &= rest - 1;
    while (rest) {
      const int t = t0 + __ffs(static_cast<int>(rest)) - 1, slot = a.slot[t];
      const float4 r = load4<F32>(a, static_cast<size_t>(t) * a.ld + static_cast<size_t>(h) * HD + d);
      uint16_t* vt = a.kv + kv_offset(slot / kPage, 1, a.nkv, head, 0, HD, 0) + vt_tile_offset(d, slot % kPage);
      vt[0] = f32_to_bf16(r.x);
      vt[8] = f32_to_bf16(r.y);
      vt[16] = f32_to_bf16(r.z);
      vt[24] = f32_to_bf16(r.w);
      for (int k = 0; k < 64 / LPV; ++k) rest &= rest - 1;
    }
  }
}

hipError_t launch_rope_append(const AppendArgs& a, hipStream_t s) {
  if (a.T <= 0) return hipSuccess;
  const int rows = a.hd == 128 ? 8 : 16, blocks = (a.T + rows - 1) / rows, heads = a.nq + 2 * a.nkv;
  // few rows: their heads over more workgroups, down to one a wave
  int slices = 1;
  while (slices < (heads + 3) / 4 && static_cast<int64_t>(blocks) * slices < 1024) ++slices;
  const dim3 grid(blocks * slices);
  if (a.hd == 128) {
    if (a.y32) launch_kernel((rope_append_kernel<128, true>), grid, dim3(256), 0, s, a, slices);
    else launch_kernel((rope_append_kernel<128, false>), grid, dim3(256), 0, s, a, slices);
  } else {
    if (a.y32) launch_kernel((rope_append_kernel<64, true>), grid, dim3(256), 0, s, a, slices);
    else launch_kernel((rope_append_kernel<64, false>), grid, dim3(256), 0, s, a, slices);
  }
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Move.  A thread owns one 16-byte chunk of the K tile (8 dims of a key) or one
// of the V^T tile (a key's two values there) for all moves of a group: eight moves
// at a time, it reads the chunk at every source before it writes the first
// destination, and writes in the list's order, so no other thread can come between
// and no barrier is needed.  Grid: (chunks of a layer's heads, layers, groups).  A key's
// 256 bytes of K lie in 16 lines, those of V as 2-byte values in the 1 KiB that its
// four keys share, so 107 moves in 32 layers of 8 heads fetch 65 MB and write 18 for 14
// and 14.  Bound by latency rather than by those (16 us at a copy's rate): the compiler
// waits for a move's slot, and so for the chunk before it, ahead of each load, and holds
// the eight chunks in 204 registers, two waves a SIMD (26 us, waves waiting 83% of the
// time; one sequence's 3 moves 3.6 us).
// ---------------------------------------------------------------------------
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <bool V>
__device__ __forceinline__ void move_run(const MoveArgs& a, uint16_t* layer, uint32_t own, int lo, int n) {
  const int slots = a.n_pages * kPage;
  const size_t page = static_cast<size_t>(2) * a.nkv * kPage * a.hd;
  // own: the thread's chunk in a page; the key's place in it is the same for all threads
  auto where = [&](int slot) __attribute__((always_inline)) {
    const uint32_t key = static_cast<uint32_t>(slot) % kPage;
    return layer + (static_cast<uint32_t>(slot) / kPage * page + (V ? key / 4 * 128 + key % 4 : key * 8)) + own;
  };
  u32x4 k[V ? 1 : kMoveRun];
  uint32_t v[V ? kMoveRun : 1];
#pragma unroll
  for (int m = 0; m < kMoveRun; ++m)
    if (m < n) {
      const uint16_t* from = where(min(max(a.src[lo + m], 0), slots - 1));
      if constexpr (V) v[m] = from[0] | (static_cast<uint32_t>(from[4]) << 16);
      else k[m] = *reinterpret_cast<const u32x4*>(from);
    }
#pragma unroll
  for (int m = 0; m < kMoveRun; ++m)
    if (m < n) {
      const int s = a.src[lo + m], d = a.dst[lo + m];
      if (s != d && s >= 0 && s < slots && d >= 0 && d < slots) {
        uint16_t* to = where(d);
        if constexpr (V) {
          to[0] = static_cast<uint16_t>(v[m]);
          to[4] = static_cast<uint16_t>(v[m] >> 16);
        } else {
          *reinterpret_cast<u32x4*>(to) = k[m];
        }
      }
    }
}

template <bool V>
__device__ __forceinline__ void move_chunk(const MoveArgs& a, uint16_t* layer, int unit, int lo, int hi) {
  const int per_head = V ? a.hd / 2 : a.hd / 8;  // chunks of a key in a tile; one of V^T holds dims d and d + 16 of four keys
  const uint32_t h = unit / per_head, c = unit % per_head;
  const uint32_t own = ((V ? a.nkv : 0) + h) * kPage * a.hd + (V ? c / 16 * 512 + c % 16 * 8 : c * 128);
#pragma unroll 1
  for (int m = lo; m < hi; m += kMoveRun) move_run<V>(a, layer, own, m, min(kMoveRun, hi - m));
}

__global__ __launch_bounds__(128) void kv_move_kernel(MoveArgs a) {
  const int lo = max(a.offsets[blockIdx.z], 0), hi = min(a.offsets[blockIdx.z + 1], a.moves);
  uint16_t* base = a.kv + static_cast<size_t>(blockIdx.y) * a.layer_stride;
  const int v_units = a.nkv * a.hd / 2, units = v_units + a.nkv * a.hd / 8;
  const int unit = blockIdx.x * 128 + threadIdx.x;
  if (unit < v_units)
    move_chunk<true>(a, base, unit, lo, hi);
  else if (unit < units)
    move_chunk<false>(a, base, unit - v_units, lo, hi);
}

hipError_t launch_kv_move(const MoveArgs& a, hipStream_t s) {
  if (a.groups <= 0 || a.moves <= 0 || a.layers <= 0) return hipSuccess;
  const int units = a.nkv * a.hd / 2 + a.nkv * a.hd / 8;
  launch_kernel(kv_move_kernel, dim3((units + 127) / 128, a.layers, a.groups), dim3(128), 0, s, a);
  return hipGetLastError();
}

}  // namespace metro
