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
// all in fp32, and rounded to bf16 once.  v is rounded as it is.  One wave per
// (row, head); lane j < hd/2 takes the pair (j, j + hd/2).
// ---------------------------------------------------------------------------
template <bool F32>
__global__ __launch_bounds__(64) void rope_append_kernel(AppendArgs a) {
  const int nh = a.nq + 2 * a.nkv, hd = a.hd, half = hd / 2;
  const int t = blockIdx.x / nh, head = blockIdx.x % nh;
  const int j = threadIdx.x;
  const bool on = j < half;
  const size_t at = static_cast<size_t>(t) * a.ld + head * hd;
  float x = 0.f, y = 0.f;
  if (on) {
    x = F32 ? a.y32[at + j] : bf16_to_f32(a.y16[at + j]);
    y = F32 ? a.y32[at + j + half] : bf16_to_f32(a.y16[at + j + half]);
  }
  const int sl = a.slot[t];
  const bool cached = sl >= 0 && sl / kPage < a.n_pages;
  if (head >= a.nq + a.nkv) {
    if (!cached || !on) return;
    uint16_t* vt = a.kv + kv_offset(sl / kPage, 1, a.nkv, head - a.nq - a.nkv, 0, hd, 0);
    vt[vt_tile_offset(j, sl % kPage)] = f32_to_bf16(x);
    vt[vt_tile_offset(j + half, sl % kPage)] = f32_to_bf16(y);
    return;
  }
  const uint16_t* gain = head < a.nq ? a.q_gain : a.k_gain;
  if (gain) {
    const float inv = rsqrtf(wave_sum(x * x + y * y) / static_cast<float>(hd) + a.eps);
    if (on) {
      x = x * inv * bf16_to_f32(gain[j]);
      y = y * inv * bf16_to_f32(gain[j + half]);
    }
  }
  if (!on) return;
  const int p = a.pos[t];
  const float nan = __builtin_nanf("");
  const float2 c = p >= 0 && p < a.n_pos ? a.rope[static_cast<size_t>(p) * half + j] : make_float2(nan, nan);
  const uint16_t ra = f32_to_bf16(x * c.x - y * c.y), rb = f32_to_bf16(x * c.y + y * c.x);
  if (head < a.nq) {
    uint16_t* dst = a.q + (static_cast<size_t>(t) * a.nq + head) * hd;
    dst[j] = ra;
    dst[j + half] = rb;
  } else if (cached) {
    uint16_t* kt = a.kv + kv_offset(sl / kPage, 0, a.nkv, head - a.nq, 0, hd, 0);
    kt[k_tile_offset(sl % kPage, j)] = ra;
    kt[k_tile_offset(sl % kPage, j + half)] = rb;
  }
}

hipError_t launch_rope_append(const AppendArgs& a, hipStream_t s) {
  if (a.T <= 0) return hipSuccess;
  const dim3 grid(a.T * (a.nq + 2 * a.nkv));
  if (a.y32)
    launch_kernel(rope_append_kernel<true>, grid, dim3(64), 0, s, a);
  else
    launch_kernel(rope_append_kernel<false>, grid, dim3(64), 0, s, a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Move.  A thread owns one 16-byte chunk of the K tile (8 dims of a key) or one
// of the V^T tile (a key's two values there) for all moves of a group: it reads
// the chunk at every source before it writes the first destination, and writes
// in the list's order, so no other thread can come between and no barrier is
// needed.  Grid: (chunks of a layer's heads, layers, groups).
// ---------------------------------------------------------------------------
template <bool V>
__device__ __forceinline__ void move_chunk(const MoveArgs& a, uint16_t* base, int unit, int lo, int hi) {
  const int per_head = V ? a.hd / 2 : a.hd / 8;  // chunks of a key in a tile
  const int h = unit / per_head, c = unit % per_head;
  const int slots = a.n_pages * kPage;
  auto where = [&](int slot) {
    const int key = slot % kPage;
    const int in = V ? (((c >> 4) * 4 + (key >> 2)) * 16 + (c & 15)) * 8 + (key & 3) : (c * 16 + key) * 8;
    return base + kv_offset(slot / kPage, V ? 1 : 0, a.nkv, h, 0, a.hd, 0) + in;
  };
  for (int m0 = lo; m0 < hi; m0 += kMoveRun) {
    const int n = min(kMoveRun, hi - m0);
    uint4 k[V ? 1 : kMoveRun];
    uint32_t v[V ? kMoveRun : 1];
#pragma unroll
    for (int m = 0; m < kMoveRun; ++m) {
      if (m >= n) continue;
      const int s = min(max(a.src[m0 + m], 0), slots - 1);
      if constexpr (V)
        v[m] = where(s)[0] | (static_cast<uint32_t>(where(s)[4]) << 16);
      else
        k[m] = *reinterpret_cast<const uint4*>(where(s));
    }
#pragma unroll
    for (int m = 0; m < kMoveRun; ++m) {
      if (m >= n) continue;
      const int s = a.src[m0 + m], d = a.dst[m0 + m];
      if (s == d || s < 0 || s >= slots || d < 0 || d >= slots) continue;
      uint16_t* to = where(d);
      if constexpr (V) {
        to[0] = static_cast<uint16_t>(v[m]);
        to[4] = static_cast<uint16_t>(v[m] >> 16);
      } else {
        *reinterpret_cast<uint4*>(to) = k[m];
      }
    }
  }
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
