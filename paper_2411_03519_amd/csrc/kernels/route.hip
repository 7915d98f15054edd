// Routing of tokens to experts (gfx950, wave64): scores, grouped top-k, weights,
// and the places of the tokens' rows in the experts' order.
//
// s = softmax or sigmoid of a token's logits, c = s + bias; of `groups` equal
// runs of experts the top_groups with the largest sum of their two best open c stay;
// of their experts the k largest c are chosen, ties to the lowest index; weights
// are their s (over their sum).  Scores are computed in fp64: which of two
// experts comes first must not hang on the rounding of an exponential.  An expert
// whose bias is -inf is chosen only where too few others are left, and weighs 0.
//
// Bytes are few (31527 tokens of 128 experts: 20 MB, 4 us at the rate of a copy), and
// the vector ALU bounds it: 25 us there for the choices, in which the k largest, the
// groups and the exponentials have about equal parts, and 5 each for the scan and the
// places, mostly launches.  Up to 64 tokens one workgroup does everything in one
// launch, 3.5 us for 25 tokens of 8 experts, since a second launch costs as much again.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "common.h"
#include "kernels_fp8.h"

namespace metro {

namespace {

// v of another lane of the same 16 (DPP control word), both halves of the double
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_mov_dpp(static_cast<int>(u), CTRL, 0xf, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_mov_dpp(static_cast<int>(u >> 32), CTRL, 0xf, 0xf, true);
  return __builtin_bit_cast(double, (static_cast<uint64_t>(hi) << 32) | lo);
}

// op over the LPT lanes of a token, the result in each of them: pairs, quads,
// 8 (the mirrored half row), 16 (the mirrored row), then the row swaps.
template <int LPT, class Op>
__device__ __forceinline__ double lanes_reduce(double v, Op op) {
  v = op(v, dpp<0xB1>(v));   // quad_perm 1 0 3 2
  v = op(v, dpp<0x4E>(v));   // quad_perm 2 3 0 1
  v = op(v, dpp<0x141>(v));  // row_half_mirror
  if (LPT >= 16) v = op(v, dpp<0x140>(v));  // row_mirror
  if (LPT >= 32) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = static_cast<uint32_t>(u), hi = static_cast<uint32_t>(u >> 32);
    const auto a = __builtin_amdgcn_permlane16_swap(lo, lo, false, false);
    const auto b = __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
    v = op(__builtin_bit_cast(double, (static_cast<uint64_t>(b[0]) << 32) | a[0]),
           __builtin_bit_cast(double, (static_cast<uint64_t>(b[1]) << 32) | a[1]));
  }
  if (LPT >= 64) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = static_cast<uint32_t>(u), hi = static_cast<uint32_t>(u >> 32);
    const auto a = __builtin_amdgcn_permlane32_swap(lo, lo, false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(hi, hi, false, false);
    v = op(__builtin_bit_cast(double, (static_cast<uint64_t>(b[0]) << 32) | a[0]),
           __builtin_bit_cast(double, (static_cast<uint64_t>(b[1]) << 32) | a[1]));
  }
  return v;
}

// the largest over the LPT lanes of a token
template <int LPT>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
  v = max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0xB1, 0xf, 0xf, true)));
  v = max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0x4E, 0xf, 0xf, true)));
  v = max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0x141, 0xf, 0xf, true)));
  if (LPT >= 16) v = max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0x140, 0xf, 0xf, true)));
  if (LPT >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max(r[0], r[1]);
  }
  if (LPT >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = max(r[0], r[1]);
  }
  return v;
}

constexpr double kNone = __builtin_nan("");  // an expert that can no longer be chosen

// a score to choose by: a NaN comes behind every number
__device__ __forceinline__ double choosable(double c) { return c == c ? c : -__builtin_inf(); }

// Order of the wave's own LDS accesses (which the hardware keeps) for the compiler.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Scores and choices of the token of this lane's LPT lanes (lane l of them has
// experts l, l + LPT, ...), t < T valid.  room: LDS of the token, E + groups
// doubles (used with groups > 1, by the token's own lanes only).  mask: LDS bit
// sets of the block's tokens, one per expert; bit: the token's.  Every lane of
// the wave calls it.  z: the logits of its experts, -inf behind the last.
template <int LPT, int EPL>
__device__ __forceinline__ void route_token(const RouteArgs& a, const float (&z)[EPL], int64_t t, bool valid, int l,
                                            double* room, unsigned long long* mask, int bit) {
  double s[EPL], c[EPL];
  int place[EPL];
  auto mx = [](double x, double y) { return fmax(x, y); };
  auto add = [](double x, double y) { return x + y; };
#pragma unroll
  for (int q = 0; q < EPL; ++q) place[q] = -1;
  if (a.sigmoid) {
#pragma unroll
    for (int q = 0; q < EPL; ++q) s[q] = 1.0 / (1.0 + exp(-static_cast<double>(z[q])));
  } else {
    double m = z[0];
#pragma unroll
    for (int q = 1; q < EPL; ++q) m = fmax(m, static_cast<double>(z[q]));
    m = lanes_reduce<LPT>(m, mx);
    double sum = 0.0;
#pragma unroll
    for (int q = 0; q < EPL; ++q) {
      // (a row of nothing but -inf has no scores: all 0)
      s[q] = z[q] == -__builtin_inff() ? 0.0 : exp(static_cast<double>(z[q]) - m);
      sum += s[q];
    }
    sum = lanes_reduce<LPT>(sum, add);
    if (sum != 0.0) {
#pragma unroll
      for (int q = 0; q < EPL; ++q) s[q] /= sum;
    }
  }
#pragma unroll
  for (int q = 0; q < EPL; ++q) {
    const int e = q * LPT + l;
    c[q] = e < a.E ? choosable(s[q] + (a.bias ? static_cast<double>(a.bias[e]) : 0.0)) : kNone;
  }
  if (a.groups > 1) {
    // `parts` neighbouring lanes to a group, each with every parts-th expert; where
    // the groups outnumber the lanes, the lanes take them in turn
    const int per = a.E / a.groups;
    int parts = 1;
    while (2 * parts * a.groups <= LPT) parts *= 2;
    const int part = l % parts, step = LPT / parts;
    double* const best = room + a.E;
    wave_fence();
#pragma unroll
    for (int q = 0; q < EPL; ++q)
      if (q * LPT + l < a.E) room[q * LPT + l] = c[q];
    wave_fence();
    for (int g0 = 0; g0 < a.groups; g0 += step) {
      const int g = g0 + l / parts;
      double first = -__builtin_inf(), second = first;
      if (g < a.groups)
        for (int i = part; i < per; i += parts) {
          const double v = room[g * per + i];
          second = fmax(second, fmin(first, v));
          first = fmax(first, v);
        }
      for (int o = 1; o < parts; o *= 2) {
        const double f = __shfl_xor(first, o), h = __shfl_xor(second, o);
        second = fmax(fmin(first, f), fmax(second, h));
        first = fmax(first, f);
      }
      // (an expert that is shut out adds nothing, and does not shut out its group)
      if (g < a.groups && part == 0) best[g] = second == -__builtin_inf() ? first : first + second;
    }
    wave_fence();
    for (int g0 = 0; g0 < a.groups; g0 += step) {
      const int g = g0 + l / parts;
      int ahead = 0;
      if (g < a.groups) {
        const double mine = best[g];
        for (int i = part; i < a.groups; i += parts) ahead += best[i] > mine || (best[i] == mine && i < g);
      }
      for (int o = 1; o < parts; o *= 2) ahead += __shfl_xor(ahead, o);
      // (in the place of the choices, which are read)
      if (g < a.groups && part == 0) room[g] = ahead < a.top_groups ? 1.0 : 0.0;
    }
    wave_fence();
#pragma unroll
    for (int q = 0; q < EPL; ++q) {
      const int e = q * LPT + l;
      if (e < a.E && room[e / per] == 0.0) c[q] = kNone;
    }
  }
  // The k largest, one after another.  A choice's upper 32 bits, as an integer of
  // the same order, mostly tell the largest alone; where two share them (in any
  // token of the wave) the doubles decide, and their ties the lowest index.
  uint32_t key[EPL];
#pragma unroll
  for (int q = 0; q < EPL; ++q) {
    const uint32_t hi = static_cast<uint32_t>(__builtin_bit_cast(uint64_t, c[q]) >> 32);
    key[q] = c[q] != c[q] ? 0u : hi ^ ((hi >> 31) ? 0xffffffffu : 0x80000000u);
  }
  uint32_t top = 0;
  for (int j = 0; j < a.k; ++j) {
    top = key[0];
#pragma unroll
    for (int q = 1; q < EPL; ++q) top = max(top, key[q]);
    top = lanes_max<LPT>(top);
    bool best[EPL];
    int sharing = 0;
#pragma unroll
    for (int q = 0; q < EPL; ++q) {
      best[q] = key[q] == top;
      sharing += __popcll(__ballot(best[q]));
    }
    if (sharing != kWave / LPT) {  // more than one in some token
      double m = kNone;
#pragma unroll
      for (int q = 0; q < EPL; ++q) m = fmax(m, key[q] ? c[q] : kNone);
      m = lanes_reduce<LPT>(m, mx);
      bool found = false;
#pragma unroll
      for (int q = 0; q < EPL; ++q) {
        const bool tie = key[q] && c[q] == m;
        uint64_t bits = __ballot(tie);
        if constexpr (LPT < 64) bits = (bits >> ((threadIdx.x & 63) / LPT * LPT)) & (~0ull >> (64 - LPT));
        best[q] = tie && !found && l == __builtin_ctzll(bits);
        found = found || bits;
      }
    }
#pragma unroll
    for (int q = 0; q < EPL; ++q) {
      place[q] = best[q] ? j : place[q];
      key[q] = best[q] ? 0u : key[q];
    }
  }
  // (the last choice tells whether there is a -inf among them: looked for ahead, every expert's bias
  // cost 2.6 us at 31527 tokens of 128 experts)
  constexpr uint32_t kLeastKey = 0x000fffffu;  // -inf's
  if (a.bias && __any(top <= kLeastKey)) {
#pragma unroll
    for (int q = 0; q < EPL; ++q)
      if (place[q] >= 0 && a.bias[q * LPT + l] == -__builtin_inff()) s[q] = 0.0;
  }
  double sum = 0.0;
#pragma unroll
  for (int q = 0; q < EPL; ++q)
    if (place[q] >= 0) sum += s[q];
  sum = lanes_reduce<LPT>(sum, add);
  const bool over_sum = a.renormalise && sum != 0.0;
  // scale / sum is infinite for the least of sums: there both sides are taken 2^800 larger, which is exact
  const double up = over_sum && sum < 0x1p-800 ? 0x1p800 : 1.0;
  const double by = over_sum ? a.scale / (sum * up) : a.scale;
#pragma unroll
  for (int q = 0; q < EPL; ++q)
    if (valid && place[q] >= 0) {
      const int e = q * LPT + l;
      a.experts[t * a.k + place[q]] = e;
      a.weights[t * a.k + place[q]] = static_cast<float>(s[q] * up * by);
      atomicOr(&mask[e], 1ull << bit);
    }
}

// exclusive prefix sum of n <= kRouteMaxExperts counts in LDS by one workgroup;
// the total behind them (v has n + 1 places)
template <int NTH>
__device__ __forceinline__ void prefix(int32_t* v, int n, int32_t* wave_sums) {
  int carry = 0;
  for (int i0 = 0; i0 < n; i0 += NTH) {
    const int i = i0 + threadIdx.x, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int own = i < n ? v[i] : 0;
    int x = own;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int y = __shfl_up(x, o);
      if (lane >= o) x += y;
    }
    if (lane == 63) wave_sums[w] = x;
    __syncthreads();
    int before = carry, total = carry;
    for (int k = 0; k < NTH / 64; ++k) {
      if (k < w) before += wave_sums[k];
      total += wave_sums[k];
    }
    if (i < n) v[i] = before + x - own;
    carry = total;
    __syncthreads();
  }
  if (threadIdx.x == 0) v[n] = carry;
  __syncthreads();
}

constexpr int kRouteThreads = 512;

// Choices of kRouteBlock tokens.  ALONE: they are all there are, and the block
// finds their places too; else it leaves its count of each expert in ws.
template <int LPT, int EPL, bool ALONE>
__global__ __launch_bounds__(kRouteThreads, 4) void route_kernel(RouteArgs a) {
  constexpr int NTH = kRouteThreads;
  extern __shared__ double room[];
  __shared__ unsigned long long mask[kRouteMaxExperts];
  __shared__ int32_t base[kRouteMaxExperts + 1], wave_sums[NTH / 64];
  for (int e = threadIdx.x; e < a.E; e += NTH) mask[e] = 0;
  __syncthreads();
  constexpr int kPerPass = NTH / LPT;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * kRouteBlock;
  const int n = static_cast<int>(min(static_cast<int64_t>(kRouteBlock), a.T - t0));
  const int mine = threadIdx.x / LPT, l = threadIdx.x % LPT;
  float z[2][EPL];  // this pass's logits and the next's, which are under way meanwhile
  auto load = [&](float (&to)[EPL], int i) {
    const float* row = a.logits + (i < n ? t0 + i : 0) * a.ldl;
#pragma unroll
    for (int q = 0; q < EPL; ++q) to[q] = q * LPT + l < a.E ? row[q * LPT + l] : -__builtin_inff();
  };
  if (n > 0) load(z[0], mine);
  for (int i0 = 0; i0 < n; i0 += kPerPass) {
    const int i = i0 + mine;
    if (i0 + kPerPass < n) load(z[1], i + kPerPass);
    route_token<LPT, EPL>(a, z[0], t0 + i, i < n, l, room + mine * (a.E + a.groups), mask, i);
#pragma unroll
    for (int q = 0; q < EPL; ++q) z[0][q] = z[1][q];
  }
  __syncthreads();
  if (!ALONE) {
    for (int e = threadIdx.x; e < a.E; e += NTH)
      a.ws[static_cast<int64_t>(e) * gridDim.x + blockIdx.x] = __popcll(mask[e]);
    return;
  }
  for (int e = threadIdx.x; e < a.E; e += NTH) base[e] = __popcll(mask[e]);
  __syncthreads();
  prefix<NTH>(base, a.E, wave_sums);
  for (int e = threadIdx.x; e <= a.E; e += NTH) a.offsets[e] = base[e];
  for (int u = threadIdx.x; u < n * a.k; u += NTH) {
    const int e = a.experts[u], i = u / a.k;
    const int sl = base[e] + __popcll(mask[e] & ((1ull << i) - 1));
    a.slot[u] = sl;
    a.src[sl] = i;
  }
}

// ws[e][b]: counts of block b -> counts of blocks 0 .. b
__global__ __launch_bounds__(256) void route_scan_kernel(int32_t* ws, int nb) {
  __shared__ int32_t wave_sums[4];
  int32_t* v = ws + static_cast<int64_t>(blockIdx.x) * nb;
  int carry = 0;
  for (int i0 = 0; i0 < nb; i0 += 256) {
    const int i = i0 + threadIdx.x, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int x = i < nb ? v[i] : 0;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int y = __shfl_up(x, o);
      if (lane >= o) x += y;
    }
    if (lane == 63) wave_sums[w] = x;
    __syncthreads();
    int before = carry;
    for (int k = 0; k < 4; ++k) {
      if (k < w) before += wave_sums[k];
      carry += wave_sums[k];
    }
    if (i < nb) v[i] = before + x;
    __syncthreads();
  }
}

// Places of a block's tokens: the rows of its experts before it, then its own
// tokens in order.  SCANNED: ws went through route_scan_kernel.
template <bool SCANNED>
__global__ __launch_bounds__(256) void route_place_kernel(RouteArgs a, int nb) {
  __shared__ unsigned long long mask[kRouteMaxExperts];
  __shared__ int32_t base[kRouteMaxExperts + 1], wave_sums[4];
  const int b = blockIdx.x;
  const int64_t t0 = static_cast<int64_t>(b) * kRouteBlock;
  const int n = static_cast<int>(min(static_cast<int64_t>(kRouteBlock), a.T - t0));
  int before[kRouteMaxExperts / 256];  // rows of the thread's experts in earlier blocks
#pragma unroll
  for (int j = 0; j < kRouteMaxExperts / 256; ++j) {
    const int e = threadIdx.x + 256 * j;
    if (e >= a.E) break;
    const int32_t* v = a.ws + static_cast<int64_t>(e) * nb;
    int here = 0, all = 0;
    if (SCANNED) {
      here = b > 0 ? v[b - 1] : 0;
      all = v[nb - 1];
    } else {
      for (int i = 0; i < nb; ++i) {
        const int n_i = v[i];
        here += i < b ? n_i : 0;
        all += n_i;
      }
    }
    mask[e] = 0;
    base[e] = all;
    before[j] = here;
  }
  __syncthreads();
  prefix<256>(base, a.E, wave_sums);
  if (b == 0)
    for (int e = threadIdx.x; e <= a.E; e += 256) a.offsets[e] = base[e];
  for (int u = threadIdx.x; u < n * a.k; u += 256) atomicOr(&mask[a.experts[t0 * a.k + u]], 1ull << (u / a.k));
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kRouteMaxExperts / 256; ++j) {
    const int e = threadIdx.x + 256 * j;
    if (e < a.E) base[e] += before[j];
  }
  __syncthreads();
  for (int u = threadIdx.x; u < n * a.k; u += 256) {
    const int e = a.experts[t0 * a.k + u], i = u / a.k;
    const int sl = base[e] + __popcll(mask[e] & ((1ull << i) - 1));
    a.slot[t0 * a.k + u] = sl;
    a.src[sl] = static_cast<int32_t>(t0 + i);
  }
}

// Lanes of a token and experts of a lane.  Up to 8 experts a lane keep most
// instructions busy for several tokens at once (31527 tokens of 128 experts, 8 of them
// chosen in 4 of 8 groups, 16 x 8 / 32 x 4 / 64 x 2: 25.0 / 28.1 / 38.4 us; of 256, 32 x 8 / 64 x 4
// 46.4 / 55.8; of 64, 16 x 4 / 32 x 2 15.6 / 19.9; 8 x 8 14.9, whose room would not fit);
// where every token has a wave of its own, more lanes are sooner done (one token
// of 64 experts 64 x 1 / 16 x 4 4.3 / 6.1, of 256 64 x 4 / 32 x 8 7.4 / 10.3).  (1024 threads: 25.6 and
// 29.0 for 16 x 8 and 32 x 4; 256: 32.4 and 37.7.)
template <bool ALONE>
void launch_choices(const RouteArgs& a, int nb, hipStream_t s) {
  auto go = [&](auto lpt, auto epl) {
    constexpr int LPT = decltype(lpt)::value, EPL = decltype(epl)::value;
    // experts and groups (no more than experts) of the tokens at a time, beside the masks and bases
    static_assert(kRouteThreads / LPT * (LPT * EPL + std::min(LPT * EPL, kRouteMaxGroups)) * sizeof(double) <= 56 * 1024);
    const uint32_t room = a.groups > 1 ? static_cast<uint32_t>(kRouteThreads / LPT * (a.E + a.groups) * sizeof(double)) : 0;
    route_kernel<LPT, EPL, ALONE><<<dim3(nb), dim3(kRouteThreads), room, s>>>(a);
  };
  using std::integral_constant;
  if constexpr (ALONE) {
    if (a.T <= kRouteThreads / 64 && a.E > 8 && a.E <= 256) {
      if (a.E <= 16) return go(integral_constant<int, 16>{}, integral_constant<int, 1>{});
      if (a.E <= 32) return go(integral_constant<int, 32>{}, integral_constant<int, 1>{});
      if (a.E <= 64) return go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
      if (a.E <= 128) return go(integral_constant<int, 64>{}, integral_constant<int, 2>{});
      return go(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    }
  }
  if (a.E <= 8) return go(integral_constant<int, 8>{}, integral_constant<int, 1>{});
  if (a.E <= 16) return go(integral_constant<int, 8>{}, integral_constant<int, 2>{});
  if (a.E <= 32) return go(integral_constant<int, 8>{}, integral_constant<int, 4>{});
  if (a.E <= 64) return go(integral_constant<int, 16>{}, integral_constant<int, 4>{});
  if (a.E <= 128) return go(integral_constant<int, 16>{}, integral_constant<int, 8>{});
  if (a.E <= 256) return go(integral_constant<int, 32>{}, integral_constant<int, 8>{});
  go(integral_constant<int, 64>{}, integral_constant<int, 8>{});
}

}  // namespace

// Blocks of kRouteBlock tokens up to which each adds up the counts of all itself.
constexpr int kRouteOwnSums = 32;

hipError_t launch_route(const RouteArgs& a, hipStream_t s) {
  const int nb = (a.T + kRouteBlock - 1) / kRouteBlock;
  if (nb <= 1) {
    launch_choices<true>(a, 1, s);
    return hipGetLastError();
  }
  launch_choices<false>(a, nb, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (nb <= kRouteOwnSums) {
    route_place_kernel<false><<<dim3(nb), dim3(256), 0, s>>>(a, nb);
    return hipGetLastError();
  }
  route_scan_kernel<<<dim3(a.E), dim3(256), 0, s>>>(a.ws, nb);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  route_place_kernel<true><<<dim3(nb), dim3(256), 0, s>>>(a, nb);
  return hipGetLastError();
}

}  // namespace metro
