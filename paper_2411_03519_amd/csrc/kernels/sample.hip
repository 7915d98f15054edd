// Sampled choice of a token (gfx950, wave64).
//
// A row's tokens stand in the order of falling logits, ties by rising index, with
// weights w = exp((x - max) / T).  min-p takes away the weights below min_p, top-k
// all but the first k, top-p all but the shortest beginning that holds top_p of
// what is left; the token is the first whose weights up to it pass u times the
// weights that are left.  All three leave a beginning of the order, so the steps
// need nothing but searches of the running sums of weights and of counts.
//
// Weights are held as whole multiples of 2^-45 (from exp in fp64), so that sums
// of up to 2^18 of them are exact in 64 bits in whatever order they are added:
// the atomics below change no result.  A weight below 2^-46 counts as none.
//
// A search goes by a histogram of (max - x) / T over [0, 32), which all weights
// that count fall into: the bin that the searched sum lies in is known from the
// bins' sums, and its tokens are ranked among themselves.  A bin of many tokens
// is cut into finer ones by the bits of its logits until few are left or all are
// the same.
#include "common.h"
#include "kernels.h"
#include "kernels_draft.h"

namespace metro {

constexpr int kSampleThreads = 1024;
constexpr int kSampleBins = 1024;
constexpr int kSampleList = 256;  // tokens that are ranked by comparing all pairs
constexpr double kSampleOne = 35184372088832.0;  // 2^45, the weight of the largest logit

// order of floats as unsigned numbers (-0 as 0)
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

struct RowRule {
  float max;
  double inv_t;     // 1 / T
  uint64_t least;   // smallest weight that counts
};

// (max - x) / T, 0 for the largest; at least 1e9 where the weight counts as none
__device__ __forceinline__ double depth(const RowRule& r, float x) {
  if (x == r.max) return 0.0;
  if (!(x > -INFINITY) || r.max == INFINITY) return 1e9;
  return (static_cast<double>(r.max) - static_cast<double>(x)) * r.inv_t;
}

__device__ __forceinline__ uint64_t weight(const RowRule& r, float x) {
  const double d = depth(r, x);
  if (!(d < 32.0)) return 0;
  const uint64_t w = static_cast<uint64_t>(rint(exp(-d) * kSampleOne));
  return w >= r.least ? w : 0;
}

__device__ __forceinline__ int depth_bin(const RowRule& r, float x) {
  return static_cast<int>(depth(r, x) * (kSampleBins / 32.0));
}

struct SampleShared {
  uint64_t mass[kSampleBins];
  uint32_t count[kSampleBins];
  uint64_t scan_m[16];
  uint32_t scan_c[16];
  uint32_t list_key[kSampleList];
  int list_index[kSampleList];
  uint32_t n_list, key_lo, key_hi;
  int bin, index;
  uint64_t before_m, upto_m, w_one;
  uint32_t before_c;
  float red_v[16];
  int red_i[16];
};

// Finds the bin b whose sums hold the searched one: before < want <= before + its own (masses, or counts).
__device__ void find_bin(SampleShared& sh, bool by_count, uint64_t want, uint64_t base_m, uint32_t base_c) {
  static_assert(kSampleBins == kSampleThreads, "a bin a thread");
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint64_t m = sh.mass[tid];
  const uint32_t c = sh.count[tid];
  uint64_t im = m;
  uint32_t ic = c;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t pm = __shfl_up(static_cast<unsigned long long>(im), o, kWave);
    const uint32_t pc = __shfl_up(ic, o, kWave);
    if (lane >= o) im += pm, ic += pc;
  }
  if (lane == 63) sh.scan_m[wave] = im, sh.scan_c[wave] = ic;
  __syncthreads();
  uint64_t bm = base_m;
  uint32_t bc = base_c;
  for (int w = 0; w < wave; ++w) bm += sh.scan_m[w], bc += sh.scan_c[w];
  im += bm, ic += bc;
  const uint64_t upto = by_count ? ic : im, before = by_count ? ic - c : im - m;
  if (before < want && want <= upto) sh.bin = tid, sh.before_m = im - m, sh.before_c = ic - c;
  __syncthreads();
}

// First token of the order whose sum up to it (of weights, or of tokens) reaches want, 1 <= want <= the sum of all;
// leaves its sum of weights in upto_m, its own weight in w_one and, with index, its index.
template <typename Get>
__device__ void locate(SampleShared& sh, const RowRule& r, Get get, int vocab, bool by_count, uint64_t want, bool index) {
  const int tid = threadIdx.x;
  find_bin(sh, by_count, want, 0, 0);
  const int bin = sh.bin;
  uint64_t before_m = sh.before_m;
  uint32_t before_c = sh.before_c, n = sh.count[bin];
  // the bin's logits lie within [lo, hi] as order keys
  uint32_t lo = 0, hi = 0xffffffffu;
  auto mine = [&](float x) {
    if (!(x == x)) return false;
    const uint32_t k = order_key(x);
    return k >= lo && k <= hi && weight(r, x) > 0 && depth_bin(r, x) == bin;
  };
  __syncthreads();
  if (n > kSampleList) {
    if (tid == 0) sh.key_lo = 0xffffffffu, sh.key_hi = 0;
    __syncthreads();
    uint32_t l = 0xffffffffu, u = 0;
    for (int i = tid; i < vocab; i += kSampleThreads) {
      const float x = get(i);
      if (mine(x)) l = min(l, order_key(x)), u = max(u, order_key(x));
    }
    atomicMin(&sh.key_lo, l);
    atomicMax(&sh.key_hi, u);
    __syncthreads();
    lo = sh.key_lo, hi = sh.key_hi;
    __syncthreads();
  }
  while (n > kSampleList && lo < hi) {
    const int shift = max(0, 32 - __clz(hi - lo) - 10);  // (hi - lo) >> shift < 1024
    sh.mass[tid] = 0, sh.count[tid] = 0;
    __syncthreads();
    for (int i = tid; i < vocab; i += kSampleThreads) {
      const float x = get(i);
      if (!mine(x)) continue;
      const uint32_t b = (hi - order_key(x)) >> shift;
      atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[b]), static_cast<unsigned long long>(weight(r, x)));
      atomicAdd(&sh.count[b], 1u);
    }
    __syncthreads();
    find_bin(sh, by_count, want, before_m, before_c);
    const uint32_t sub = sh.bin;
    before_m = sh.before_m, before_c = sh.before_c, n = sh.count[sub];
    const uint64_t to = static_cast<uint64_t>(hi) - (static_cast<uint64_t>(sub) << shift);
    const uint64_t from = (static_cast<uint64_t>(sub) + 1) << shift;
    lo = max(static_cast<uint64_t>(lo), static_cast<uint64_t>(hi) + 1 > from ? static_cast<uint64_t>(hi) + 1 - from : 0);
    hi = static_cast<uint32_t>(to);
    __syncthreads();
  }
  if (n > kSampleList) {  // all the same
    const uint64_t w = weight(r, key_value(hi));
    const uint64_t nth = by_count ? want - before_c : (want - before_m + w - 1) / w;  // 1, 2, ...
    if (tid == 0) sh.upto_m = before_m + nth * w, sh.w_one = w;
    if (index) {
      const int chunk = (vocab + kSampleThreads - 1) / kSampleThreads, i0 = tid * chunk, i1 = min(i0 + chunk, vocab);
      uint32_t c = 0;
      for (int i = i0; i < i1; ++i) c += get(i) == key_value(hi) ? 1 : 0;
      sh.mass[tid] = 0, sh.count[tid] = c;
      __syncthreads();
      find_bin(sh, true, nth, 0, 0);
      if (tid == sh.bin) {
        uint32_t left = static_cast<uint32_t>(nth) - sh.before_c;
        for (int i = i0; i < i1; ++i)
          if (get(i) == key_value(hi) && --left == 0) {
            sh.index = i;
            break;
          }
      }
    }
    __syncthreads();
    return;
  }
  if (tid == 0) sh.n_list = 0;
  __syncthreads();
  for (int i = tid; i < vocab; i += kSampleThreads) {
    const float x = get(i);
    if (!mine(x)) continue;
    const uint32_t at = atomicAdd(&sh.n_list, 1u);
    if (at < kSampleList) sh.list_key[at] = order_key(x), sh.list_index[at] = i;
  }
  __syncthreads();
  if (tid < static_cast<int>(sh.n_list)) {
    const uint32_t key = sh.list_key[tid];
    const int at = sh.list_index[tid];
    uint64_t m = before_m;
    uint32_t c = before_c;
    for (uint32_t j = 0; j < sh.n_list; ++j) {
      const uint32_t k = sh.list_key[j];
      if (k > key || (k == key && sh.list_index[j] < at)) m += weight(r, key_value(k)), ++c;
    }
    const uint64_t w = weight(r, key_value(key));
    if (by_count ? c + 1 == want : m < want && want <= m + w) sh.upto_m = m + w, sh.w_one = w, sh.index = at;
  }
  __syncthreads();
}

__global__ __launch_bounds__(kSampleThreads) void sample_kernel(SampleArgs a) {
  __shared__ SampleShared sh;
  const int row = blockIdx.x, tid = threadIdx.x;
  const float* x = a.logits + static_cast<size_t>(row) * a.ldl;
  auto get = [&](int i) { return x[i]; };
  // the largest and its lowest index, NaN skipped
  float best = -INFINITY;
  int at = INT32_MAX;
  for (int i = tid; i < a.vocab; i += kSampleThreads)
    if (const float v = get(i); v > best) best = v, at = i;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const float v = __shfl_xor(best, o, kWave);
    const int i = __shfl_xor(at, o, kWave);
    if (v > best || (v == best && i < at)) best = v, at = i;
  }
  if ((tid & 63) == 0) sh.red_v[tid >> 6] = best, sh.red_i[tid >> 6] = at;
  __syncthreads();
  for (int w = 0; w < kSampleThreads / 64; ++w) {
    const float v = sh.red_v[w];
    const int i = sh.red_i[w];
    if (v > best || (v == best && i < at)) best = v, at = i;
  }
  const float t = a.temperature ? a.temperature[row] : 1.f;
  if (!(best > -INFINITY) || !(t > 0.f)) {
    if (tid == 0) {
      a.out[row] = best > -INFINITY ? at : -1;
      if (a.prob) a.prob[row] = best > -INFINITY ? 1.f : 0.f;
    }
    return;
  }
  const float min_p = a.min_p ? a.min_p[row] : 0.f, top_p = a.top_p ? a.top_p[row] : 1.f;
  const int top_k = a.top_k ? a.top_k[row] : 0;
  RowRule r;
  r.max = best;
  r.inv_t = 1.0 / static_cast<double>(t);
  r.least = min_p > 0.f ? static_cast<uint64_t>(ceil(fmin(static_cast<double>(min_p), 1.0) * kSampleOne)) : 1;
  auto fill = [&] {
    sh.mass[tid] = 0, sh.count[tid] = 0;
    __syncthreads();
    for (int i = tid; i < a.vocab; i += kSampleThreads) {
      const float v = get(i);
      const uint64_t w = weight(r, v);
      if (w == 0) continue;
      const int b = depth_bin(r, v);
      atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[b]), static_cast<unsigned long long>(w));
      atomicAdd(&sh.count[b], 1u);
    }
    __syncthreads();
  };
  fill();
  uint64_t total = 0;
  uint32_t tokens = 0;
  for (int b = tid & 63; b < kSampleBins; b += 64) total += sh.mass[b], tokens += sh.count[b];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    total += __shfl_xor(static_cast<unsigned long long>(total), o, kWave);
    tokens += __shfl_xor(tokens, o, kWave);
  }
  __syncthreads();
  if (top_k > 0 && static_cast<uint32_t>(top_k) < tokens) {
    locate(sh, r, get, a.vocab, true, top_k, false);
    total = sh.upto_m;
    fill();
  }
  if (top_p < 1.f) {
    const double want = ceil(static_cast<double>(fmaxf(top_p, 0.f)) * static_cast<double>(total));
    locate(sh, r, get, a.vocab, false, min(max(static_cast<uint64_t>(want), uint64_t{1}), total), false);
    total = sh.upto_m;
    fill();
  }
  const float u = a.u[row];
  const double want = floor(static_cast<double>(u > 0.f ? u : 0.f) * static_cast<double>(total));
  const uint64_t goal = want < static_cast<double>(total) ? static_cast<uint64_t>(want) + 1 : total;
  locate(sh, r, get, a.vocab, false, min(goal, total), true);
  if (tid == 0) {
    a.out[row] = sh.index;
    if (a.prob) a.prob[row] = static_cast<float>(static_cast<double>(sh.w_one) / static_cast<double>(total));
  }
}

int64_t sample_workspace(int, int) { return 0; }

hipError_t launch_sample(const SampleArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  launch_kernel(sample_kernel, dim3(a.rows), dim3(kSampleThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace metro
