// Sampled choice of a token (gfx950, wave64).
//
// A row's tokens stand in the order of falling logits, ties by rising index, with
// weights w = exp((x - max) / T).  min-p takes away the weights below min_p, top-k
// all but the first k, top-p all but the shortest beginning that holds top_p of
// what is left; the token is the first whose weights up to it pass u times the
// weights that are left.  All three leave a beginning of the order, so the steps
// need nothing but searches of the running sums of weights and of counts.  From
// u = 1 on the last token left is found by its count: the sums round, and a weight
// that they lose, or the same sum formed another way, would end such a search early
// or late.
//
// A search goes by a histogram.  Bins lie about the whole numbers of t = 32 x / T,
// the same for every part of a row, counted down from the row's largest; 1024 of them
// hold all weights above e^-32 of the largest, the others count as none.  Within
// its bin a weight is held relative to the bin's upper edge, exp(-g), 0 < g <=
// 1/32, as a whole multiple of 2^-34: so its relative error is the same 2^-35
// wherever in the row it lies, and the bins' sums are whole numbers, exact in any
// order of adding, of which one 64-bit word holds the sum and the count.  Running
// sums over bins are fp64, in one order.
//
// Two launches.  The first reads the logits once: a workgroup for each 16384 of a
// row leaves its maximum, its histogram, and the tokens of its top bins (up to 256
// of them).  The second, a workgroup for each row, adds the histograms up, finds
// the bins that the searched sums lie in and ranks their tokens among themselves.
// Mostly those bins are top ones of every part, whose tokens are at hand; else the
// row is read again for them.  A bin of many tokens is cut into finer ones by the
// bits of its logits until few are left or all are the same.
//
// What bounds it: the first launch the vector ALU, which issues 87% of the time (49
// instructions a logit, 16 of them fp64; LDS is active 39%, a third of that in
// conflicts; 325 rows of 128256 logits 71 to 76 us, 2.3 TB/s; a row in fewer, larger
// workgroups 78), one row 9.7 us from end to end; the second the latency of its some 15
// barriers and of what every wave forms alike between them, 11 to 17 us a row whose
// bins are listed, up to 36 where the row is read again or its bins are crowded (marked
// tokens fetched two or four at a time, or the lists with the maxima, gave nothing), and
// its 90 KB of LDS and 127 registers, which leave a CU one workgroup: more than 256 rows
// go in two rounds.  One workgroup a row for everything, with weights in fp64 exp():
// 344 us for one row, 764 for 325.
#include "common.h"
#include "kernels.h"
#include "kernels_draft.h"

// Bins and weights of a logit are formed in several places and have to be the same in all of them: products and sums
// are joined to one rounding only where the code says so.
#pragma clang fp contract(off)

namespace metro {

constexpr int kSampleThreads = 1024;
constexpr int kSampleBins = 1024;
constexpr int kSampleChunk = 16384;  // logits of a workgroup, 16 a thread
constexpr int kSampleList = 256;     // tokens of a chunk that are listed
constexpr int kSampleChunks = kSampleMaxVocab / kSampleChunk;
constexpr int kMassBits = 49;  // of a bin's word, the count above them: 16384 * 2^34 < 2^49
constexpr uint64_t kMassMask = (1ull << kMassBits) - 1;
constexpr double kMassOne = 17179869184.0;  // 2^34

// What the first launch leaves of a chunk.
struct SampleChunk {
  float max;      // -inf: no token above it
  int index;      // of the maximum, the lowest
  int covered;    // the tokens of its bins 0 .. covered - 1 are listed
  int listed;     // so many
  uint64_t bin[kSampleBins];  // from its own largest down
  float2 list[kSampleList];   // (logit, index as bits)
};

// order of floats as unsigned numbers (-0 as 0)
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// The bins' grid: t = x * per, bins about its whole numbers; top is the bin of the largest logit (infinite with it).  From
// 2^50 on, where other logits than the largest lie further than all bins below it, bins have no width.
struct SampleGrid {
  double per, top, step;
  double width;  // of a bin in logits, 1 / per
};

// The nearest whole number of |t| < 2^51, ties to even; the adding leaves no room behind the point.
__device__ __forceinline__ double nearest_whole(double t) { return (t + 6755399441055744.0) - 6755399441055744.0; }

__device__ __forceinline__ SampleGrid sample_grid(float max, float t) {
  SampleGrid g;
  g.per = 32.0 / static_cast<double>(t);
  g.width = static_cast<double>(t) / 32.0;
  g.top = max == INFINITY ? static_cast<double>(INFINITY) : nearest_whole(static_cast<double>(max) * g.per);
  g.step = fabs(g.top) < 1125899906842624.0 ? 1.0 / 32.0 : 0.0;
  return g;
}

// How many bins a logit lies below the top one (not below 1024, or NaN, where its weight counts as none), for a finite
// top; *mass: its weight relative to the bin's upper edge, exp(g), in units of 2^-34.  The adding of 2^18 leaves 34 bits
// behind the point in a double's mantissa.
__device__ __forceinline__ double bins_below(const SampleGrid& grid, float x, uint64_t* mass) {
  const double t = static_cast<double>(x) * grid.per, whole = nearest_whole(t);
  const double g = fma(t - whole, grid.step, -0.5 * grid.step);  // -1/32 .. 0; the series' next term is below 2^-39
  double e = fma(g, 1.0 / 120.0, 1.0 / 24.0);
  e = fma(e, g, 1.0 / 6.0);
  e = fma(e, g, 0.5);
  e = fma(e, g, 1.0);
  e = fma(e, g, 1.0);
  *mass = __double_as_longlong(e + 262144.0) & ((1ull << 52) - 1);
  return grid.top - whole;
}

// A whole number below 2^31 of a double: the adding of 2^52 leaves it in the lower bits (conversions of fp64 run at a
// quarter of the rate).
__device__ __forceinline__ int whole_bits(double d) { return static_cast<int>(__double_as_longlong(d + 4503599627370496.0)); }

// Bin of a logit below the top one, or -1 where its weight counts as none.
__device__ __forceinline__ int sample_bin(const SampleGrid& grid, float x, uint64_t* mass) {
  if (grid.top == static_cast<double>(INFINITY)) {
    *mass = 1ull << 34;
    return x == INFINITY ? 0 : -1;
  }
  const double below = bins_below(grid, x, mass);
  return below < static_cast<double>(kSampleBins) ? whole_bits(below) : -1;  // (NaN and -inf: -1)
}

struct SampleRange {
  float lo, hi;
  __device__ __forceinline__ bool has(float v) const { return v >= lo && v <= hi; }
};

// A range that holds the logits of bins first .. last, from their edges in t with room for their rounding.
__device__ __forceinline__ SampleRange range_of(const SampleGrid& grid, double first, double last) {
  const double lo = (grid.top - last - 0.5) * grid.width, hi = (grid.top - first + 0.5) * grid.width;
  return SampleRange{isfinite(lo) ? static_cast<float>(lo - fabs(lo) * 1e-6 - 1e-37) : -INFINITY,
                     isfinite(hi) ? static_cast<float>(hi + fabs(hi) * 1e-6 + 1e-37) : INFINITY};
}

struct SampleBest {
  float v;
  int i;
};
__device__ __forceinline__ SampleBest best_of(SampleBest a, SampleBest b) {
  return b.v > a.v || (b.v == a.v && b.i < a.i) ? b : a;
}

__device__ __forceinline__ void lds_add(uint64_t* p, uint64_t v) {
  atomicAdd(reinterpret_cast<unsigned long long*>(p), static_cast<unsigned long long>(v));
}

__global__ __launch_bounds__(kSampleThreads, 8) void sample_chunk_kernel(SampleArgs a, int chunks) {
  constexpr int V = kSampleChunk / kSampleThreads;
  __shared__ uint64_t bin[kSampleBins];
  __shared__ SampleBest best[kSampleThreads / 64];
  __shared__ uint32_t sums[kSampleThreads / 64];
  __shared__ int n_list;
  const int row = blockIdx.x / chunks, c = blockIdx.x % chunks, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float* x = a.logits + static_cast<size_t>(row) * a.ldl;
  const int first = c * kSampleChunk + 4 * tid;
  const bool wide = (reinterpret_cast<uintptr_t>(x) & 15) == 0;
  float v[V];
#pragma unroll
  for (int j = 0; j < V / 4; ++j) {
    const int i = first + j * 4 * kSampleThreads;
    if (wide && i + 3 < a.vocab) {
      const float4 w = *reinterpret_cast<const float4*>(x + i);
      v[4 * j] = w.x, v[4 * j + 1] = w.y, v[4 * j + 2] = w.z, v[4 * j + 3] = w.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * j + e] = i + e < a.vocab ? x[i + e] : __builtin_nanf("");
    }
  }
  const float t = a.temperature ? a.temperature[row] : 1.f;
  bin[tid] = 0;
  if (tid == 0) n_list = 0;
  SampleBest b{-INFINITY, INT32_MAX};
#pragma unroll
  for (int j = 0; j < V; ++j) b.v = fmaxf(b.v, v[j]);  // (NaN aside)
#pragma unroll
  for (int j = V - 1; j >= 0; --j) b.i = v[j] == b.v ? first + j / 4 * 4 * kSampleThreads + j % 4 : b.i;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) b = best_of(b, SampleBest{__shfl_xor(b.v, o, kWave), __shfl_xor(b.i, o, kWave)});
  if (lane == 0) best[wave] = b;
  __syncthreads();
  b = best[lane % (kSampleThreads / 64)];
#pragma unroll
  for (int o = kSampleThreads / 128; o > 0; o >>= 1) b = best_of(b, SampleBest{__shfl_xor(b.v, o, kWave), __shfl_xor(b.i, o, kWave)});
  SampleChunk* out = reinterpret_cast<SampleChunk*>(a.ws) + blockIdx.x;
  if (tid == 0) out->max = b.v, out->index = b.i;
  if (!(t > 0.f) || !(b.v > -INFINITY)) return;  // (greedy, or nothing to choose: the rest is not read)
  const SampleGrid grid = sample_grid(b.v, t);
  if (b.v == INFINITY) {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (v[j] == INFINITY) lds_add(&bin[0], (1ull << 34) + (1ull << kMassBits));
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      uint64_t mass;
      const double below = bins_below(grid, v[j], &mass);
      if (below < static_cast<double>(kSampleBins)) lds_add(&bin[whole_bits(below)], mass + (1ull << kMassBits));
      if (j % 2) __builtin_amdgcn_sched_barrier(0);  // (two at a time: all at once take more than 64 registers)
    }
  }
  __syncthreads();
  const uint64_t mine = bin[tid];
  out->bin[tid] = mine;
  uint32_t n = static_cast<uint32_t>(mine >> kMassBits);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t p = __shfl_up(n, o, kWave);
    if (lane >= o) n += p;
  }
  if (lane == 63) sums[wave] = n;
  __syncthreads();
  for (int w = 0; w < wave; ++w) n += sums[w];
  const int covered = __syncthreads_count(n <= kSampleList);
  // (a range that may hold a few of the next bin's too: with more than there is room for, nothing counts as covered)
  const float from = covered > 0 ? range_of(grid, 0, covered - 1).lo : INFINITY;
#pragma unroll
  for (int j = 0; j < V; ++j)
    if (v[j] >= from) {
      const int at = atomicAdd(&n_list, 1);
      if (at < kSampleList) out->list[at] = make_float2(v[j], __int_as_float(first + j / 4 * 4 * kSampleThreads + j % 4));
    }
  __syncthreads();
  if (tid == 0) out->covered = n_list <= kSampleList ? covered : 0, out->listed = min(n_list, kSampleList);
}

constexpr int kSampleGather = 4096;  // tokens that the second launch holds in LDS (2048: 25 rows 54 us for 48)
constexpr int kSampleRank = 96;      // tokens that are ranked by comparing all pairs
constexpr int kSampleRankStep = 4;   // so many at a time (one: 325 rows 106 us for 100; eight: 103)
static_assert(kSampleRank % kSampleRankStep == 0, "");

constexpr int kSampleSearches = 8;   // for bins, each with room of its own

// A token among those of its bin: `place` is larger for one that stands before it in the row's order, 0 is none.
struct __attribute__((aligned(16))) SampleToken {
  uint64_t place, mass;
};

struct SampleShared {
  double before[kSampleBins], with[kSampleBins];    // weight of the bins above, and with this one
  double scale[kSampleBins];                        // of a bin's masses
  uint32_t count[kSampleBins], above[kSampleBins];  // tokens of a bin, and of the bins above
  uint64_t sub_mass[kSampleBins];
  uint32_t sub_count[kSampleBins];
  uint32_t key[kSampleGather];  // the gathered tokens
  int index[kSampleGather];
  uint16_t bin[kSampleGather];
  uint8_t wanted[kSampleBins];  // bins that are gathered
  SampleToken rank[kSampleRank];
  double scan_w[16];
  uint64_t scan_m[16];
  uint32_t scan_c[16];
  int scan_last[16];
  uint32_t n, n_wanted, some_n;
  uint64_t some;
  int first, sub;
  int found_bin[kSampleSearches][kSampleThreads / 64];
  // what a search leaves: the weights up to its token and with it, the token's own weight, its index, and how many tokens
  // of the order it ends
  double upto, own;
  int found;
  uint32_t ends;
  int shift[kSampleChunks];    // bins between the row's largest and a chunk's; all of them where it counts for nothing
  int covered[kSampleChunks];  // bins of a chunk whose tokens are listed
  int listed[kSampleChunks];   // its list's length
};

enum SampleWant { kByCount, kReach, kPass };  // the first token whose count, or weight, up to it reaches, or passes, the wanted

__device__ __forceinline__ double bin_scale(int b) { return exp(-b / 32.0) / kMassOne; }

// The weight up to a token of a bin.  One rounding wherever it is formed, so that equal sums compare equal.
__device__ __forceinline__ double weight_up_to(double before, uint64_t mass, double scale) {
  return fma(static_cast<double>(mass), scale, before);
}

constexpr SampleRange kNoRange{INFINITY, -INFINITY};

// f(logit, index) of a row's logits within either range.  The few that are, of 32 at a time, are marked first and then taken
// one by one from memory again: tested where they are, nearly every wave would go through f for some lane.
template <typename F>
__device__ __forceinline__ void each_of_row(const float* x, int vocab, SampleRange a, SampleRange b, F f) {
  const int tid = threadIdx.x;
  const int head = min(static_cast<int>(((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / 4), vocab);
  const int n4 = (vocab - head) / 4, tail = head + 4 * n4;
  auto test = [&](int i) {
    const float v = x[i];
    if (a.has(v) || b.has(v)) f(v, i);
  };
  if (tid < head) test(tid);
  if (tid < vocab - tail) test(tail + tid);
  const float4* x4 = reinterpret_cast<const float4*>(x + head);
  constexpr int U = 8;
  for (int j0 = tid; j0 < n4; j0 += U * kSampleThreads) {
    float4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = x4[min(j0 + u * kSampleThreads, n4 - 1)];
    uint32_t in = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      auto bit = [&](float v, uint32_t one) { return a.has(v) || b.has(v) ? one : 0u; };
      const uint32_t some = bit(w[u].x, 1u) | bit(w[u].y, 2u) | bit(w[u].z, 4u) | bit(w[u].w, 8u);
      in |= j0 + u * kSampleThreads < n4 ? some << (4 * u) : 0u;
    }
    for (; in; in &= in - 1) {
      const int k = __ffs(static_cast<int>(in)) - 1, i = head + 4 * (j0 + k / 4 * kSampleThreads) + k % 4;
      f(x[i], i);
    }
  }
}

__global__ __launch_bounds__(kSampleThreads) void sample_kernel(SampleArgs a, int chunks) {
  __shared__ SampleShared sh;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, vocab = a.vocab;
  const float* x = a.logits + static_cast<size_t>(row) * a.ldl;
  const SampleChunk* chunk = reinterpret_cast<const SampleChunk*>(a.ws) + static_cast<size_t>(row) * chunks;
  const SampleChunk& own_chunk = chunk[min(lane % kSampleChunks, chunks - 1)];
  SampleBest b{own_chunk.max, own_chunk.index};
  const float chunk_max = b.v;
  const int own_covered = own_chunk.covered, own_listed = own_chunk.listed;
  const float t = a.temperature ? a.temperature[row] : 1.f;
  const float min_p = a.min_p ? a.min_p[row] : 0.f, top_p = a.top_p ? a.top_p[row] : 1.f, u = a.u[row];
  const int top_k = a.top_k ? a.top_k[row] : 0;
#pragma unroll
  for (int o = kSampleChunks / 2; o > 0; o >>= 1) b = best_of(b, SampleBest{__shfl_xor(b.v, o, kWave), __shfl_xor(b.i, o, kWave)});
  if (!(b.v > -INFINITY) || !(t > 0.f)) {
    if (tid == 0) {
      a.out[row] = b.v > -INFINITY ? b.i : -1;
      if (a.prob) a.prob[row] = b.v > -INFINITY ? 1.f : 0.f;
    }
    return;
  }
  const SampleGrid grid = sample_grid(b.v, t);
  if (tid < chunks) {
    // (an infinite difference, or that of infinities: all of the chunk or nothing)
    const double d = chunk_max == b.v ? 0.0 : grid.top - sample_grid(chunk_max, t).top;
    const bool any = chunk_max > -INFINITY && d < static_cast<double>(kSampleBins);
    sh.shift[tid] = any ? static_cast<int>(d) : kSampleBins;
    sh.covered[tid] = any ? own_covered : 0;
    sh.listed[tid] = any ? own_listed : 0;
  }
  if (tid == 0) sh.n = 0, sh.n_wanted = 0, sh.some = 0, sh.some_n = 0;
  sh.wanted[tid] = 0;
  __syncthreads();

  // The row's histogram and its running sums.
  uint64_t mass = 0;
  uint32_t count = 0;
#pragma unroll 8
  for (int c = 0; c < chunks; ++c) {
    const int at = tid - sh.shift[c];
    uint64_t v = chunk[c].bin[max(at, 0)];
    v = at < 0 ? 0 : v;
    mass += v & kMassMask;
    count += static_cast<uint32_t>(v >> kMassBits);
  }
  const double scale_here = bin_scale(tid);
  double iw = static_cast<double>(mass) * scale_here;
  uint32_t ic = count;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double pw = __shfl_up(iw, o, kWave);
    const uint32_t pc = __shfl_up(ic, o, kWave);
    if (lane >= o) iw += pw, ic += pc;
  }
  const uint64_t any = __ballot(count > 0);
  if (lane == 63) sh.scan_w[wave] = iw, sh.scan_c[wave] = ic, sh.scan_last[wave] = any ? 64 * wave + 63 - __clzll(any) : 0;
  double bw = __shfl_up(iw, 1, kWave);
  if (lane == 0) bw = 0.0;
  __syncthreads();
  double head = 0.0;
  uint32_t bc = ic - count;
  int last_bin = 0;
#pragma unroll
  for (int k = 0; k < kSampleThreads / 64; ++k) {
    head += k < wave ? sh.scan_w[k] : 0.0;
    bc += k < wave ? sh.scan_c[k] : 0;
    last_bin = max(last_bin, sh.scan_last[k]);
  }
  const double my_with = weight_up_to(head + bw, mass, scale_here);
  const uint32_t my_tokens = bc + count;
  sh.scale[tid] = scale_here;
  sh.before[tid] = head + bw;
  sh.with[tid] = my_with;
  sh.above[tid] = bc;
  sh.count[tid] = count;
  __syncthreads();

  // The first bin that holds any token and whose count or weight, with the bins above, is as wanted; the last one with a
  // token where none is.
  int searches = 0;
  auto begin_search = [&](SampleWant how, uint32_t n, double want) {
    const uint64_t ok = __ballot(count > 0 && (how == kByCount ? my_tokens >= n : how == kReach ? my_with >= want : my_with > want));
    if (lane == 0) sh.found_bin[searches][wave] = ok ? 64 * wave + __ffsll(static_cast<unsigned long long>(ok)) - 1 : last_bin;
    return searches++;
  };
  auto end_search = [&](int search) {  // (behind a barrier)
    int bin = last_bin;
#pragma unroll
    for (int k = 0; k < kSampleThreads / 64; ++k) bin = min(bin, sh.found_bin[search][k]);
    return __builtin_amdgcn_readfirstlane(bin);
  };
  auto search_bins = [&](SampleWant how, uint32_t n, double want) {
    const int search = begin_search(how, n, want);
    __syncthreads();
    return end_search(search);
  };

  // Which bins the searches may end in: each takes the sums at the edges of the bin, or bins, of the one before.
  double lo = sh.with[last_bin], hi = lo;
  uint32_t most = sh.above[last_bin] + sh.count[last_bin], fewest = most;  // tokens
  int top_bin = kSampleBins, low_bin = -1;  // the first and the last of those of the filters
  SampleRange token_range;                  // of the token's
  struct Ends {
    int first, last;
  };
  auto search_ends = [&](SampleWant how, uint32_t n_lo, uint32_t n_hi, double want_lo, double want_hi) {
    const int f = begin_search(how, n_lo, want_lo), l = begin_search(how, n_hi, want_hi);
    __syncthreads();
    return Ends{end_search(f), end_search(l)};
  };
  auto want_bins = [&](int first, int last) {
    for (int k = first + tid; k <= last; k += kSampleThreads) sh.wanted[k] = 1;
    lo = sh.before[first], hi = sh.with[last];
    fewest = sh.above[first], most = sh.above[last] + sh.count[last];
  };
  const double least = fmin(static_cast<double>(min_p), 1.0);
  int min_bin = -1;  // the bin that the least weight falls into
  if (min_p > 0.f) {
    const double depth = grid.top == static_cast<double>(INFINITY)
                             ? 0.0
                             : grid.top - nearest_whole(static_cast<double>(b.v) * grid.per + 32.0 * log(least));
    if (depth <= static_cast<double>(last_bin)) {
      min_bin = top_bin = low_bin = static_cast<int>(depth);
      want_bins(min_bin, min_bin);
    }
  }
  if (top_k > 0 && static_cast<uint32_t>(top_k) < most) {
    const int k = search_bins(kByCount, top_k, 0.0);
    const uint32_t n = min(fewest, static_cast<uint32_t>(top_k));
    want_bins(k, k);
    fewest = n, most = top_k;
    top_bin = min(top_bin, k), low_bin = max(low_bin, k);
  }
  const double share = static_cast<double>(fmaxf(top_p, 0.f));
  if (top_p < 1.f) {
    const auto [first, last] = search_ends(kReach, 0, 0, share * lo, share * hi);
    want_bins(first, last);
    top_bin = min(top_bin, first), low_bin = max(low_bin, last);
  }
  const double part = static_cast<double>(u > 0.f ? u : 0.f);
  {
    const auto [first, last] = search_ends(u >= 1.f ? kByCount : kPass, fewest, most, part * lo, part * hi);
    want_bins(first, last);
    token_range = range_of(grid, first, last);
  }
  __syncthreads();

  // Gather them: from the chunks' lists where those hold them all, else from the row.
  const bool mine_wanted = sh.wanted[tid] != 0;
  bool listed = true;
  for (int c = 0; c < chunks; ++c) listed &= !mine_wanted || tid < sh.shift[c] + sh.covered[c];
  if (mine_wanted && count > 0) atomicAdd(&sh.n_wanted, count);
  const bool lists = __syncthreads_and(listed);
  const bool gather = sh.n_wanted <= kSampleGather;
  auto take = [&](float v, int i) {
    uint64_t m;
    const int at = sample_bin(grid, v, &m);
    if (at < 0 || !sh.wanted[at]) return;
    const uint32_t k = atomicAdd(&sh.n, 1u);
    if (k < kSampleGather) sh.key[k] = order_key(v), sh.index[k] = i, sh.bin[k] = static_cast<uint16_t>(at);
  };
  if (gather) {
    if (lists) {
#pragma unroll
      for (int k = 0; k < kSampleChunks * kSampleList / kSampleThreads; ++k) {
        const int c = (tid + k * kSampleThreads) / kSampleList;
        if (c >= chunks || tid % kSampleList >= sh.listed[c]) continue;
        const float2 e = chunk[c].list[tid % kSampleList];
        take(e.x, __float_as_int(e.y));
      }
    } else {
      each_of_row(x, vocab, token_range, low_bin >= 0 ? range_of(grid, top_bin, low_bin) : kNoRange, take);
    }
  }
  __syncthreads();
  const int held = gather ? min(sh.n, static_cast<uint32_t>(kSampleGather)) : 0;

  double total = sh.with[last_bin];
  uint32_t tokens = sh.above[last_bin] + sh.count[last_bin];
  if (min_bin >= 0) {
    // its tokens are taken by their weights in fp64
    const double inv = 1.0 / static_cast<double>(t);
    auto add = [&](float v) {
      uint64_t m;
      if (sample_bin(grid, v, &m) != min_bin) return;
      const double e = v == b.v ? 1.0 : exp((static_cast<double>(v) - static_cast<double>(b.v)) * inv);
      if (e >= least) {
        lds_add(&sh.some, m);
        atomicAdd(&sh.some_n, 1u);
      }
    };
    if (gather) {
      for (int k = tid; k < held; k += kSampleThreads)
        if (sh.bin[k] == min_bin) add(key_value(sh.key[k]));
    } else {
      each_of_row(x, vocab, range_of(grid, min_bin, min_bin), kNoRange, [&](float v, int) { add(v); });
    }
    __syncthreads();
    total = weight_up_to(sh.before[min_bin], sh.some, sh.scale[min_bin]);
    tokens = sh.above[min_bin] + sh.some_n;
  }

  // top-k, top-p, the token
#pragma unroll 1
  for (int step = 0; step < 3; ++step) {
    const SampleWant how = step == 1 ? kReach : step == 0 || u >= 1.f ? kByCount : kPass;
    const double want = (step == 1 ? share : part) * total;
    if (step == 0 && !(top_k > 0 && static_cast<uint32_t>(top_k) < tokens)) continue;
    if (step == 1 && !(top_p < 1.f)) continue;
    const uint32_t want_n = step == 0 ? static_cast<uint32_t>(top_k) : tokens;
    const int bin = search_bins(how, want_n, want);
    const double before = sh.before[bin], scale = sh.scale[bin];
    const uint32_t above = sh.above[bin];
    const bool from_row = !gather || !sh.wanted[bin];
    auto there = [&](uint32_t c, uint64_t m) {
      const double upto = weight_up_to(before, m, scale);
      return how == kByCount ? above + c >= want_n : how == kReach ? upto >= want : upto > want;
    };
    const SampleRange range = range_of(grid, bin, bin);
    // f(order key, index, mass) of the bin's tokens
    auto each = [&](auto f) {
      if (from_row) {
        each_of_row(x, vocab, range, kNoRange, [&](float v, int i) {
          uint64_t m;
          if (sample_bin(grid, v, &m) == bin) f(order_key(v), i, m);
        });
      } else {
        for (int k = tid; k < held; k += kSampleThreads)
          if (sh.bin[k] == bin) {
            uint64_t m = 0;
            sample_bin(grid, key_value(sh.key[k]), &m);
            f(sh.key[k], sh.index[k], m);
          }
      }
    };
    uint64_t base_m = 0;  // of the bin's tokens above those of [klo, khi], order keys
    uint32_t base_c = 0, n = sh.count[bin], klo = order_key(range.lo), khi = order_key(range.hi);
    while (n > kSampleRank && klo < khi) {
      const int shift = max(0, 32 - __clz(khi - klo) - 10);  // (khi - klo) >> shift < 1024
      sh.sub_mass[tid] = 0, sh.sub_count[tid] = 0;
      if (tid == 0) sh.sub = -1, sh.first = kSampleBins;
      __syncthreads();
      each([&](uint32_t k, int, uint64_t m) {
        if (k < klo || k > khi) return;
        const uint32_t s = (khi - k) >> shift;
        lds_add(&sh.sub_mass[s], m);
        atomicAdd(&sh.sub_count[s], 1u);
      });
      __syncthreads();
      const uint64_t m = sh.sub_mass[tid];
      const uint32_t c = sh.sub_count[tid];
      uint64_t im = m;
      uint32_t jc = c;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint64_t pm = __shfl_up(static_cast<unsigned long long>(im), o, kWave);
        const uint32_t pc = __shfl_up(jc, o, kWave);
        if (lane >= o) im += pm, jc += pc;
      }
      if (lane == 63) sh.scan_m[wave] = im, sh.scan_c[wave] = jc;
      __syncthreads();
      im += base_m, jc += base_c;
      for (int k = 0; k < wave; ++k) im += sh.scan_m[k], jc += sh.scan_c[k];
      // the first that is as wanted, or the last that holds any
      if (c > 0) atomicMax(&sh.sub, tid);
      if (c > 0 && there(jc, im)) atomicMin(&sh.first, tid);
      __syncthreads();
      const int sub = sh.first < kSampleBins ? sh.first : sh.sub;
      if (tid == sub) sh.some = im - m, sh.some_n = jc - c, sh.n = c;
      __syncthreads();
      base_m = sh.some, base_c = sh.some_n, n = sh.n;
      const uint64_t top = khi, from = (static_cast<uint64_t>(sub) + 1) << shift;
      klo = top + 1 > from ? max(klo, static_cast<uint32_t>(top + 1 - from)) : klo;
      khi = static_cast<uint32_t>(top - (static_cast<uint64_t>(sub) << shift));
      __syncthreads();
    }
    if (n > kSampleRank) {  // all the same
      uint64_t m1;
      sample_bin(grid, key_value(khi), &m1);
      uint32_t nth = 1;  // the least that is as wanted, by halves: `there` only ever turns true
      for (uint32_t l = 1, h = n; l < h;) {
        const uint32_t mid = l + (h - l) / 2;
        if (there(base_c + mid, base_m + mid * m1)) h = mid;
        else l = mid + 1;
        nth = l;
      }
      if (tid == 0) {
        sh.upto = weight_up_to(before, base_m + nth * m1, scale);
        sh.own = static_cast<double>(m1) * scale;
        sh.ends = above + base_c + nth;
      }
      if (step == 2) {
        const int span = (vocab + kSampleThreads - 1) / kSampleThreads, i0 = tid * span, i1 = min(i0 + span, vocab);
        const float same = key_value(khi);
        uint32_t c = 0;
        for (int i = i0; i < i1; ++i) c += x[i] == same ? 1 : 0;
        uint32_t jc = c;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const uint32_t pc = __shfl_up(jc, o, kWave);
          if (lane >= o) jc += pc;
        }
        if (lane == 63) sh.scan_c[wave] = jc;
        __syncthreads();
        for (int k = 0; k < wave; ++k) jc += sh.scan_c[k];
        if (jc - c < nth && nth <= jc) {
          uint32_t left = nth - (jc - c);
          for (int i = i0; i < i1; ++i)
            if (x[i] == same && --left == 0) {
              sh.found = i;
              break;
            }
        }
      }
    } else {
      if (tid == 0) sh.n = 0;
      if (tid < kSampleRank) sh.rank[tid] = SampleToken{0, 0};
      __syncthreads();
      each([&](uint32_t k, int i, uint64_t m) {
        if (k < klo || k > khi) return;
        const uint32_t at = atomicAdd(&sh.n, 1u);
        if (at < kSampleRank) sh.rank[at] = SampleToken{static_cast<uint64_t>(k) << 32 | ~static_cast<uint32_t>(i), m};
      });
      __syncthreads();
      const int have = min(sh.n, static_cast<uint32_t>(kSampleRank));
      if (tid < have) {
        const uint64_t place = sh.rank[tid].place, own = sh.rank[tid].mass;
        uint64_t m = base_m;
        uint32_t rank = 0;
        for (int j = 0; j < have; j += kSampleRankStep) {
          SampleToken other[kSampleRankStep];
#pragma unroll
          for (int e = 0; e < kSampleRankStep; ++e) other[e] = sh.rank[j + e];
#pragma unroll
          for (int e = 0; e < kSampleRankStep; ++e) {
            const bool higher = other[e].place > place;
            m += higher ? other[e].mass : 0;
            rank += higher ? 1 : 0;
          }
        }
        // the first that is as wanted, or the last
        const bool ok = there(base_c + rank + 1, m + own);
        if (ok ? rank == 0 || !there(base_c + rank, m) : static_cast<int>(rank) == have - 1) {
          sh.upto = weight_up_to(before, m + own, scale);
          sh.own = static_cast<double>(own) * scale;
          sh.found = static_cast<int>(~static_cast<uint32_t>(place));
          sh.ends = above + base_c + rank + 1;
        }
      }
    }
    __syncthreads();
    // (the next step writes them behind its search's barrier)
    if (step < 2) total = fmin(total, sh.upto), tokens = min(tokens, sh.ends);
  }
  if (tid == 0) {
    a.out[row] = sh.found;
    if (a.prob) a.prob[row] = static_cast<float>(sh.own / total);
  }
}

static int sample_chunks(int vocab) { return (vocab + kSampleChunk - 1) / kSampleChunk; }

int64_t sample_workspace(int rows, int vocab) {
  return static_cast<int64_t>(rows) * sample_chunks(vocab) * static_cast<int64_t>(sizeof(SampleChunk));
}

hipError_t launch_sample(const SampleArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  const int chunks = sample_chunks(a.vocab);
  launch_kernel(sample_chunk_kernel, dim3(a.rows * chunks), dim3(kSampleThreads), 0, s, a, chunks);
  launch_kernel(sample_kernel, dim3(a.rows), dim3(kSampleThreads), 0, s, a, chunks);
  return hipGetLastError();
}

}  // namespace metro
