// Sampled choice of a token (gfx950, wave64).
//
// A row's tokens stand in the order of falling logits, ties by rising index, with
// weights w = exp((x - max) / T).  min-p takes away the weights below min_p, top-k
// all but the first k, top-p all but the shortest beginning that holds top_p of
// what is left; the token is the first whose weights up to it pass u times the
// weights that are left.  All three leave a beginning of the order, so the steps
// need nothing but searches of the running sums of weights and of counts.
//
// A search goes by a histogram.  Bins are the whole numbers of t = 32 x / T, the
// same for every part of a row, counted down from the row's largest; 1024 of them
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
#include "common.h"
#include "kernels.h"
#include "kernels_draft.h"

namespace metro {

constexpr int kSampleThreads = 1024;
constexpr int kSampleBins = 1024;
constexpr int kSampleChunk = 16384;  // logits of a workgroup, 16 a thread
constexpr int kSampleList = 256;     // tokens that are listed, and that are ranked by comparing all pairs
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

// The bins' grid: t = x * per; top is the bin of the largest logit (infinite with it).
struct SampleGrid {
  double per, top;
};

__device__ __forceinline__ SampleGrid sample_grid(float max, float t) {
  SampleGrid g;
  g.per = 32.0 / static_cast<double>(t);
  g.top = max == INFINITY ? static_cast<double>(INFINITY) : floor(static_cast<double>(max) * g.per);
  return g;
}

// Bin of a logit below the top one, or -1 where its weight counts as none; *mass: its weight relative to the bin's upper
// edge in units of 2^-34.  The adding of 2^18 leaves 34 bits behind the point in a double's mantissa, rounded to nearest.
__device__ __forceinline__ int sample_bin(const SampleGrid& grid, float x, uint64_t* mass) {
  if (grid.top == static_cast<double>(INFINITY)) {
    *mass = 1ull << 34;
    return x == INFINITY ? 0 : -1;
  }
  const double t = static_cast<double>(x) * grid.per, whole = floor(t);
  const double below = grid.top - whole;
  if (!(below < static_cast<double>(kSampleBins))) return -1;  // (NaN and -inf too)
  const double g = (t - whole - 1.0) * (1.0 / 32.0);           // -1/32 .. 0; the next term of the series is below 2^-39
  double e = fma(g, 1.0 / 120.0, 1.0 / 24.0);
  e = fma(e, g, 1.0 / 6.0);
  e = fma(e, g, 0.5);
  e = fma(e, g, 1.0);
  e = fma(e, g, 1.0);
  *mass = __double_as_longlong(e + 262144.0) & ((1ull << 52) - 1);
  return static_cast<int>(below);
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

__global__ __launch_bounds__(kSampleThreads) void sample_chunk_kernel(SampleArgs a, int chunks) {
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
  for (int j = 0; j < V; ++j)
    if (v[j] > b.v) b = SampleBest{v[j], first + j / 4 * 4 * kSampleThreads + j % 4};
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) b = best_of(b, SampleBest{__shfl_xor(b.v, o, kWave), __shfl_xor(b.i, o, kWave)});
  if (lane == 0) best[wave] = b;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSampleThreads / 64; ++w) b = best_of(b, best[w]);
  SampleChunk* out = reinterpret_cast<SampleChunk*>(a.ws) + blockIdx.x;
  if (tid == 0) out->max = b.v, out->index = b.i;
  if (!(t > 0.f) || !(b.v > -INFINITY)) return;  // (greedy, or nothing to choose: the rest is not read)
  const SampleGrid grid = sample_grid(b.v, t);
  int at[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    uint64_t mass;
    at[j] = sample_bin(grid, v[j], &mass);
    if (at[j] >= 0) lds_add(&bin[at[j]], mass + (1ull << kMassBits));
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
#pragma unroll
  for (int j = 0; j < V; ++j)
    if (at[j] >= 0 && at[j] < covered)
      out->list[atomicAdd(&n_list, 1)] = make_float2(v[j], __int_as_float(first + j / 4 * 4 * kSampleThreads + j % 4));
  __syncthreads();
  if (tid == 0) out->covered = covered, out->listed = n_list;
}

struct SampleShared {
  double before[kSampleBins], with[kSampleBins];  // weight of the bins above, and with this one
  uint32_t count[kSampleBins], above[kSampleBins];  // tokens of a bin, and of the bins above
  double scan_w[16];
  uint32_t scan_c[16];
  uint64_t sub_mass[kSampleBins];
  uint32_t sub_count[kSampleBins];
  uint64_t scan_m[16];
  uint32_t key[kSampleList];
  int index[kSampleList];
  uint64_t weight[kSampleList];
  uint32_t n_list, key_lo, key_hi;
  int bin, sub;
  // what a search leaves: the sums up to the token and with it, the token's own weight and index
  double upto;
  uint64_t some;
  uint32_t tokens, some_n;
  double own;
  int found;
  int shift[kSampleChunks];  // bins between the row's largest and a chunk's, or so many that it has none
  int covered[kSampleChunks];  // bins of a chunk whose tokens are listed
};

enum SampleWant { kByCount, kReach, kPass };  // the first token whose count, or weight, up to it reaches, or passes, the wanted

struct SampleRow {
  const float* x;
  const SampleChunk* chunk;
  int vocab, chunks, last_bin;
  SampleGrid grid;

  // the listed tokens of all chunks, four a thread (absent ones NaN)
  static constexpr int L = kSampleChunks * kSampleList / kSampleThreads;
  float listed[L];
  int listed_at[L];

  // f(logit, index) of the tokens that may be in a bin: the listed ones, where they hold all of it, else the row's.
  template <typename F>
  __device__ __forceinline__ void each(bool lists, F f) const {
    if (lists) {
#pragma unroll
      for (int k = 0; k < L; ++k) f(listed[k], listed_at[k]);
      return;
    }
    const int head = min(static_cast<int>(((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / 4), vocab);
    const int n4 = (vocab - head) / 4, tail = head + 4 * n4;
    if (static_cast<int>(threadIdx.x) < head) f(x[threadIdx.x], threadIdx.x);
    if (static_cast<int>(threadIdx.x) < vocab - tail) f(x[tail + threadIdx.x], tail + threadIdx.x);
    const float4* x4 = reinterpret_cast<const float4*>(x + head);
    constexpr int U = 4;
    for (int j0 = threadIdx.x; j0 < n4; j0 += U * kSampleThreads) {
      float4 w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) w[u] = x4[min(j0 + u * kSampleThreads, n4 - 1)];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int j = j0 + u * kSampleThreads, i = head + 4 * j;
        if (j >= n4) continue;
        f(w[u].x, i);
        f(w[u].y, i + 1);
        f(w[u].z, i + 2);
        f(w[u].w, i + 3);
      }
    }
  }
  // whether every chunk lists its tokens of bin b
  __device__ __forceinline__ bool at_hand(const SampleShared& sh, int b) const {
    bool all = true;
    for (int c = 0; c < chunks; ++c) all &= b < sh.shift[c] + sh.covered[c];
    return all;
  }
};

__device__ __forceinline__ double bin_scale(int b) { return exp(-b / 32.0) / kMassOne; }

// The first token of the order whose count or weight up to it is as wanted; the last one where none is (a sum's rounding).
__device__ void locate(SampleShared& sh, const SampleRow& r, SampleWant how, uint32_t count, double want, bool index) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) sh.bin = r.last_bin;
  __syncthreads();
  {
    const double upto = sh.with[tid];
    const bool ok = how == kByCount ? sh.above[tid] + sh.count[tid] >= count : how == kReach ? upto >= want : upto > want;
    if (sh.count[tid] > 0 && ok) atomicMin(&sh.bin, tid);
  }
  __syncthreads();
  const int bin = sh.bin;
  const double before = sh.before[bin], scale = bin_scale(bin);
  const uint32_t above = sh.above[bin];
  const bool lists = r.at_hand(sh, bin);
  auto there = [&](uint32_t c, uint64_t m) {
    const double upto = before + static_cast<double>(m) * scale;
    return how == kByCount ? above + c >= count : how == kReach ? upto >= want : upto > want;
  };
  uint64_t base_m = 0;  // of the bin's tokens above those of [lo, hi]
  uint32_t base_c = 0, n = sh.count[bin], lo = 0, hi = 0xffffffffu;
  auto mine = [&](float x, uint64_t* m) {
    const uint32_t k = order_key(x);
    return k >= lo && k <= hi && sample_bin(r.grid, x, m) == bin;
  };
  if (n > kSampleList) {
    if (tid == 0) sh.key_lo = 0xffffffffu, sh.key_hi = 0;
    __syncthreads();
    uint32_t l = 0xffffffffu, u = 0;
    r.each(lists, [&](float x, int) {
      uint64_t m;
      if (mine(x, &m)) l = min(l, order_key(x)), u = max(u, order_key(x));
    });
    atomicMin(&sh.key_lo, l);
    atomicMax(&sh.key_hi, u);
    __syncthreads();
    lo = sh.key_lo, hi = sh.key_hi;
  }
  while (n > kSampleList && lo < hi) {
    const int shift = max(0, 32 - __clz(hi - lo) - 10);  // (hi - lo) >> shift < 1024
    __syncthreads();
    sh.sub_mass[tid] = 0, sh.sub_count[tid] = 0;
    __syncthreads();
    r.each(lists, [&](float x, int) {
      uint64_t m;
      if (!mine(x, &m)) return;
      const uint32_t b = (hi - order_key(x)) >> shift;
      lds_add(&sh.sub_mass[b], m);
      atomicAdd(&sh.sub_count[b], 1u);
    });
    if (tid == 0) sh.sub = -1;
    __syncthreads();
    const uint64_t m = sh.sub_mass[tid];
    const uint32_t c = sh.sub_count[tid];
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
    im += base_m, ic += base_c;
    for (int w = 0; w < wave; ++w) im += sh.scan_m[w], ic += sh.scan_c[w];
    // the first that is as wanted, or the last that holds any
    const bool first = c > 0 && there(ic, im) && (ic - c == base_c || !there(ic - c, im - m));
    if (c > 0) atomicMax(&sh.sub, tid);
    __syncthreads();
    if (first) sh.sub = -2 - tid;
    __syncthreads();
    const int sub = sh.sub <= -2 ? -2 - sh.sub : sh.sub;
    __syncthreads();
    if (tid == sub) sh.some = im - m, sh.some_n = ic - c;
    __syncthreads();
    base_m = sh.some, base_c = sh.some_n, n = sh.sub_count[sub];
    const uint64_t top = hi, from = (static_cast<uint64_t>(sub) + 1) << shift;
    lo = top + 1 > from ? max(lo, static_cast<uint32_t>(top + 1 - from)) : lo;
    hi = static_cast<uint32_t>(top - (static_cast<uint64_t>(sub) << shift));
  }
  __syncthreads();
  if (n > kSampleList) {  // all the same
    uint64_t w;
    sample_bin(r.grid, key_value(hi), &w);
    uint32_t nth = 1;  // the least that is as wanted, by halves: `there` only ever turns true
    for (uint32_t l = 1, h = n; l < h;) {
      const uint32_t mid = l + (h - l) / 2;
      if (there(base_c + mid, base_m + mid * w)) h = mid;
      else l = mid + 1;
      nth = l;
    }
    if (tid == 0) {
      sh.upto = before + static_cast<double>(base_m + nth * w) * scale;
      sh.tokens = above + base_c + nth;
      sh.own = static_cast<double>(w) * scale;
    }
    if (index) {
      const int chunk = (r.vocab + kSampleThreads - 1) / kSampleThreads, i0 = tid * chunk, i1 = min(i0 + chunk, r.vocab);
      const float same = key_value(hi);
      uint32_t c = 0;
      for (int i = i0; i < i1; ++i) c += r.x[i] == same ? 1 : 0;
      uint32_t ic = c;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t pc = __shfl_up(ic, o, kWave);
        if (lane >= o) ic += pc;
      }
      if (lane == 63) sh.scan_c[wave] = ic;
      __syncthreads();
      for (int k = 0; k < wave; ++k) ic += sh.scan_c[k];
      if (ic - c < nth && nth <= ic) {
        uint32_t left = nth - (ic - c);
        for (int i = i0; i < i1; ++i)
          if (r.x[i] == same && --left == 0) {
            sh.found = i;
            break;
          }
      }
    }
    __syncthreads();
    return;
  }
  if (tid == 0) sh.n_list = 0;
  __syncthreads();
  r.each(lists, [&](float x, int i) {
    uint64_t m;
    if (!mine(x, &m)) return;
    const uint32_t at = atomicAdd(&sh.n_list, 1u);
    if (at < kSampleList) sh.key[at] = order_key(x), sh.index[at] = i, sh.weight[at] = m;
  });
  __syncthreads();
  const int have = min(sh.n_list, static_cast<uint32_t>(kSampleList));
  if (tid < have) {
    const uint32_t key = sh.key[tid];
    const int at = sh.index[tid];
    const uint64_t w = sh.weight[tid];
    uint64_t m = base_m;
    uint32_t c = base_c, rank = 0;
    for (int j = 0; j < have; ++j) {
      const uint32_t k = sh.key[j];
      if (k > key || (k == key && sh.index[j] < at)) m += sh.weight[j], ++rank;
    }
    c += rank;
    // the first that is as wanted, or the last
    const bool ok = there(c + 1, m + w);
    if ((ok && (rank == 0 || !there(c, m))) || (!ok && static_cast<int>(rank) == have - 1)) {
      sh.upto = before + static_cast<double>(m + w) * scale;
      sh.tokens = above + c + 1;
      sh.own = static_cast<double>(w) * scale;
      sh.found = at;
    }
  }
  __syncthreads();
}

__global__ __launch_bounds__(kSampleThreads) void sample_kernel(SampleArgs a, int chunks) {
  __shared__ SampleShared sh;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  SampleRow r;
  r.x = a.logits + static_cast<size_t>(row) * a.ldl;
  r.chunk = reinterpret_cast<const SampleChunk*>(a.ws) + static_cast<size_t>(row) * chunks;
  r.vocab = a.vocab, r.chunks = chunks;
  const SampleChunk& own_chunk = r.chunk[min(lane % kSampleChunks, chunks - 1)];
  SampleBest b{own_chunk.max, own_chunk.index};
  const float chunk_max = b.v;
#pragma unroll
  for (int o = kSampleChunks / 2; o > 0; o >>= 1) b = best_of(b, SampleBest{__shfl_xor(b.v, o, kWave), __shfl_xor(b.i, o, kWave)});
  const float t = a.temperature ? a.temperature[row] : 1.f;
  if (!(b.v > -INFINITY) || !(t > 0.f)) {
    if (tid == 0) {
      a.out[row] = b.v > -INFINITY ? b.i : -1;
      if (a.prob) a.prob[row] = b.v > -INFINITY ? 1.f : 0.f;
    }
    return;
  }
  r.grid = sample_grid(b.v, t);
  if (tid < chunks) {
    // (an infinite difference, or that of infinities: all of the chunk or nothing)
    const double d = chunk_max == b.v ? 0.0 : r.grid.top - sample_grid(chunk_max, t).top;
    const bool any = chunk_max > -INFINITY && d < static_cast<double>(kSampleBins);
    sh.shift[tid] = any ? static_cast<int>(d) : kSampleBins;
    sh.covered[tid] = any ? own_chunk.covered : 0;
  }
#pragma unroll
  for (int k = 0; k < SampleRow::L; ++k) {
    const int at = tid + k * kSampleThreads, c = at / kSampleList;
    const SampleChunk& from = r.chunk[min(c, chunks - 1)];
    const bool on = c < chunks && from.max > -INFINITY && at % kSampleList < from.listed;
    const float2 e = on ? from.list[at % kSampleList] : make_float2(__builtin_nanf(""), 0.f);
    r.listed[k] = e.x;
    r.listed_at[k] = __float_as_int(e.y);
  }
  __syncthreads();
  // the row's histogram and its running sums
  uint64_t mass = 0;
  uint32_t count = 0;
#pragma unroll 8
  for (int c = 0; c < chunks; ++c) {
    const int at = tid - sh.shift[c];
    uint64_t v = r.chunk[c].bin[max(at, 0)];
    v = at < 0 ? 0 : v;
    mass += v & kMassMask;
    count += static_cast<uint32_t>(v >> kMassBits);
  }
  const double w = static_cast<double>(mass) * bin_scale(tid);
  double iw = w;
  uint32_t ic = count;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double pw = __shfl_up(iw, o, kWave);
    const uint32_t pc = __shfl_up(ic, o, kWave);
    if (lane >= o) iw += pw, ic += pc;
  }
  if (lane == 63) sh.scan_w[wave] = iw, sh.scan_c[wave] = ic;
  // (the sum before a bin is that of its lower neighbours' lanes, not the sum with it less its own)
  double bw = __shfl_up(iw, 1, kWave);
  if (lane == 0) bw = 0.0;
  if (tid == 0) sh.bin = 0;
  __syncthreads();
  double head = 0.0;
  uint32_t bc = ic - count;
  for (int k = 0; k < wave; ++k) head += sh.scan_w[k], bc += sh.scan_c[k];
  sh.before[tid] = head + bw;
  sh.with[tid] = (head + bw) + w;
  sh.above[tid] = bc;
  sh.count[tid] = count;
  if (count > 0) atomicMax(&sh.bin, tid);
  __syncthreads();
  r.last_bin = sh.bin;
  double total = sh.with[r.last_bin];
  uint32_t tokens = sh.above[r.last_bin] + sh.count[r.last_bin];
  __syncthreads();

  const float min_p = a.min_p ? a.min_p[row] : 0.f, top_p = a.top_p ? a.top_p[row] : 1.f;
  const int top_k = a.top_k ? a.top_k[row] : 0;
  if (min_p > 0.f) {
    // the bin that the least weight falls into; its tokens are taken by their weights in fp64
    const double least = fmin(static_cast<double>(min_p), 1.0), inv = 1.0 / static_cast<double>(t);
    const double depth = r.grid.top == static_cast<double>(INFINITY)
                             ? 0.0
                             : r.grid.top - floor(static_cast<double>(b.v) * r.grid.per + 32.0 * log(least));
    if (depth < static_cast<double>(kSampleBins) && static_cast<int>(depth) <= r.last_bin) {
      const int bin = static_cast<int>(depth);
      if (tid == 0) sh.some = 0, sh.some_n = 0;
      __syncthreads();
      const bool lists = r.at_hand(sh, bin);
      uint64_t m_sum = 0;
      uint32_t n = 0;
      r.each(lists, [&](float x, int) {
        uint64_t m;
        if (sample_bin(r.grid, x, &m) != bin) return;
        const double e = x == b.v ? 1.0 : exp((static_cast<double>(x) - static_cast<double>(b.v)) * inv);
        if (e >= least) m_sum += m, ++n;
      });
      if (n > 0) {
        lds_add(&sh.some, m_sum);
        atomicAdd(&sh.some_n, n);
      }
      __syncthreads();
      total = sh.before[bin] + static_cast<double>(sh.some) * bin_scale(bin);
      tokens = sh.above[bin] + sh.some_n;
      __syncthreads();
    }
  }
  if (top_k > 0 && static_cast<uint32_t>(top_k) < tokens) {
    locate(sh, r, kByCount, top_k, 0.0, false);
    total = sh.upto;
    __syncthreads();
  }
  if (top_p < 1.f) {
    locate(sh, r, kReach, 0, static_cast<double>(fmaxf(top_p, 0.f)) * total, false);
    total = fmin(total, sh.upto);
    __syncthreads();
  }
  // u from 1 on: the last kept token, the first whose sum reaches all of it
  const float u = a.u[row];
  if (u >= 1.f)
    locate(sh, r, kReach, 0, total, true);
  else
    locate(sh, r, kPass, 0, static_cast<double>(u > 0.f ? u : 0.f) * total, true);
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
