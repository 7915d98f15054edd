// 8-bit products on the matrix cores of gfx950 (v_mfma_scale_f32_16x16x128_f8f6f4,
// fp32 accumulation):  acc[m, n] = sum over blocks kb of 128 columns of
// 2^(sx[m, kb] + sw[n, kb] - 254) * sum_k X[m, k] W[n, k], dense or with the rows of
// each expert against its own W, then bf16 rows or SwiGLU and 8-bit rows.
//
// One instruction takes 16 rows of W (A), 16 rows of X (B) and 128 columns, and
// applies both rows' powers of two itself.  Lane l = 16 g + r supplies 32
// columns of W row r and X row r and one byte of power for each, and receives
// D[4 g + i][r]: four consecutive W rows of X row r.
//
// Precision: accumulators are fp32.  Within one instruction the products of
// each run of eight columns are aligned to the largest of them and cut below
// 2^-13 of it: 1.5e-5 of the result's 2-norm on normal data (2.6e-5 where X is
// a product of normals), against 1.7e-3 that the rounding to bf16 adds behind it.
#include <algorithm>
#include <cmath>
#include <type_traits>
#include <utility>

#include "fp8.h"
#include "kernels_fp8.h"

namespace metro {

namespace {

constexpr int kSlices = 3;  // epilogue of a k slice: its fp32 sums

__device__ __forceinline__ f32x4 mfma8(uint4 a0, uint4 a1, uint4 b0, uint4 b1, f32x4 c, int sa, int sb) {
  const i32x8 a = {static_cast<int>(a0.x), static_cast<int>(a0.y), static_cast<int>(a0.z), static_cast<int>(a0.w),
                   static_cast<int>(a1.x), static_cast<int>(a1.y), static_cast<int>(a1.z), static_cast<int>(a1.w)};
  const i32x8 b = {static_cast<int>(b0.x), static_cast<int>(b0.y), static_cast<int>(b0.z), static_cast<int>(b0.w),
                   static_cast<int>(b1.x), static_cast<int>(b1.y), static_cast<int>(b1.z), static_cast<int>(b1.w)};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb);
}

// z / (1 + exp(-z)) by the hardware's 2^x and reciprocal (an ulp each; the
// product with log2(e) is off by |z| / 2 ulp of the exponent's result): far below
// the step of the e4m3 value that it ends in, at a fifth of expf's and the
// division's instructions.  The reciprocal flushes what is below 2^-126, so gates
// below -87.33 (ln 2^126) give 0, as the operator's definition says.  (Their
// products in two factors, behind a look at every tile's deepest gate, cost 8192 x
// 28672 x 4096 729 -> 735 us and 8 spilled registers.)
__device__ __forceinline__ float silu_f32(float z) {
  return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
}

// Rows m0 .. m1 - 1 of row block b of BM rows, and their expert.  By experts,
// every expert's rows are cut into blocks of their own; offsets are held within
// 0 .. M, so that whatever they say, rows lie in range.  False: no such block.
__device__ __forceinline__ bool row_block(const GemmFp8Args& a, int b, int BM, int& e, int& m0, int& m1) {
  if (!a.offsets) {
    e = 0;
    m0 = b * BM;
    m1 = min(m0 + BM, a.M);
    return m0 < a.M;
  }
  const int lane = threadIdx.x & 63;
  int carry = 0;
  for (int c = 0; c < a.E; c += 64) {
    const int i = c + lane;
    const int lo = i < a.E ? min(max(a.offsets[i], 0), a.M) : 0;
    const int hi = i < a.E ? min(max(a.offsets[i + 1], 0), a.M) : 0;
    const int nb = (max(hi - lo, 0) + BM - 1) / BM;
    int incl = nb;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int y = __shfl_up(incl, o);
      if (lane >= o) incl += y;
    }
    const int first = carry + incl - nb;
    const uint64_t here = __ballot(b >= first && b < first + nb);
    if (here) {
      const int l = __builtin_ctzll(here);
      e = c + l;
      m0 = __builtin_amdgcn_readlane(lo, l) + (b - __builtin_amdgcn_readlane(first, l)) * BM;
      m1 = min(m0 + BM, __builtin_amdgcn_readlane(hi, l));
      return true;
    }
    carry += __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

// all row blocks of BM rows
__device__ __forceinline__ int total_row_blocks(const GemmFp8Args& a, int BM) {
  if (!a.offsets) return (a.M + BM - 1) / BM;
  const int lane = threadIdx.x & 63;
  int n = 0;
  for (int i = lane; i < a.E; i += 64) {
    const int lo = min(max(a.offsets[i], 0), a.M), hi = min(max(a.offsets[i + 1], 0), a.M);
    n += (max(hi - lo, 0) + BM - 1) / BM;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o);
  return __builtin_amdgcn_readfirstlane(n);
}

// row of X that slot m reads (indexes are held within x_rows)
__device__ __forceinline__ int64_t source_row(const GemmFp8Args& a, int m) {
  return a.src ? min(max(a.src[m], 0), a.x_rows - 1) : m;
}

// ---------------------------------------------------------------------------
// Tiled kernel: 4 waves, one per SIMD (2 x 2, each 16 TN rows of W x 16 TM rows of
// X); operands come through LDS in stages of 128 columns, one per instruction.
//
// A stage's work is cut in two halves of TN / 2 row tiles of W.  LDS rings hold
// chunks: the W rows of one half (of both wave rows), and half the X rows of a
// stage.  During half h = 2 s + p the wave multiplies from registers, reads the W
// fragments of half h + 1 and half of the X fragments of stage s + 1 (chunk h + 2),
// and requests chunk h + D of both, into slots whose last reads lie behind the
// previous barrier (W ring of D chunks, X ring of D - 1).  The barrier that ends
// the half stands for: W chunk h + 2 and X chunk h + 3 have landed, and what this
// half read is in registers.  Every memory instruction rides behind a matrix
// instruction.  Scales: four stages' bytes of a row are one word; they have a ring
// of their own of two groups of four stages, requested four stages ahead.
// ---------------------------------------------------------------------------
template <int TN_, int TM_, int D_ = 5>
struct TileShape8 {
  static constexpr int TN = TN_, TM = TM_, D = D_;
  static constexpr int BN = 32 * TN, BM = 32 * TM;
  static constexpr int WR = D, XR = D - 1;
  static constexpr int kW = TN * 2048, kX = TM * 2048;  // bytes of a chunk
  static constexpr int LW = TN / 2, LX = TM / 2;        // wave loads of a chunk, per wave
  static constexpr int kYoung = (D - 2) * LW + (D - 3) * LX;  // loads that may be under way at a barrier
  static constexpr int kScales = 4 * (BN + BM);         // bytes of a group of four stages
  static constexpr int kLds = WR * kW + XR * kX + 2 * kScales;
  static constexpr int OCC = kLds <= 80 * 1024 ? 2 : 1;
  static_assert(TN % 4 == 0 && TM % 2 == 0, "halves and fragments are shared evenly");
  static_assert(D >= 4 && kYoung < 63 && kLds <= 160 * 1024, "the ring's loads can be counted and held");
};

// c += a . b scaled by 2^(sa - 127 + sb - 127) (lowest bytes), the accumulator in
// place.  The compiler does not see these instructions' hazards: no operand is
// written by a vector instruction within two wait states of one, and the
// accumulators are read behind drained_barrier.
__device__ __forceinline__ void mfma8_acc(f32x4& c, i32x8 a, i32x8 b, int sa, int sb) {
  asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]"
               : "+a"(c)
               : "v"(a), "v"(b), "v"(sa), "v"(sb));
}
// The same with a direct load of 16 bytes per lane into LDS bytes lds_base + INC +
// 16 * lane behind it (NT: of data that nobody reads again soon); the matrix
// instruction is the wait state between the M0 write and the load.
template <int INC, bool NT>
__device__ __forceinline__ void mfma8_acc_load(f32x4& c, i32x8 a, i32x8 b, int sa, int sb, const void* base,
                                               uint32_t off, uint32_t lds_base) {
#define METRO_MFMA8_LOAD(HINT)                                                                                      \
  asm volatile(                                                                                                     \
      "s_add_u32 m0, %5, %6\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]\n\t"       \
      "global_load_lds_dwordx4 %7, %8" HINT                                                                         \
      : "+a"(c)                                                                                                     \
      : "v"(a), "v"(b), "v"(sa), "v"(sb), "s"(lds_base), "n"(INC), "v"(off), "s"(base)                               \
      : "memory", "m0", "scc")
  if constexpr (NT)
    METRO_MFMA8_LOAD(" nt");
  else
    METRO_MFMA8_LOAD("");
#undef METRO_MFMA8_LOAD
}
// 4 bytes per lane into LDS bytes lds_base + 4 * lane
__device__ __forceinline__ void lds_load4s(const void* base, uint32_t off, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(off), "s"(base), "s"(lds_base)
               : "memory", "m0");
}
// The end of a half: what it read from LDS is in registers everywhere.
__device__ __forceinline__ void half_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
// The end of a stage: also 8 wait states, behind which the last matrix
// instruction's accumulator may be read (the loop may end here) and the scales
// that vector instructions shifted may be operands.  (Behind both halves of a stage
// it cost 1.5% at 8192 x 28672 x 16384.)
__device__ __forceinline__ void drained_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_nop 7\n\ts_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// first of the n memory operations that ride behind instruction u of nm, spread
// evenly (those before instruction u: first_of(u + 1) is the end of its own)
constexpr int first_of(int u, int nm, int n) { return (u * n + nm - 1) / nm; }

// Work item of workgroup b (of `total`) such that each of the 8 XCDs, which take
// workgroups in turn and have an L2 each, gets a contiguous run of the list.
__device__ __forceinline__ int xcd_run(int b, int total) {
  constexpr int kXcds = 8;
  const int q = total / kXcds, r = total % kXcds, x = b % kXcds, s = b / kXcds;
  return x * q + min(x, r) + s;
}

// Tile t of mb row blocks x nb column tiles: groups of GM row blocks, rows
// fastest within a group, so that tiles in flight share X and W tiles: an XCD's 32
// 256 x 256 tiles cover 8 x 4.  (GM 2 / 4 / 8 / 16, us: 8192 x 28672 x 4096 757 / 735 /
// 723 / 756; eight experts' down of 8192 rows 454 / 434 / 425 / 429; QKV at 301 rows in
// blocks of 64 16.8 / 16.1 / 14.6 / 14.5.)
constexpr int kGroupRows = 8;
template <int GM>
__device__ __forceinline__ void tile_at(int t, int mb, int nb, int& bm, int& bn) {
  const int group = t / (GM * nb), first = group * GM, gm = min(mb - first, GM), in = t % (GM * nb);
  bn = in / gm;
  bm = first + in % gm;
}

// 4 x 4 transposition of words over the lanes r + 16 g: word p of lane group g
// becomes word g of lane group p
__device__ __forceinline__ void transpose4(uint32_t (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const auto t = __builtin_amdgcn_permlane32_swap(v[i], v[i + 2], false, false);
    v[i] = t[0];
    v[i + 2] = t[1];
  }
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    const auto t = __builtin_amdgcn_permlane16_swap(v[i], v[i + 1], false, false);
    v[i] = t[0];
    v[i + 1] = t[1];
  }
}

// k slice y of ks: whole groups of four 128-column blocks
struct KSpan {
  int first, blocks;
};
__device__ __forceinline__ KSpan k_span(int nk, int ks, int y) {
  const int units = (nk + 3) / 4, lo = units * y / ks * 4, hi = units * (y + 1) / ks * 4;
  return {lo, min(hi, nk) - lo};
}

// EPI: kEpi8Bf16, kEpi8SwiGLU or kSlices: the grid's ks k slices leave their
// fp32 sums in ws[slice][m][n] for gemm_fp8_finish_kernel.  NT: W passes the
// caches by (plan_gemm_fp8 says when).
template <class S, int EPI, bool NT>
__global__ __launch_bounds__(256, S::OCC) void gemm_fp8_tiled_kernel(GemmFp8Args a, int ks) {
  constexpr int TN = S::TN, TM = S::TM, HN = TN / 2, HM = TM / 2, LW = S::LW, LX = S::LX;
  __shared__ uint4 lds[S::kLds / 16];
  const int nb = (a.N + S::BN - 1) / S::BN;
  const int mb = total_row_blocks(a, S::BM);
  const int items = mb * nb * ks;
  if (static_cast<int>(blockIdx.x) >= items) return;
  int bm, bn, e, m0, m1;
  const int item = xcd_run(blockIdx.x, items);
  const int slice = item / (mb * nb);
  tile_at<kGroupRows>(item % (mb * nb), mb, nb, bm, bn);
  if (!row_block(a, bm, S::BM, e, m0, m1)) return;
  e = __builtin_amdgcn_readfirstlane(e);
  m0 = __builtin_amdgcn_readfirstlane(m0);
  m1 = __builtin_amdgcn_readfirstlane(m1);
  const int n0 = bn * S::BN;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wn = wave >> 1, wm = wave & 1;
  const int r16 = lane & 15, g = lane >> 4;
  const int groups = padded_groups(a.Kp);
  const KSpan span = k_span(a.Kp / kGroup, ks, slice);
  const int nk = span.blocks;

  // Loads of a chunk: W chunk p of a stage has tiles wn' * HN + i of wave row wn',
  // two KiB halves each; X chunk p has rows 16 (wm' TM + p HM) .. of wave column
  // wm', in blocks of 8.  Tiles and rows past the ends re-read the last ones,
  // whose products only reach outputs that are not stored.
  const char* const wbase = reinterpret_cast<const char*>(a.W) + static_cast<int64_t>(e) * a.N * a.Kp +
                            static_cast<int64_t>(n0) * a.Kp + span.first * 2048;
  const int64_t xrow0 = a.src ? 0 : m0;
  const char* const xbase = reinterpret_cast<const char*>(a.X) + xrow0 * a.ldx + span.first * kGroup;
  uint32_t woff[2][LW], xoff[2][LX];
#pragma unroll
  for (int p = 0; p < 2; ++p) {
#pragma unroll
    for (int j = 0; j < LW; ++j) {
      const int u = wave * LW + j, t = u >> 1;  // half-tile u of 2 TN
      const int tile = min((t / HN) * TN + p * HN + t % HN, a.N / 16 - 1 - n0 / 16);
      woff[p][j] = static_cast<uint32_t>(tile) * (a.Kp * 16) + (u & 1) * 1024 + lane * 16;
    }
#pragma unroll
    for (int j = 0; j < LX; ++j) {
      const int u = wave * LX + j, t = u >> 1;  // block of 8 rows u of 2 TM
      const int row = 16 * ((t / HM) * TM + p * HM + t % HM) + 8 * (u & 1) + (lane >> 3);
      const int m = min(m0 + row, m1 - 1);
      xoff[p][j] = static_cast<uint32_t>(source_row(a, m) - xrow0) * static_cast<uint32_t>(a.ldx) +
                   16 * ((lane & 7) ^ (lane >> 3));
    }
  }
  const uint32_t lds0 = lds_address(lds);
  constexpr uint32_t kXAt = S::WR * S::kW, kSAt = kXAt + S::XR * S::kX;
  const uint32_t wdst = lds0 + wave * LW * 1024, xdst = lds0 + kXAt + wave * LX * 1024;
  // scales: a wave loads words of 64 W rows and of 64 X rows of a group
  const char* const wsbase = reinterpret_cast<const char*>(a.w_scale) + static_cast<int64_t>(e) * a.N * groups +
                             span.first * 16;
  const char* const xsbase = reinterpret_cast<const char*>(a.x_scale) + xrow0 * a.ldxs + span.first;
  const int ws64 = wave % (S::BN / 64), xs64 = wave % (S::BM / 64);
  const uint32_t wsoff = static_cast<uint32_t>(min(n0 / 16 + ws64 * 4 + g, a.N / 16 - 1)) * (groups * 16) + r16 * 4;
  const uint32_t xsoff = static_cast<uint32_t>(source_row(a, min(m0 + xs64 * 64 + lane, m1 - 1)) - xrow0) *
                         static_cast<uint32_t>(a.ldxs);
  auto load_scales = [&](int q) __attribute__((always_inline)) {  // group q (at most the last)
    const int at = min(q, (nk + 3) / 4 - 1);
    const uint32_t slot = lds0 + kSAt + (q & 1) * S::kScales;
    lds_load4s(wsbase + at * 64, wsoff, slot + ws64 * 256);
    lds_load4s(xsbase + at * 4, xsoff, slot + S::BN * 4 + xs64 * 256);
  };

  f32x4 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  const char* const ldsb = reinterpret_cast<const char*>(lds);
  const uint32_t wfrag = wn * HN * 2048 + lane * 16;
  const uint32_t xfrag = kXAt + wm * HM * 2048 + (r16 >> 3) * 1024 + (r16 & 7) * 128 + 16 * (g ^ (r16 & 7));
  union Frag {
    uint4 half[2];
    i32x8 all;
  };
  Frag fa[2][HN], fb[2][TM];
  int sw[TN], sx[TM];
  // W tile i of the chunk at ring offset wo; X tile j of the chunk at xo
  auto read_a = [&](Frag (&to)[HN], int u, uint32_t wo) __attribute__((always_inline)) {
    to[u >> 1].half[u & 1] = *reinterpret_cast<const uint4*>(ldsb + (wfrag + wo) + u * 1024);
  };
  auto read_b = [&](Frag& to, int h, int j, uint32_t xo) __attribute__((always_inline)) {
    to.half[h] = *reinterpret_cast<const uint4*>(ldsb + ((xfrag ^ (64 * h)) + xo) + j * 2048);
  };
  auto read_scales = [&](int q) __attribute__((always_inline)) {
    const uint32_t slot = kSAt + (q & 1) * S::kScales;
#pragma unroll
    for (int i = 0; i < TN; ++i)
      sw[i] = *reinterpret_cast<const int*>(ldsb + slot + ((wn * TN + i) * 16 + r16) * 4);
#pragma unroll
    for (int j = 0; j < TM; ++j)
      sx[j] = *reinterpret_cast<const int*>(ldsb + slot + S::BN * 4 + ((wm * TM + j) * 16 + r16) * 4);
  };
  auto stage_at = [&](int c) __attribute__((always_inline)) { return min(c >> 1, nk - 1); };
  auto load_w = [&](int c) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < LW; ++j)
      lds_load16s(wbase + stage_at(c) * 2048, woff[c & 1][j], wdst + (c % S::WR) * S::kW + j * 1024);
  };
  auto load_x = [&](int c) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < LX; ++j)
      lds_load16s(xbase + stage_at(c) * kGroup, xoff[c & 1][j], xdst + (c % S::XR) * S::kX + j * 1024);
  };

  load_scales(0);
  load_x(0);
  load_x(1);
  load_w(0);
  load_w(1);
#pragma unroll
  for (int c = 2; c < S::D - 1; ++c) {
    load_x(c);
    load_w(c);
  }
  wait_vmcnt<S::kYoung>();
  lds_barrier();
#pragma unroll
  for (int u = 0; u < TN; ++u) read_a(fa[0], u, 0);
#pragma unroll
  for (int j = 0; j < TM; ++j)
#pragma unroll
    for (int h = 0; h < 2; ++h) read_b(fb[0][j], h, j % HM, (j / HM) * S::kX);
  read_scales(0);
  drained_barrier();
  load_x(S::D - 1);
  load_w(S::D - 1);
  wait_vmcnt<S::kYoung>();
  drained_barrier();

  // One half: P parity of the stage, H half; its W fragments are fa[H].  wo, xo:
  // ring offsets of the chunks to read; wsrc .. xd: sources and places of the
  // chunks to request.
  auto half = [&](auto par, auto hlf, uint32_t wo, uint32_t xo, const char* wsrc, uint32_t wd, const char* xsrc,
                  uint32_t xd) __attribute__((always_inline)) {
    constexpr int P = decltype(par)::value, H = decltype(hlf)::value, NM = HN * TM, ND = LW + LX, NR = TN + TM;
    // direct loads behind the odd instructions of NM, or where they are many of any
    constexpr int kSlots = 2 * ND <= NM ? NM / 2 : NM;
    static_assert(ND <= NM, "at most one direct load behind an instruction");
    [&]<int... U>(std::integer_sequence<int, U...>) __attribute__((always_inline)) {
      (([&]() __attribute__((always_inline)) {
         constexpr int i = U / TM, j = (i & 1) ? TM - 1 - U % TM : U % TM;
         constexpr int slot = kSlots == NM ? U : U / 2;
         constexpr bool takes = kSlots == NM || U % 2 == 1;
         constexpr int l = takes && first_of(slot, kSlots, ND) < first_of(slot + 1, kSlots, ND) ? first_of(slot, kSlots, ND) : ND;
         f32x4& c = acc[H * HN + i][j];
         // chunks h + D
         if constexpr (l < LX)
           mfma8_acc_load<l * 1024, false>(c, fa[H][i].all, fb[P][j].all, sw[H * HN + i], sx[j], xsrc, xoff[(H + S::D) & 1][l], xd);
         else if constexpr (l < ND)
           mfma8_acc_load<(l - LX) * 1024, NT>(c, fa[H][i].all, fb[P][j].all, sw[H * HN + i], sx[j], wsrc,
                                           woff[(H + S::D) & 1][l - LX], wd);
         else
           mfma8_acc(c, fa[H][i].all, fb[P][j].all, sw[H * HN + i], sx[j]);
#pragma unroll
         for (int u = first_of(U, NM, NR); u < first_of(U + 1, NM, NR); ++u) {
           if (u < TN)
             read_a(fa[H ^ 1], u, wo);
           else
             read_b(fb[P ^ 1][H * HM + (u - TN) / 2], (u - TN) % 2, (u - TN) / 2, xo);
         }
         __builtin_amdgcn_sched_barrier(0);
       }()),
       ...);
    }(std::make_integer_sequence<int, NM>{});
    wait_vmcnt<S::kYoung>();
  };
  // ring offsets of chunk h + 1 (W) and h + 2 (X) to read; of chunk h + D: W's slot is that of h, X's that of h + 1
  uint32_t w_read = S::kW, w_put = 0, x_read = 2 * S::kX % (S::XR * S::kX), x_put = S::kX;
  auto turn = [&]() __attribute__((always_inline)) {
    w_put = w_read;
    w_read = w_read + S::kW == S::WR * S::kW ? 0 : w_read + S::kW;
    x_put = x_read;
    x_read = x_read + S::kX == S::XR * S::kX ? 0 : x_read + S::kX;
  };
  auto stage = [&](auto par, int s) __attribute__((always_inline)) {
    if ((s & 3) == 0) load_scales((s >> 2) + 1);
    const int s0 = min(s + S::D / 2, nk - 1), s1 = min(s + (S::D + 1) / 2, nk - 1);
    half(par, std::integral_constant<int, 0>{}, w_read, x_read, wbase + s0 * 2048, wdst + w_put, xbase + s0 * kGroup,
         xdst + x_put);
    turn();
    half_barrier();
    half(par, std::integral_constant<int, 1>{}, w_read, x_read, wbase + s1 * 2048, wdst + w_put, xbase + s1 * kGroup,
         xdst + x_put);
    turn();
    if (s + 1 >= nk) {
      // a stage behind an odd last one repeats its columns with both powers
      // 2^-127, in which every product is below the least fp32 value
#pragma unroll
      for (int i = 0; i < TN; ++i) sw[i] = 0;
#pragma unroll
      for (int j = 0; j < TM; ++j) sx[j] = 0;
    } else if ((s & 3) == 3) {
      read_scales((s >> 2) + 1);
    } else {
#pragma unroll
      for (int i = 0; i < TN; ++i) sw[i] = static_cast<uint32_t>(sw[i]) >> 8;
#pragma unroll
      for (int j = 0; j < TM; ++j) sx[j] = static_cast<uint32_t>(sx[j]) >> 8;
    }
    drained_barrier();
  };
  for (int s = 0; s < nk; s += 2) {
    stage(std::integral_constant<int, 0>{}, s);
    stage(std::integral_constant<int, 1>{}, s + 1);
  }
  wait_vmcnt<0>();
  drained_barrier();

  const int mw = m0 + wm * 16 * TM, nw = n0 + wn * 16 * TN;
  if constexpr (EPI == kSlices) {
    float* const out = a.ws + static_cast<int64_t>(slice) * a.M * a.N;
#pragma unroll
    for (int j = 0; j < TM; ++j) {
      const int m = mw + 16 * j + r16;
#pragma unroll
      for (int i = 0; i < TN; ++i) {
        const int n = nw + 16 * i + 4 * g;
        if (m < m1 && n < a.N) *reinterpret_cast<f32x4*>(out + static_cast<int64_t>(m) * a.N + n) = acc[i][j];
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  } else if constexpr (EPI == kEpi8Bf16) {
    // four tiles' words are transposed over the lane groups, so that a lane has
    // the 16 columns of one tile and four lanes a whole line of a row
#pragma unroll
    for (int j = 0; j < TM; ++j) {
      const int m = mw + 16 * j + r16;
#pragma unroll
      for (int i = 0; i < TN; i += 4) {
        uint32_t lo[4], hi[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          lo[t] = pack_bf16x2(acc[i + t][j][0], acc[i + t][j][1]);
          hi[t] = pack_bf16x2(acc[i + t][j][2], acc[i + t][j][3]);
        }
        transpose4(lo);
        transpose4(hi);
        const int n = nw + 16 * (i + g);
        if (m < m1 && n < a.N) {
          uint2* o = reinterpret_cast<uint2*>(a.out16 + static_cast<int64_t>(m) * a.ldo + n);
#pragma unroll
          for (int t = 0; t < 4; ++t) o[t] = make_uint2(lo[t], hi[t]);  // (rows are 8-byte aligned)
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  } else {
    static_assert(S::BN == 256, "a workgroup has a group of 128 features");
    float* const top = reinterpret_cast<float*>(lds);  // [2][BM]
    f32x4 y[TM][HN];
    auto activate = [&](auto whole) __attribute__((always_inline)) {  // whole: all the wave's rows of W are there
#pragma unroll
      for (int j = 0; j < TM; ++j) {
        float best = 0.f;
#pragma unroll
        for (int p = 0; p < HN; ++p) {
          f32x4 gate, up;
          gate_and_up(acc[2 * p][j], acc[2 * p + 1][j], gate, up);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            y[j][p][i] = silu_f32(gate[i]) * up[i];
            if (!decltype(whole)::value) y[j][p][i] = nw + 32 * p < a.N ? y[j][p][i] : 0.f;
            best = fmaxf(best, fabsf(y[j][p][i]));
          }
        }
        best = max_xor32(max_xor16(best));
        if (g == 0) top[wn * S::BM + (wm * TM + j) * 16 + r16] = best;
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    if (nw + 16 * TN <= a.N)
      activate(std::true_type{});
    else
      activate(std::false_type{});
    __syncthreads();
    const int F = a.N / 2, f = nw / 2 + 16 * g;
#pragma unroll
    for (int j = 0; j < TM; ++j) {
      const int m = mw + 16 * j + r16, at = (wm * TM + j) * 16 + r16;
      const int ex = e8m0_of(fmaxf(top[at], top[S::BM + at]));
      const float s = e8m0_inverse(ex);
      uint32_t c[4];
#pragma unroll
      for (int p = 0; p < 4; ++p) c[p] = pack_e4m3(y[j][p][0] * s, y[j][p][1] * s, y[j][p][2] * s, y[j][p][3] * s);
      transpose4(c);
      if (m < m1) {
        if (f < (F + kGroup - 1) / kGroup * kGroup)
          *reinterpret_cast<uint4*>(a.out8 + static_cast<int64_t>(m) * a.ldo + f) = make_uint4(c[0], c[1], c[2], c[3]);
        if (wn == 0 && g == 0) a.out_scale[static_cast<int64_t>(m) * a.ldos + bn] = static_cast<uint8_t>(ex);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// 256 rows of W x 16 MT rows of X per workgroup, operands straight from global
// memory through 64-bit addresses, K whole: for rows that lie too far apart for
// the tiled kernel.  A wave has 64 rows of W; the 128 features of a workgroup's
// SwiGLU output are one group, whose maximum the four waves find through LDS.
// ---------------------------------------------------------------------------
template <int MT, int EPI>
__global__ __launch_bounds__(256) void gemm_fp8_kernel(GemmFp8Args a) {
  const int nb = (a.N + 255) / 256, bn = blockIdx.x % nb;
  int e, m0, m1;
  if (!row_block(a, blockIdx.x / nb, 16 * MT, e, m0, m1)) return;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int groups = padded_groups(a.Kp), nkb = a.Kp / kGroup;
  const uint8_t* W = a.W + static_cast<int64_t>(e) * a.N * a.Kp;
  const uint8_t* ws = a.w_scale + static_cast<int64_t>(e) * a.N * groups;
  const int n0 = bn * 256 + wave * 64;
  const uint8_t *wp[4], *wsp[4], *xp[MT], *xsp[MT];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int tn = min(n0 / 16 + i, a.N / 16 - 1);
    wp[i] = W + static_cast<int64_t>(tn) * a.Kp * 16 + lane * 16;
    wsp[i] = ws + static_cast<int64_t>(tn) * groups * 16 + r * 4;
  }
#pragma unroll
  for (int j = 0; j < MT; ++j) {
    const int64_t row = source_row(a, min(m0 + 16 * j + r, m1 - 1));
    xp[j] = a.X + row * a.ldx + 16 * g;
    xsp[j] = a.x_scale + row * a.ldxs;
  }
  f32x4 acc[4][MT];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int kb = 0; kb < nkb; ++kb) {
    uint4 x0[MT], x1[MT];
    int sx[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      x0[j] = *reinterpret_cast<const uint4*>(xp[j] + kb * kGroup);
      x1[j] = *reinterpret_cast<const uint4*>(xp[j] + kb * kGroup + 64);
      sx[j] = xsp[j][kb];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 w0 = *reinterpret_cast<const uint4*>(wp[i] + static_cast<int64_t>(kb) * 2048);
      const uint4 w1 = *reinterpret_cast<const uint4*>(wp[i] + static_cast<int64_t>(kb) * 2048 + 1024);
      const int sw = wsp[i][(kb >> 2) * 64 + (kb & 3)];
#pragma unroll
      for (int j = 0; j < MT; ++j) acc[i][j] = mfma8(w0, w1, x0[j], x1[j], acc[i][j], sw, sx[j]);
    }
  }
  if constexpr (EPI == kEpi8Bf16) {
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      const int m = m0 + 16 * j + r;
      if (m >= m1) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int n = n0 + 16 * i + 4 * g;
        if (n < a.N)
          *reinterpret_cast<uint2*>(a.out16 + static_cast<int64_t>(m) * a.ldo + n) =
              make_uint2(pack_bf16x2(acc[i][j][0], acc[i][j][1]), pack_bf16x2(acc[i][j][2], acc[i][j][3]));
      }
    }
  } else {
    __shared__ float top[4][MT][16];
    const int F = a.N / 2;
    f32x4 y[2][MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      float best = 0.f;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        f32x4 gate, up;
        gate_and_up(acc[2 * p][j], acc[2 * p + 1][j], gate, up);
        const bool in = n0 + 32 * p < a.N;  // (N % 32 == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[p][j][i] = in ? silu_f32(gate[i]) * up[i] : 0.f;
          best = fmaxf(best, fabsf(y[p][j][i]));
        }
      }
      best = max_xor32(max_xor16(best));
      if (g == 0) top[wave][j][r] = best;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      const int m = m0 + 16 * j + r;
      if (m >= m1) continue;
      const int ex = e8m0_of(fmaxf(fmaxf(top[0][j][r], top[1][j][r]), fmaxf(top[2][j][r], top[3][j][r])));
      const float s = e8m0_inverse(ex);
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int f = n0 / 2 + 16 * p + 8 * (g >> 1) + 4 * (g & 1);
        if (f < (F + kGroup - 1) / kGroup * kGroup)  // (columns that fill the last group: zero codes)
          *reinterpret_cast<uint32_t*>(a.out8 + static_cast<int64_t>(m) * a.ldo + f) =
              pack_e4m3(y[p][j][0] * s, y[p][j][1] * s, y[p][j][2] * s, y[p][j][3] * s);
      }
      if (wave == 0 && g == 0) a.out_scale[static_cast<int64_t>(m) * a.ldos + bn] = static_cast<uint8_t>(ex);
    }
  }
}

// ---------------------------------------------------------------------------
// Streaming kernel for few rows (16 MT): the weights' bytes are the cost.  A
// workgroup of NW waves owns 16 NT rows of W; the waves take the slice's groups
// of four 128-column blocks in turn, each group 8 KiB a row tile of contiguous
// loads, straight into registers and all in flight at once, and one word of
// powers for each row.  The waves' sums meet in LDS, in wave order.
// ---------------------------------------------------------------------------
template <int MT, int NT, int NW, int EPI>
__global__ __launch_bounds__(NW * 64) void gemm_fp8_stream_kernel(GemmFp8Args a, int ks) {
  static_assert(EPI == kEpi8Bf16 || EPI == kSlices, "a group of SwiGLU features spans workgroups");
  const int nb = (a.N + 16 * NT - 1) / (16 * NT);
  const int mb = total_row_blocks(a, 16 * MT);
  const int items = mb * nb * ks;
  if (static_cast<int>(blockIdx.x) >= items) return;
  const int item = xcd_run(blockIdx.x, items);
  const int slice = item / (mb * nb), bn = item % (mb * nb) / mb;
  int e, m0, m1;
  if (!row_block(a, item % mb, 16 * MT, e, m0, m1)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int r = lane & 15, g = lane >> 4;
  const int groups = padded_groups(a.Kp), n0 = bn * 16 * NT;
  const KSpan span = k_span(a.Kp / kGroup, ks, slice);
  const uint8_t *wp[NT], *wsp[NT], *xp[MT], *xsp[MT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int64_t tn = min(n0 / 16 + i, a.N / 16 - 1) + static_cast<int64_t>(e) * (a.N / 16);
    wp[i] = a.W + tn * a.Kp * 16 + static_cast<int64_t>(span.first) * 2048 + lane * 16;
    wsp[i] = a.w_scale + tn * groups * 16 + span.first * 16 + r * 4;
  }
#pragma unroll
  for (int j = 0; j < MT; ++j) {
    const int64_t row = source_row(a, min(m0 + 16 * j + r, m1 - 1));
    xp[j] = a.X + row * a.ldx + static_cast<int64_t>(span.first) * kGroup + 16 * g;
    xsp[j] = a.x_scale + row * a.ldxs + span.first;
  }
  f32x4 acc[NT][MT];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int u = wave; 4 * u < span.blocks; u += NW) {
    uint4 w[4][NT][2], x[4][MT][2];
    int sw[NT], sx[MT];
    // (blocks behind the slice's last re-read it and are not multiplied)
#pragma unroll
    for (int i = 0; i < NT; ++i) sw[i] = *reinterpret_cast<const int*>(wsp[i] + u * 64);
#pragma unroll
    for (int j = 0; j < MT; ++j) sx[j] = *reinterpret_cast<const int*>(xsp[j] + u * 4);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t kb = min(4 * u + q, span.blocks - 1);
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) w[q][i][h] = *reinterpret_cast<const uint4*>(wp[i] + kb * 2048 + h * 1024);
#pragma unroll
      for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) x[q][j][h] = *reinterpret_cast<const uint4*>(xp[j] + kb * kGroup + h * 64);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (4 * u + q >= span.blocks) break;
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j)
          acc[i][j] = mfma8(w[q][i][0], w[q][i][1], x[q][j][0], x[q][j][1], acc[i][j], sw[i] >> (8 * q), sx[j] >> (8 * q));
    }
  }
  __shared__ f32x4 red[NW][NT * MT][kWave];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) red[wave][i * MT + j][lane] = acc[i][j];
  __syncthreads();
  for (int t = wave; t < NT * MT; t += NW) {
    f32x4 sum = red[0][t][lane];
#pragma unroll
    for (int w = 1; w < NW; ++w) sum += red[w][t][lane];
    const int m = m0 + 16 * (t % MT) + r, n = n0 + 16 * (t / MT) + 4 * g;
    if (m >= m1 || n >= a.N) continue;
    if constexpr (EPI == kSlices)
      *reinterpret_cast<f32x4*>(a.ws + (static_cast<int64_t>(slice) * a.M + m) * a.N + n) = sum;
    else
      *reinterpret_cast<uint2*>(a.out16 + static_cast<int64_t>(m) * a.ldo + n) =
          make_uint2(pack_bf16x2(sum[0], sum[1]), pack_bf16x2(sum[2], sum[3]));
  }
}

// Sum of ks slices in slice order, and the epilogue: bf16 rows (a thread 4
// columns), or SwiGLU to 8-bit rows (32 lanes a group of 128 features, 4 each).
// By experts, rows that no expert has are left alone.
template <int EPI>
__global__ __launch_bounds__(256) void gemm_fp8_finish_kernel(GemmFp8Args a, int ks) {
  constexpr bool kGate = EPI == kEpi8SwiGLU;
  const int per_row = kGate ? (a.N / 2 + kGroup - 1) / kGroup * 32 : a.N / 4;
  const int64_t n = static_cast<int64_t>(a.M) * per_row, slice = static_cast<int64_t>(a.M) * a.N;
  int lo = 0, hi = a.M;
  if (a.offsets) {
    lo = a.offsets[0];
    hi = a.offsets[a.E];
  }
  for (int64_t u = blockIdx.x * 256ll + threadIdx.x; u < n; u += 256ll * gridDim.x) {
    const int m = static_cast<int>(u / per_row), c = static_cast<int>(u % per_row) * 4;
    if (m < lo || m >= hi) continue;  // (whole groups of lanes)
    auto sum = [&](int col) {
      const float* p = a.ws + static_cast<int64_t>(m) * a.N + col;
      f32x4 v = *reinterpret_cast<const f32x4*>(p);
      for (int k = 1; k < ks; ++k) v += *reinterpret_cast<const f32x4*>(p + k * slice);
      return v;
    };
    if constexpr (kGate) {
      const int col = 16 * (c / 8) + c % 8;  // gate column of feature c
      f32x4 y = {0.f, 0.f, 0.f, 0.f};
      float best = 0.f;
      if (col < a.N) {
        const f32x4 gate = sum(col), up = sum(col + 8);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[i] = silu_f32(gate[i]) * up[i];
          best = fmaxf(best, fabsf(y[i]));
        }
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) best = fmaxf(best, __shfl_xor(best, o, 32));
      const int ex = e8m0_of(best);
      const float s = e8m0_inverse(ex);
      *reinterpret_cast<uint32_t*>(a.out8 + static_cast<int64_t>(m) * a.ldo + c) =
          pack_e4m3(y[0] * s, y[1] * s, y[2] * s, y[3] * s);
      if (c % kGroup == 0) a.out_scale[static_cast<int64_t>(m) * a.ldos + c / kGroup] = static_cast<uint8_t>(ex);
    } else {
      const f32x4 v = sum(c);
      *reinterpret_cast<uint2*>(a.out16 + static_cast<int64_t>(m) * a.ldo + c) =
          make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    }
  }
}

// Row blocks of BM rows that M rows can make: by experts, each may leave one
// partly filled.
int row_blocks(const GemmFp8Args& a, int BM) {
  if (!a.offsets) return (a.M + BM - 1) / BM;
  return static_cast<int>(std::min<int64_t>(a.M, (a.M + static_cast<int64_t>(a.E) * (BM - 1)) / BM));
}

// go with the smallest number of LO, LO + STEP .. HI that is at least v (HI if none)
template <int LO, int STEP, int HI, class Go>
void one_of(int v, Go&& go) {
  if constexpr (LO < HI) {
    if (v > LO) return one_of<LO + STEP, STEP, HI>(v, go);
  }
  go(std::integral_constant<int, LO>{});
}

// Row blocks to expect of M rows; by experts, half a partly filled one each on
// top, and at least one for each expert.
double expected_blocks(const GemmFp8Args& a, int BM) {
  if (!a.offsets) return (a.M + BM - 1) / BM;
  const int live = std::min(a.E, a.M);
  return std::max<double>(live, static_cast<double>(a.M) / BM + 0.5 * live);
}

// us that a plan is expected to take: the launch, the rounds of workgroups and the
// stream of the weights (which overlap, not freely), and what k slices cost
// behind them.
double expected_us(const GemmFp8Args& a, int epilogue, const GemmFp8Plan& p) {
  constexpr double kLaunch = 3.0;
  constexpr int kCus = 256;
  const bool tiled = p.kind == GemmFp8Kind::kTiled;
  const int ks = std::max(p.ks, 1), stages = (a.Kp / kGroup + ks - 1) / ks;
  const int live = a.offsets ? std::min(a.E, a.M) : 1;  // matrices that have rows
  const double finish = p.ks ? 3.9 + 8e-6 * ks * a.M * a.N / 6.8 : 0.0;
  const int bm = 16 * p.mt * (tiled ? 2 : 1), bn = 16 * p.nt * (tiled ? 2 : 1);
  const double row_blocks = expected_blocks(a, bm), blocks = row_blocks * ((a.N + bn - 1) / bn) * ks;
  // MB; further row blocks of the same weights find most of them in the caches
  const double weights = 1e-6 * a.N * a.Kp * (live + 0.11 * (row_blocks - live));
  if (!tiled) return kLaunch + weights / std::min(p.mt == 1 ? 5.3 : 3.0, 0.027 * blocks) + finish;
  double rounds = std::ceil(blocks / kCus);
  if (a.offsets) {  // the number of blocks is a guess: a round begun counts by how sure it is
    const double some = blocks / kCus + 0.07, whole = std::floor(some);
    rounds = std::max(1.0, whole + std::min(1.0, 3.5 * (some - whole)));
  }
  const double gate = epilogue == kEpi8SwiGLU && !p.ks ? 0.64 * p.mt : 0.0;
  const double c = rounds * (stages * (0.25 + 0.011 * p.nt * p.mt) + gate), h = weights / std::min(6.2, 0.042 * blocks);
  return kLaunch + std::sqrt(std::sqrt(c * c * c * c + h * h * h * h)) + finish;
}

// Whether W should pass the caches by.  It gains where W streams from HBM and few
// row blocks read each matrix, more so by experts, whose row blocks of one
// matrix are neighbours in time (W kept / passed, us): 8B gate/up at 128 / 301 /
// 1001 rows 33.0 / 29.9, 45.0 / 43.3, 106.7 / 104.1, at 4096 377 / 388; 70B down at 128
// rows 55.2 / 54.0, at 301 (two row blocks) 87.0 / 90.5; a product of 4096 x 4096 at
// 301 rows, kept between calls, 14.3 / 17.8; eight experts' gate/up of 50 rows 168.9 /
// 156.5, of 2000 362 / 355, their down of 50 80.5 / 70.6, of 8192 448 / 426.
bool passes_caches(const GemmFp8Args& a, const GemmFp8Plan& p) {
  const int live = a.offsets ? std::min(a.E, a.M) : 1;
  const double per = expected_blocks(a, 32 * p.mt) / live;
  return 1e-6 * a.N * a.Kp * live >= 96 && per <= (a.offsets ? 5.6 : a.N >= 16384 ? 8 : 1);
}

}  // namespace

// Kernel and k slices: of the plans that the shape and the workspace allow, the
// one with the least expected time.  The expectation's constants are fitted to
// the times of all plans of 175 products of 1 to 10000 rows (the 8B, 70B and tiny
// widths, 4 to 32 experts, weights out of the caches); over those the chosen plan
// is 2% slower than the best one in the mean, 19% at most.  What they say, us:
//  - a tiled stage (128 columns) costs 0.25 + 0.011 TN TM of a CU: LDS first (128 x 64
//    blocks move 72 KiB a stage, 595 clocks; two parts of k in one workgroup or one
//    barrier a stage change little), the matrix cores from TN TM = 48 on, so rows are not rounded up to
//    large tiles (8B gate/up at 301 rows as 256 x 256 / 256 x 192 / 256 x 128 tiles
//    53.6 / 43.2 / 59.6, at 200 rows 48.5 / 43.8 / 37.4), and rounds of 256 workgroups
//    count whole (8192 rows of 8 experts' down as 256 x 256 / 256 x 192 477 / 438).
//  - weights stream at 6.2 TB/s where enough workgroups ask: 8B gate/up at 25 rows as
//    112 workgroups of 256 W rows with SwiGLU in place 27.8, as 224 of 128 with the
//    finishing launch 24.2.
//  - k slices fill the CUs of narrow products and cost a launch and their sums'
//    traffic: 70B down at 128 rows in 1 / 2 / 4 / 8 slices of 128 x 128 tiles 113 / 86 /
//    57 / 64, QKV at 301 rows in 1 / 2 14.9 / 21.0.
//  - up to 32 rows (of each expert) the streaming kernel keeps a narrow product of
//    few bytes in flight at once: QKV at 25 rows 8.4 against 10.9 of 4 tiled slices,
//    8B down at 16 rows 15.8 / 17.5, but 70B QKV at 32 rows 26.9 / 23.6.
GemmFp8Plan plan_gemm_fp8(const GemmFp8Args& a, int epilogue) {
  // The tiled kernel reaches rows and their powers by 32-bit byte offsets from its
  // block's first row, or from the first row of X where rows are gathered.
  constexpr int64_t kMax = int64_t{1} << 32;
  const bool fits = static_cast<int64_t>(a.src ? a.x_rows : 256) * std::max(a.ldx, a.ldxs) <= kMax && 256ll * a.Kp <= kMax &&
                    static_cast<int64_t>(a.N) * (a.Kp / kGroup + 3) <= kMax;
  if (!fits) return {GemmFp8Kind::kDirect, 16, 4, 0, false};
  const bool swiglu = epilogue == kEpi8SwiGLU;
  const int units = (a.Kp / kGroup + 3) / 4;
  GemmFp8Plan best{GemmFp8Kind::kTiled, 8, 2, 0, false};
  double least = expected_us(a, epilogue, best);
  auto offer = [&](GemmFp8Plan p) {
    if (p.ks > units || static_cast<int64_t>(p.ks) * a.M * a.N > a.ws_floats) return;
    const int bm = 16 * p.mt * (p.kind == GemmFp8Kind::kTiled ? 2 : 1), bn = 16 * p.nt * (p.kind == GemmFp8Kind::kTiled ? 2 : 1);
    if (static_cast<int64_t>(row_blocks(a, bm)) * ((a.N + bn - 1) / bn) * std::max(p.ks, 1) >= (1 << 23)) return;  // (2^32 threads)
    const double t = expected_us(a, epilogue, p);
    if (t < least) {
      least = t;
      best = p;
    }
  };
  for (int ks = 0; ks <= 8; ks = ks ? 2 * ks : 1) {
    if (ks == 1 && !swiglu) continue;  // (a product in one slice needs no finishing launch)
    for (int mt = 2; mt <= 8; mt += 2) {
      if (ks || !swiglu) offer({GemmFp8Kind::kTiled, 4, mt, ks, false});
      if (ks != 1) offer({GemmFp8Kind::kTiled, 8, mt, ks, false});
    }
    if (a.M <= 32 * a.E && (ks || !swiglu)) offer({GemmFp8Kind::kStream, 2, a.M <= 16 * a.E ? 1 : 2, ks, false});
  }
  best.nt_hint = best.kind == GemmFp8Kind::kTiled && passes_caches(a, best);
  return best;
}

static hipError_t run_plan(const GemmFp8Plan& p, const GemmFp8Args& a, int epilogue, hipStream_t s) {
  const int ks = std::max(p.ks, 1);
  auto grid = [&](int bm, int bn) {
    return dim3(static_cast<uint32_t>(static_cast<int64_t>(row_blocks(a, bm)) * ((a.N + bn - 1) / bn) * ks));
  };
  if (p.kind == GemmFp8Kind::kDirect) {
    if (epilogue == kEpi8SwiGLU)
      gemm_fp8_kernel<4, kEpi8SwiGLU><<<grid(64, 256), dim3(256), 0, s>>>(a);
    else
      gemm_fp8_kernel<4, kEpi8Bf16><<<grid(64, 256), dim3(256), 0, s>>>(a);
  } else if (p.kind == GemmFp8Kind::kStream) {
    one_of<1, 1, 2>(p.mt, [&](auto mt) {
      if (p.ks)
        gemm_fp8_stream_kernel<mt, 2, 8, kSlices><<<grid(16 * mt, 32), dim3(512), 0, s>>>(a, ks);
      else
        gemm_fp8_stream_kernel<mt, 2, 8, kEpi8Bf16><<<grid(16 * mt, 32), dim3(512), 0, s>>>(a, ks);
    });
  } else {
    one_of<4, 4, 8>(p.nt, [&](auto tn) {
      one_of<2, 2, 8>(p.mt, [&](auto tm) {
        using S = TileShape8<tn, tm>;
        auto go = [&](auto epi, auto nt) {
          gemm_fp8_tiled_kernel<S, epi, nt><<<grid(S::BM, S::BN), dim3(256), 0, s>>>(a, ks);
        };
        auto hinted = [&](auto epi) {
          if (p.nt_hint)
            go(epi, std::true_type{});
          else
            go(epi, std::false_type{});
        };
        if (p.ks) return hinted(std::integral_constant<int, kSlices>{});
        if constexpr (S::BN == 256) {
          if (epilogue == kEpi8SwiGLU) return hinted(std::integral_constant<int, kEpi8SwiGLU>{});
        }
        hinted(std::integral_constant<int, kEpi8Bf16>{});
      });
    });
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.ks) return e;
  const int64_t items = static_cast<int64_t>(a.M) * (epilogue == kEpi8SwiGLU ? (a.N / 2 + kGroup - 1) / kGroup * 32 : a.N / 4);
  const dim3 g(static_cast<uint32_t>(std::min<int64_t>((items + 255) / 256, 65536)));
  if (epilogue == kEpi8SwiGLU)
    gemm_fp8_finish_kernel<kEpi8SwiGLU><<<g, dim3(256), 0, s>>>(a, ks);
  else
    gemm_fp8_finish_kernel<kEpi8Bf16><<<g, dim3(256), 0, s>>>(a, ks);
  return hipGetLastError();
}

hipError_t launch_gemm_fp8(const GemmFp8Args& a, int epilogue, hipStream_t s) {
  if (a.M <= 0) return hipSuccess;
  return run_plan(plan_gemm_fp8(a, epilogue), a, epilogue, s);
}

}  // namespace metro
