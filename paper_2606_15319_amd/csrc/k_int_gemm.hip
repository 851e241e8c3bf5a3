// Linear layers over 8-bit integer codes: y = epilogue(sx_i sw_j sum_k X_ik W_jk).
//
// X [M][K] and W [N][K] are both K-contiguous.  v_mfma_i32_16x16x64_i8 sums exactly in 32 bits
// (|sum| <= 2^30 at K = 65536), at twice the bf16 rate per operand byte.  The MFMA computes
// C^T = W X^T: W rows feed the A operand and X rows the B operand, so a lane ends with one row i
// and four consecutive columns j of every 16 x 16 block.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "launch.h"

namespace ardit {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// A scale as mantissa in [0.5, 1) and exponent: sum * mx * mw stays a normal number whatever the
// scales are, and one ldexp puts the exponents back (their plain product may leave fp32's range
// where the result does not).
struct Scale {
  float m;
  int e;
};
__device__ __forceinline__ Scale split_scale(float s) {
  return Scale{__builtin_amdgcn_frexp_mantf(s), __builtin_amdgcn_frexp_expf(s)};
}

// One element after the product.  Every kernel below ends in this, so a row has the same bits
// whichever of them computes it.
template <int EPI>
__device__ __forceinline__ float finish(int sum, Scale sx, Scale sw, float bias, float res, float gate) {
  float z = __builtin_amdgcn_ldexpf(static_cast<float>(sum) * sx.m * sw.m, sx.e + sw.e) + bias;
  if (EPI == kEpiBiasGelu) z = gelu_tanh(z);
  if (EPI == kEpiBiasRes) z = res + z;
  if (EPI == kEpiBiasGateRes) z = fmaf(gate, z, res);
  return z;
}

template <typename T>
__device__ __forceinline__ float as_float(T v) {
  if constexpr (sizeof(T) == 4) return v;
  else return bf2f(v);
}

// Four consecutive elements, the first `left` of them: all at once, in pairs or one by one (width 4,
// 2, 1: what the tensor's base and stride allow).
template <typename T>
__device__ __forceinline__ void load4(const T* p, int left, int width, float* f) {
  if (width == 4 && left >= 4) {
    if constexpr (sizeof(T) == 4) {
      const float4 r = *reinterpret_cast<const float4*>(p);
      f[0] = r.x; f[1] = r.y; f[2] = r.z; f[3] = r.w;
    } else {
      const uint2 r = *reinterpret_cast<const uint2*>(p);
      f[0] = __uint_as_float(r.x << 16); f[1] = __uint_as_float(r.x & 0xffff0000u);
      f[2] = __uint_as_float(r.y << 16); f[3] = __uint_as_float(r.y & 0xffff0000u);
    }
  } else if (width >= 2 && left >= 4) {
#pragma unroll
    for (int h = 0; h < 4; h += 2) {
      if constexpr (sizeof(T) == 4) {
        const float2 r = *reinterpret_cast<const float2*>(p + h);
        f[h] = r.x; f[h + 1] = r.y;
      } else {
        const uint32_t r = *reinterpret_cast<const uint32_t*>(p + h);
        f[h] = __uint_as_float(r << 16); f[h + 1] = __uint_as_float(r & 0xffff0000u);
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = e < left ? as_float(p[e]) : 0.f;
  }
}
// (fp32 results go past the L2: 4680 x 5120 of them 147 us for 161 with the residual's read, 4680 x
// 1536 26 for 33; bf16 ones, whose lines fill in pieces of 32 bytes, take longer that way, 117 for 101.)
template <typename T>
__device__ __forceinline__ void store4(T* p, int left, int width, const float* y) {
  if (width == 4 && left >= 4) {
    if constexpr (sizeof(T) == 4) __builtin_nontemporal_store(f32x4{y[0], y[1], y[2], y[3]}, reinterpret_cast<f32x4*>(p));
    else *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
  } else if (width >= 2 && left >= 4) {
#pragma unroll
    for (int h = 0; h < 4; h += 2) {
      if constexpr (sizeof(T) == 4) *reinterpret_cast<float2*>(p + h) = make_float2(y[h], y[h + 1]);
      else *reinterpret_cast<uint32_t*>(p + h) = pack_bf16x2(y[h], y[h + 1]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) {
        if constexpr (sizeof(T) == 4) p[e] = y[e];
        else p[e] = f2bf(y[e]);
      }
  }
}

// What a lane needs of its columns after the product: NB_ times four, 16 apart.
template <int NB_>
struct Columns {
  float s[NB_][4], bias[NB_][4];   // (scales are split where they are used: half the registers)
};
template <int NB_>
__device__ __forceinline__ void load_columns(const IntGemmArgs& p, int n0, Columns<NB_>& c) {
#pragma unroll
  for (int b = 0; b < NB_; ++b) {
    const int n = n0 + 16 * b, left = p.N - n;
    load4(p.sw + n, left, p.width_cols, c.s[b]);
#pragma unroll
    for (int e = 0; e < 4; ++e) c.bias[b][e] = 0.f;
    if (p.bias) load4(p.bias + n, left, p.width_cols, c.bias[b]);
  }
}

// What the result takes of row m besides the product.
template <int EPI, typename ResT, int NB_>
struct RowIn {
  float sx, res[NB_][4];
};
template <int EPI, typename ResT, int NB_>
__device__ __forceinline__ void load_row(const IntGemmArgs& p, int m, int n0, RowIn<EPI, ResT, NB_>& r) {
  m = min(m, p.M - 1);
  r.sx = p.sx[m];
  if (EPI == kEpiBiasRes || EPI == kEpiBiasGateRes)
#pragma unroll
    for (int b = 0; b < NB_; ++b)
      load4(static_cast<const ResT*>(p.res) + m * p.ldr + n0 + 16 * b, p.N - n0 - 16 * b, p.width_res, r.res[b]);
}
template <int NB_>
__device__ __forceinline__ void load_gate(const IntGemmArgs& p, int stream, int n0, float (&gate)[NB_][4]) {
  const float* mod = p.mod + (static_cast<size_t>(stream) * 6 + p.gate_row) * p.N;
#pragma unroll
  for (int b = 0; b < NB_; ++b) {
    const int n = n0 + 16 * b, left = p.N - n;
    load4(mod + n, left, p.width_cols, gate[b]);
    if (p.table) {
      float t[4];
      load4(p.table + static_cast<size_t>(p.gate_row) * p.N + n, left, p.width_cols, t);
#pragma unroll
      for (int e = 0; e < 4; ++e) gate[b][e] += t[e];
    }
  }
}

// The rows m0, m0 + 16, ... of a lane's columns: epilogue and store.  A row's residual is requested
// AHEAD rows before it is used (the residual may be y: a row is read before it is written), the
// gate once where all rows of the wave are one stream's.
template <int EPI, typename ResT, typename OutT, int MB, int NB_>
__device__ __forceinline__ void finish_rows(const IntGemmArgs& p, int m0, int n0, const i32x4 (&acc)[MB][NB_]) {
  // (by registers: of all, only gated fp32 results of 256 rows spill, four registers)
  constexpr int AHEAD = MB >= 8 ? (EPI == kEpiBiasGateRes ? 1 : 2) : MB < 3 ? MB : 3;
  RowIn<EPI, ResT, NB_> in[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) load_row<EPI, ResT, NB_>(p, m0 + 16 * i, n0, in[i]);
  Columns<NB_> c;
  load_columns<NB_>(p, n0, c);
  float gate[NB_][4];
  int stream = -1;
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) {
    const int m = m0 + 16 * mb;
    RowIn<EPI, ResT, NB_>& r = in[mb % AHEAD];
    if (EPI == kEpiBiasGateRes) {
      const int s = static_cast<int>(fdiv(min(m, p.M - 1), p.rows_per_stream));
      if (s != stream) load_gate<NB_>(p, s, n0, gate);
      stream = s;
    }
    const Scale sx = split_scale(r.sx);
    float y[NB_][4];
#pragma unroll
    for (int b = 0; b < NB_; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        y[b][e] = finish<EPI>(acc[mb][b][e], sx, split_scale(c.s[b][e]), c.bias[b][e], EPI >= kEpiBiasGateRes ? r.res[b][e] : 0.f,
                              EPI == kEpiBiasGateRes ? gate[b][e] : 0.f);
    if (mb + AHEAD < MB) load_row<EPI, ResT, NB_>(p, m + 16 * AHEAD, n0, r);
    if (m < p.M) {
      OutT* o = static_cast<OutT*>(p.y) + m * p.ldy + n0;
#pragma unroll
      for (int b = 0; b < NB_; ++b) store4(o + 16 * b, p.N - n0 - 16 * b, p.width_y, y[b]);
    }
  }
}

// The same with the result's kind known at run time (small products, whose code is not worth a
// kernel for each).
template <int MB, int NB_>
__device__ __forceinline__ void finish_rows_any(const IntGemmArgs& p, int epi, int m0, int n0, const i32x4 (&acc)[MB][NB_]) {
  const bool rf = p.res_f32, of = p.y_f32;
  if (epi == kEpiBias) {
    if (of) finish_rows<kEpiBias, bf16_t, float, MB, NB_>(p, m0, n0, acc);
    else finish_rows<kEpiBias, bf16_t, bf16_t, MB, NB_>(p, m0, n0, acc);
  } else if (epi == kEpiBiasGelu) {
    finish_rows<kEpiBiasGelu, bf16_t, bf16_t, MB, NB_>(p, m0, n0, acc);
  } else if (epi == kEpiBiasRes) {
    if (rf && of) finish_rows<kEpiBiasRes, float, float, MB, NB_>(p, m0, n0, acc);
    else if (rf) finish_rows<kEpiBiasRes, float, bf16_t, MB, NB_>(p, m0, n0, acc);
    else if (of) finish_rows<kEpiBiasRes, bf16_t, float, MB, NB_>(p, m0, n0, acc);
    else finish_rows<kEpiBiasRes, bf16_t, bf16_t, MB, NB_>(p, m0, n0, acc);
  } else {
    if (rf && of) finish_rows<kEpiBiasGateRes, float, float, MB, NB_>(p, m0, n0, acc);
    else if (rf) finish_rows<kEpiBiasGateRes, float, bf16_t, MB, NB_>(p, m0, n0, acc);
    else if (of) finish_rows<kEpiBiasGateRes, bf16_t, float, MB, NB_>(p, m0, n0, acc);
    else finish_rows<kEpiBiasGateRes, bf16_t, bf16_t, MB, NB_>(p, m0, n0, acc);
  }
}

// ------------------------------------------------------------------ large tiles
constexpr int BN = 256, BK = 128, NT = 512, NWAVES = 8;   // (a K step is 128 bytes of every row)
constexpr int WN = 64, NB = WN / 16, NWN = BN / WN;
constexpr int W_INS = BN * BK / 1024 / NWAVES;
constexpr int GROUP_M = 8;   // m-tiles per raster group (L2 reuse of W columns)
// LDS: a ring of five places of one operand and step each (X0 W0 X1 W1 X2 ...)
constexpr int SLOT = 32 * 1024, SLOTS = 5, RING = SLOT * SLOTS;

template <int BM_>
struct Cfg {
  static constexpr int WM = BM_ / 2, MB = WM / 16;
  static constexpr int A_INS = BM_ * BK / 1024 / NWAVES;
  static_assert(A_INS * NWAVES * 1024 == BM_ * BK && BM_ * BK <= SLOT, "");
};

__device__ __forceinline__ int swz(int r) { return (r >> 1) & 7; }

template <int BM, int EPI, typename ResT, typename OutT>
__global__ __launch_bounds__(NT, 1) void int_gemm_kernel(const IntGemmArgs p, int tiles_m, int tiles_n, int per_xcd) {
  using G = Cfg<BM>;
  constexpr int WM = G::WM, MB = G::MB, A_INS = G::A_INS;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[RING];

  // XCD-aware tile order: consecutive logical tiles land on one XCD (shared L2)
  const int L = (blockIdx.x % kNumXcd) * per_xcd + blockIdx.x / kNumXcd;
  if (L >= tiles_m * tiles_n) return;
  const int group = GROUP_M * tiles_n;
  const int g0 = (L / group) * GROUP_M;
  const int gm = min(tiles_m - g0, GROUP_M);
  const int tm = g0 + (L % group) % gm, tn = (L % group) / gm;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int wm = wave / NWN, wn = wave % NWN;

  // Load j of this wave fills the 8 LDS rows 8 (wave * INS + j) .. + 7: lane i writes place i % 8
  // of row 8 (...) + i / 8, which holds chunk (i % 8) ^ swz(row).
  const char* a_base = uniform_ptr(p.x + static_cast<int64_t>(tm) * BM * p.ldx);
  const char* w_base = uniform_ptr(p.w + static_cast<int64_t>(tn) * BN * p.ldw);
  const int ldx = static_cast<int>(p.ldx), ldw = static_cast<int>(p.ldw);
  uint32_t a_off[A_INS], w_off[W_INS];
#pragma unroll
  for (int j = 0; j < A_INS; ++j) {
    const int r = 8 * (wave * A_INS + j) + (lane >> 3);
    a_off[j] = static_cast<uint32_t>(min(r, p.M - 1 - tm * BM) * ldx + ((lane & 7) ^ swz(r)) * 16);
  }
#pragma unroll
  for (int j = 0; j < W_INS; ++j) {
    const int r = 8 * (wave * W_INS + j) + (lane >> 3);
    w_off[j] = static_cast<uint32_t>(min(r, p.N - 1 - tn * BN) * ldw + ((lane & 7) ^ swz(r)) * 16);
  }
  const uint32_t smem_s = lds_address(smem);
  // the last K step may hold fewer chunks of 16 bytes: the others load the row's last chunk, and
  // are zeroed as fragments of W
  const int chunks = (p.K + 15) / 16, nk = (chunks + 7) / 8, last = chunks - 8 * (nk - 1);
  auto back = [&](int r) __attribute__((always_inline)) {
    const int c = (lane & 7) ^ swz(r);
    return 16u * (c - min(c, last - 1));
  };
  // one load of step kt's X or W into the ring at byte `at` (end: it is the last step)
  auto load_a = [&](int kt, uint32_t at, int j, bool end) __attribute__((always_inline)) {
    lds_dma16(a_base + kt * BK, end ? a_off[j] - back(8 * (wave * A_INS + j) + (lane >> 3)) : a_off[j],
              smem_s + at + 1024u * (wave * A_INS + j));
  };
  auto load_w = [&](int kt, uint32_t at, int j, bool end) __attribute__((always_inline)) {
    lds_dma16(w_base + kt * BK, end ? w_off[j] - back(8 * (wave * W_INS + j) + (lane >> 3)) : w_off[j],
              smem_s + at + 1024u * (wave * W_INS + j));
  };

  i32x4 acc[MB][NB];
#pragma unroll
  for (int a = 0; a < MB; ++a)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[a][b] = i32x4{0, 0, 0, 0};

  // fragments of 64-byte half kk: rows 16 b + l16 of the wave's piece of W, of X
  const int half[2] = {16 * (g ^ swz(l16)), 16 * ((4 + g) ^ swz(l16))};
  const unsigned char* fr_w = smem + (WN * wn + l16) * BK;
  const unsigned char* fr_a = smem + (WM * wm + l16) * BK;
  auto read = [&](const unsigned char* f, uint32_t at, int kk, int b) __attribute__((always_inline)) {
    return *reinterpret_cast<const i32x4*>(f + at + half[kk] + 16 * BK * b);
  };
  i32x4 fa[MB], fw[2][NB];

#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (i < nk) {
#pragma unroll
      for (int j = 0; j < A_INS; ++j) load_a(i, 2 * i * SLOT, j, i == nk - 1);
#pragma unroll
      for (int j = 0; j < W_INS; ++j) load_w(i, (2 * i + 1) * SLOT, j, i == nk - 1);
    }
  if (nk > 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(A_INS + W_INS));
  else asm volatile("s_waitcnt vmcnt(0)");
  __syncthreads();
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) fw[0][nb] = read(fr_w, SLOT, 0, nb);
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) fa[mb] = read(fr_a, 0, 0, mb);
  // Step kt in two halves of 64 bytes of K.  Each half multiplies the fragments in registers and
  // reads those of the next: a fragment of X as soon as the products that use its register are
  // issued, so that it has the products of the other row blocks to arrive.  The barrier, after
  // AT + 1 row blocks of the second half, publishes step kt + 1 and closes the reads of step kt.
  // X of step kt + 2 is requested in the first half (into the place of W of step kt - 1), W behind
  // the barrier (into the place of X of step kt), one load behind each row block: requested
  // together they hold up the products.
  constexpr int AT = 1;
  uint32_t at_a = 0;                        // place of step kt's X, W behind it
  auto around = [](uint32_t at) { return at >= RING ? at - RING : at; };
  auto products = [&](int mb, int kk) __attribute__((always_inline)) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
      acc[mb][nb] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[kk][nb], fa[mb], acc[mb][nb], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  auto cut = [&](int kk) __attribute__((always_inline)) {   // W past the row's end
    if (4 * kk + g >= last)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) fw[kk][nb] = i32x4{0, 0, 0, 0};
  };
  // LEFT: steps behind this one, 3 for three or more
  auto step = [&](int kt, auto left_c) __attribute__((always_inline)) {
    constexpr int LEFT = decltype(left_c)::value;
    const uint32_t at_w = around(at_a + SLOT), next_a = around(at_a + 2 * SLOT), next_w = around(at_a + 3 * SLOT);
    const uint32_t old_w = around(at_a + 4 * SLOT);
    if (LEFT == 0) cut(0);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      products(mb, 0);
      if (mb < NB) fw[1][mb] = read(fr_w, at_w, 1, mb);
      fa[mb] = read(fr_a, at_a, 1, mb);
      if (LEFT >= 2 && mb < A_INS) load_a(kt + 2, old_w, mb, LEFT == 2);
    }
    if (LEFT == 0) cut(1);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      products(mb, 1);
      if (LEFT >= 1) {
        if (mb == AT) {
          asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT >= 2 ? A_INS : 0));
          __syncthreads();
          fw[0][0] = read(fr_w, next_w, 0, 0);
          fw[0][1] = read(fr_w, next_w, 0, 1);
#pragma unroll
          for (int i = 0; i < AT; ++i) fa[i] = read(fr_a, next_a, 0, i);
        }
        if (mb >= AT) fa[mb] = read(fr_a, next_a, 0, mb);
        if (mb == AT + 1) {
          fw[0][2] = read(fr_w, next_w, 0, 2);
          fw[0][3] = read(fr_w, next_w, 0, 3);
        }
        if (LEFT >= 2 && mb >= AT)
#pragma unroll
          for (int j = 0; j < W_INS; ++j)
            if (min(j, MB - 1 - AT) == mb - AT) load_w(kt + 2, at_a, j, LEFT == 2);
      }
    }
    at_a = next_a;
  };
  int kt = 0;
  for (; kt + 3 < nk; ++kt) step(kt, std::integral_constant<int, 3>{});
  if (kt + 2 < nk) step(kt++, std::integral_constant<int, 2>{});
  if (kt + 1 < nk) step(kt++, std::integral_constant<int, 1>{});
  step(kt, std::integral_constant<int, 0>{});

  finish_rows<EPI, ResT, OutT, MB, NB>(p, tm * BM + WM * wm + l16, tn * BN + WN * wn + 4 * g, acc);
}

// ------------------------------------------------------------------ small tiles
// Tiles of 16 MB WM_ x 16 NB WN_ on KS groups of WM_ x WN_ waves, for products too small to give
// every CU a large tile.  A group takes every KS-th K step, S - 1 of them under way through its
// ring of S stages in LDS; one barrier an iteration publishes the stages of step kt and closes the
// reads of the one before, into which a later step is requested.  Groups are joined in LDS (whole
// sums: in any order the same bits).
template <int WM_, int WN_, int MB, int NB_, int S, int KS>
__global__ __launch_bounds__(64 * WM_ * WN_ * KS, 1) void int_gemm_small(const IntGemmArgs p, int epi, int tiles_m,
                                                                         int tiles_n) {
  constexpr int NW = WM_ * WN_, BM = 16 * MB * WM_, BNS = 16 * NB_ * WN_;
  constexpr int AB = BM * BK, WB = BNS * BK, STAGE = AB + WB;
  constexpr int A_INS = AB / 1024 / NW, WI = WB / 1024 / NW, INS = A_INS + WI;
  static_assert(A_INS * NW * 1024 == AB && WI * NW * 1024 == WB, "whole loads per wave");
  static_assert(KS * S * STAGE <= 160 * 1024 && S >= 3 && (S - 2) * INS < 64, "LDS, counter");
  static_assert((KS - 1) * NW * MB * NB_ * 1024 <= KS * S * STAGE, "join");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[KS * S * STAGE];
  // XCD-aware order: each XCD takes a run of column tiles with all their row tiles
  const int total = tiles_m * tiles_n, per_xcd = (total + kNumXcd - 1) / kNumXcd;
  const int L = static_cast<int>(blockIdx.x % kNumXcd) * per_xcd + static_cast<int>(blockIdx.x / kNumXcd);
  if (L >= total) return;
  const int tm = L % tiles_m, tn = L / tiles_m;

  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int grp = wid / NW, wave = wid % NW;
  const int l16 = lane & 15, g = lane >> 4;
  const int wm = wave / WN_, wn = wave % WN_;
  const char* a_base = uniform_ptr(p.x + static_cast<int64_t>(tm) * BM * p.ldx);
  const char* w_base = uniform_ptr(p.w + static_cast<int64_t>(tn) * BNS * p.ldw);
  const int ldx = static_cast<int>(p.ldx), ldw = static_cast<int>(p.ldw);
  uint32_t off[INS];
#pragma unroll
  for (int j = 0; j < INS; ++j) {
    const int r = 8 * (j < A_INS ? wave * A_INS + j : wave * WI + j - A_INS) + (lane >> 3);
    const int row = j < A_INS ? min(r, p.M - 1 - tm * BM) * ldx : min(r, p.N - 1 - tn * BNS) * ldw;
    off[j] = static_cast<uint32_t>(row + ((lane & 7) ^ swz(r)) * 16);
  }
  const uint32_t lds_g = lds_address(smem) + grp * (S * STAGE);
  const uint32_t lds_a = lds_g + 1024u * (wave * A_INS), lds_w = lds_g + AB + 1024u * (wave * WI);
  const int chunks = (p.K + 15) / 16, nk = (chunks + 7) / 8, last = chunks - 8 * (nk - 1);
  const int iters = (nk + KS - 1) / KS;
  // iteration it is this group's K step it * KS + grp, where there is one
  auto issue = [&](int it, int slot) __attribute__((always_inline)) {
    const int kt = it * KS + grp;
    if (KS > 1 && kt >= nk) return;
    const uint32_t so = static_cast<uint32_t>(slot * STAGE);
    const bool end = kt == nk - 1 && last < 8;   // (the row's last chunk in the place of missing ones)
#pragma unroll
    for (int j = 0; j < INS; ++j) {
      uint32_t o = off[j];
      if (end) {
        const int c = (lane & 7) ^ swz(8 * (j < A_INS ? wave * A_INS + j : wave * WI + j - A_INS) + (lane >> 3));
        o -= 16u * (c - min(c, last - 1));
      }
      if (j < A_INS) lds_dma16(a_base + kt * BK, o, lds_a + so + 1024u * j);
      else lds_dma16(w_base + kt * BK, o, lds_w + so + 1024u * (j - A_INS));
    }
  };

  i32x4 acc[MB][NB_];
#pragma unroll
  for (int a = 0; a < MB; ++a)
#pragma unroll
    for (int b = 0; b < NB_; ++b) acc[a][b] = i32x4{0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < S - 1; ++i)
    if (i < iters) issue(i, i);
  int slot = 0;
  for (int it = 0; it < iters; ++it) {
    const int kt = it * KS + grp;
    // (the last step requested by then is (it + S - 2) KS + grp)
    if (kt + (S - 2) * KS < nk) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 2) * INS));
    else asm volatile("s_waitcnt vmcnt(0)");
    __syncthreads();
    if (it + S - 1 < iters) issue(it + S - 1, slot == 0 ? S - 1 : slot - 1);
    if (KS == 1 || kt < nk) {
      const unsigned char* sa = smem + grp * (S * STAGE) + slot * STAGE + (16 * MB * wm + l16) * BK;
      const unsigned char* sw = smem + grp * (S * STAGE) + slot * STAGE + AB + (16 * NB_ * wn + l16) * BK;
      i32x4 fa[2][MB], fw[2][NB_];
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        const int c = 16 * ((4 * kk + g) ^ swz(l16));
#pragma unroll
        for (int nb = 0; nb < NB_; ++nb) fw[kk][nb] = *reinterpret_cast<const i32x4*>(sw + 16 * BK * nb + c);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) fa[kk][mb] = *reinterpret_cast<const i32x4*>(sa + 16 * BK * mb + c);
        if (kt == nk - 1 && 4 * kk + g >= last)
#pragma unroll
          for (int nb = 0; nb < NB_; ++nb) fw[kk][nb] = i32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int nb = 0; nb < NB_; ++nb)
            acc[mb][nb] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[kk][nb], fa[kk][mb], acc[mb][nb], 0, 0, 0);
    }
    slot = slot == S - 1 ? 0 : slot + 1;
  }
  if constexpr (KS > 1) {
    i32x4* part = reinterpret_cast<i32x4*>(smem);
    __syncthreads();
    if (grp > 0)
#pragma unroll
      for (int a = 0; a < MB; ++a)
#pragma unroll
        for (int b = 0; b < NB_; ++b) part[(((grp - 1) * NW + wave) * MB * NB_ + a * NB_ + b) * 64 + lane] = acc[a][b];
    __syncthreads();
    if (grp > 0) return;
#pragma unroll
    for (int s = 0; s < KS - 1; ++s)
#pragma unroll
      for (int a = 0; a < MB; ++a)
#pragma unroll
        for (int b = 0; b < NB_; ++b) acc[a][b] += part[((s * NW + wave) * MB * NB_ + a * NB_ + b) * 64 + lane];
  }
  finish_rows_any<MB, NB_>(p, epi, tm * BM + 16 * MB * wm + l16, tn * BNS + 16 * NB_ * wn + 4 * g, acc);
}

// -------------------------------------------------------------------- few rows
// The waves of a workgroup share its columns and take every NW-th step of 128 bytes of K, joined
// in LDS: whole sums, so in any order the same bits.
template <int NW, int MB, int NBW>
__device__ __forceinline__ void join_waves(const IntGemmArgs& p, int epi, i32x4* part, const i32x4 (&acc)[MB][NBW], int nt,
                                           int wave, int lane) {
#pragma unroll
  for (int a = 0; a < MB; ++a)
#pragma unroll
    for (int b = 0; b < NBW; ++b) part[(wave * MB * NBW + a * NBW + b) * 64 + lane] = acc[a][b];
  __syncthreads();
  for (int i = wave; i < MB * NBW; i += NW) {
    i32x4 sum[1][1] = {{part[i * 64 + lane]}};
#pragma unroll
    for (int w = 1; w < NW; ++w) sum[0][0] += part[(w * MB * NBW + i) * 64 + lane];
    finish_rows_any<1, 1>(p, epi, 16 * (i / NBW) + (lane & 15), nt + 16 * (i % NBW) + 4 * (lane >> 4), sum);
  }
}

// At most 16 MB rows: every wave has a ring of S stages in LDS to itself (its steps' X and W
// rows), and waits for nothing but its own loads.
template <int NW, int MB, int NBW, int S>
__global__ __launch_bounds__(64 * NW) void int_gemm_split(const IntGemmArgs p, int epi) {
  constexpr int INS = 2 * (MB + NBW), STAGE = INS * 1024;
  static_assert(NW * S * STAGE <= 160 * 1024 && S >= 2, "LDS");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[NW * S * STAGE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int nt = blockIdx.x * 16 * NBW;
  const int ldx = static_cast<int>(p.ldx), ldw = static_cast<int>(p.ldw);
  const char* x_base = uniform_ptr(p.x);
  const char* w_base = uniform_ptr(p.w + static_cast<int64_t>(nt) * p.ldw);
  uint32_t off[INS];
#pragma unroll
  for (int j = 0; j < INS; ++j) {
    const int r = 8 * j + (lane >> 3);   // X rows first
    const int row = j < 2 * MB ? min(r, p.M - 1) * ldx : min(r - 16 * MB, p.N - 1 - nt) * ldw;
    off[j] = static_cast<uint32_t>(row + ((lane & 7) ^ swz(r)) * 16);
  }
  const uint32_t lds0 = lds_address(smem) + wave * (S * STAGE);
  const unsigned char* ring = smem + wave * (S * STAGE);
  const int chunks = (p.K + 15) / 16, nk = (chunks + 7) / 8, last = chunks - 8 * (nk - 1);
  auto issue = [&](int kt, int slot) __attribute__((always_inline)) {
    const bool end = kt == nk - 1 && last < 8;   // (the row's last chunk in the place of missing ones)
#pragma unroll
    for (int j = 0; j < INS; ++j) {
      uint32_t o = off[j];
      if (end) {
        const int c = (lane & 7) ^ swz(8 * j + (lane >> 3));
        o -= 16u * (c - min(c, last - 1));
      }
      lds_dma16((j < 2 * MB ? x_base : w_base) + kt * BK, o, lds0 + slot * STAGE + 1024u * j);
    }
  };
  i32x4 acc[MB][NBW];
#pragma unroll
  for (int a = 0; a < MB; ++a)
#pragma unroll
    for (int b = 0; b < NBW; ++b) acc[a][b] = i32x4{0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < S; ++i)
    if (wave + NW * i < nk) issue(wave + NW * i, i);
  int slot = 0;
  for (int kt = wave; kt < nk; kt += NW) {
    if (kt + NW * (S - 1) < nk) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 1) * INS) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const unsigned char* st = ring + slot * STAGE + l16 * BK;
    i32x4 fx[2][MB], fw[2][NBW];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      const int c = 16 * ((4 * kk + g) ^ swz(l16));
#pragma unroll
      for (int a = 0; a < MB; ++a) fx[kk][a] = *reinterpret_cast<const i32x4*>(st + 16 * BK * a + c);
#pragma unroll
      for (int b = 0; b < NBW; ++b) fw[kk][b] = *reinterpret_cast<const i32x4*>(st + 16 * BK * (MB + b) + c);
      if (kt == nk - 1 && 4 * kk + g >= last)
#pragma unroll
        for (int b = 0; b < NBW; ++b) fw[kk][b] = i32x4{0, 0, 0, 0};
    }
    // the fragments are in registers before the stage is requested again
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    if (kt + NW * S < nk) issue(kt + NW * S, slot);
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int a = 0; a < MB; ++a)
#pragma unroll
        for (int b = 0; b < NBW; ++b)
          acc[a][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[kk][b], fx[kk][a], acc[a][b], 0, 0, 0);
    slot = slot == S - 1 ? 0 : slot + 1;
  }
  __syncthreads();   // (the rings become the join's)
  join_waves<NW, MB, NBW>(p, epi, reinterpret_cast<i32x4*>(smem), acc, nt, wave, lane);
}

}  // namespace

template <int BM, int EPI, typename ResT, typename OutT>
static void launch_tile(hipStream_t st, const IntGemmArgs& a) {
  const int tiles_m = (a.M + BM - 1) / BM, tiles_n = (a.N + BN - 1) / BN;
  const int per_xcd = (tiles_m * tiles_n + kNumXcd - 1) / kNumXcd;
  hipLaunchKernelGGL((int_gemm_kernel<BM, EPI, ResT, OutT>), dim3(per_xcd * kNumXcd), dim3(NT), 0, st, a, tiles_m,
                     tiles_n, per_xcd);
}

template <int WM_, int WN_, int MB, int NB_, int S, int KS>
static void launch_small(hipStream_t st, int epi, const IntGemmArgs& a) {
  constexpr int BM = 16 * MB * WM_, BNS = 16 * NB_ * WN_;
  const int tiles_m = (a.M + BM - 1) / BM, tiles_n = (a.N + BNS - 1) / BNS;
  const int wgs = (tiles_m * tiles_n + kNumXcd - 1) / kNumXcd * kNumXcd;
  hipLaunchKernelGGL((int_gemm_small<WM_, WN_, MB, NB_, S, KS>), dim3(wgs), dim3(64 * WM_ * WN_ * KS), 0, st, a, epi,
                     tiles_m, tiles_n);
}

template <int NW, int MB, int NBW, int S>
static void launch_split_t(hipStream_t st, int epi, const IntGemmArgs& a) {
  hipLaunchKernelGGL((int_gemm_split<NW, MB, NBW, S>), dim3((a.N + 16 * NBW - 1) / (16 * NBW)), dim3(64 * NW), 0, st, a,
                     epi);
}

// Few rows: as few columns to a workgroup as one round of the chip allows (one workgroup holds a
// CU's LDS).  us at 16, 32 and 64 columns a workgroup: one row, 1536 x 8960 (96 workgroups of 16
// columns) 5.9, 7.4, 9.6; 5120 x 13824 (320) 20.2, 15.9, 23.2; 13824 x 5120 (864) 20.5, 16.5, 14.9.
template <int MB>
static void launch_split(hipStream_t st, int epi, const IntGemmArgs& a) {
  const int blocks = (a.N + 15) / 16, per = (blocks + 255) / 256;
  if constexpr (MB == 1) {
    if (per == 1) launch_split_t<8, 1, 1, 5>(st, epi, a);
    else if (per == 2) launch_split_t<8, 1, 2, 3>(st, epi, a);
    else if (per == 3) launch_split_t<8, 1, 3, 2>(st, epi, a);
    else launch_split_t<8, 1, 4, 2>(st, epi, a);
  } else if constexpr (MB == 2) {
    if (per == 1) launch_split_t<8, 2, 1, 3>(st, epi, a);
    else if (per == 2) launch_split_t<8, 2, 2, 2>(st, epi, a);
    else if (per == 3) launch_split_t<8, 2, 3, 2>(st, epi, a);
    else launch_split_t<4, 2, 4, 3>(st, epi, a);
  } else {
    if (per == 1) launch_split_t<8, 4, 1, 2>(st, epi, a);
    else if (per == 2) launch_split_t<4, 4, 2, 3>(st, epi, a);
    else if (per == 3) launch_split_t<4, 4, 3, 2>(st, epi, a);
    else launch_split_t<4, 4, 4, 2>(st, epi, a);
  }
}

// The kernel of a product of more than 64 rows, by its estimated end (us):
//   start + rounds (fixed + steps (step + load fill))
// with the tiles over the CUs' places (256; two of the 64 x 64 tiles share a CU, and are counted by
// half rounds), `fill` the share of the places taken, and K in steps of 128.  The constants are
// fitted to warm calls of one card.  Estimate and measurement of the kernel taken and of the next
// best, M x N x K: 128 x 1536 x 8960 16.1 / 15.7 (32 x 64), 21.4 / 21.6; 300 x 2600 x 700 5.4 / 5.4
// (64 x 64), 6.5 / 7.0; 512 x 1536 x 1536 7.3 / 6.8 (64 x 64 in two groups), 7.4 / 7.3; 256 x 5120 x
// 5120 18.4 / 17.9 (64 x 128 in two groups), 24.0 / 21.6; 512 x 5120 x 5120 28.3 / 29.0 (128 x 128),
// 34.5 / 34.5; 1560 x 4608 x 1536 17.0 / 17.8 (128 x 256), 18.7 / 21.1; 4680 x 5120 x 13824 241 / 253
// (192 x 256), 289 / 272; 16384 x 8192 x 8192 767 / 785 (256 x 256), 808 / 826.  Of 45 products
// measured on all of them it takes the fastest of 36.  Of the others small ones lose up to 1.2 us; large
// results of few steps, whose bytes the estimate does not know, up to 19%: 5000 x 5000 x 128 26.0 us for 22.3,
// 9360 x 1536 x 256 with an fp32 residual 35.1 for 29.5 (both 128 x 256 for 256 x 256).
enum Tile { kT32x64, kT64x64, kT64x64Pair, kT64x128, kT128x128, kT128x256, kT192x256, kT256x256, kTiles };
static Tile choose_tile(int M, int N, int K) {
  struct Cost {
    int m, n;
    double start, fixed, step, load;
  };
  static const Cost cost[kTiles] = {{32, 64, 1.5, 1.5, 0.15, 0.10},   {64, 64, 2.3, 1.0, 0.345, 0},
                                    {64, 64, 1.7, 2.5, 0.24, 0.03},   {64, 128, 1.7, 2.5, 0.33, 0.04},
                                    {128, 128, 3.0, 3.0, 0.52, 0.06}, {128, 256, 3.0, 3.5, 0.61, 0.29},
                                    {192, 256, 3.0, 6.5, 0.70, 0.35}, {256, 256, 3.0, 8.5, 0.91, 0.45}};
  const int steps = (K + 127) / 128;
  int best = 0;
  double least = 0;
  for (int i = 0; i < kTiles; ++i) {
    const Cost& c = cost[i];
    const double tiles = static_cast<double>((M + c.m - 1) / c.m) * ((N + c.n - 1) / c.n);
    double rounds = ceil(tiles / 256), fill = tiles / (256 * rounds);
    if (i == kT64x64) rounds = std::max(1.0, 0.5 * ceil(tiles / 128));
    const double t = c.start + rounds * (c.fixed + steps * (c.step + c.load * fill));
    if (i == 0 || t < least) least = t, best = i;
  }
  return static_cast<Tile>(best);
}

template <int EPI, typename ResT, typename OutT>
static void launch_t(hipStream_t st, Tile tile, const IntGemmArgs& a) {
  if (tile == kT128x256) launch_tile<128, EPI, ResT, OutT>(st, a);
  else if (tile == kT192x256) launch_tile<192, EPI, ResT, OutT>(st, a);
  else launch_tile<256, EPI, ResT, OutT>(st, a);
}

hipError_t launch_int_gemm(hipStream_t st, int epi, const IntGemmArgs& args) {
  if (args.M == 0) return hipSuccess;
  IntGemmArgs a = args;
  // elements of a row that may be read or written at once
  auto width = [](const void* p, int size, int64_t ld) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(ld) * size;
    return at % (4 * size) == 0 ? 4 : at % (2 * size) == 0 ? 2 : 1;
  };
  a.width_cols = std::min(std::min(width(a.sw, 4, 4), width(a.bias, 2, 4)),
                          std::min(width(a.mod, 4, a.mod ? a.N : 4), width(a.table, 4, 4)));
  a.width_res = width(a.res, a.res_f32 ? 4 : 2, a.ldr);
  a.width_y = width(a.y, a.y_f32 ? 4 : 2, a.ldy);
  if (a.M <= 64) {
    if (a.M <= 16) launch_split<1>(st, epi, a);
    else if (a.M <= 32) launch_split<2>(st, epi, a);
    else launch_split<4>(st, epi, a);
    return hipGetLastError();
  }
  const Tile tile = choose_tile(a.M, a.N, a.K);
  switch (tile) {
    case kT32x64: launch_small<2, 2, 1, 2, 3, 4>(st, epi, a); return hipGetLastError();
    case kT64x64: launch_small<2, 2, 2, 2, 5, 1>(st, epi, a); return hipGetLastError();
    case kT64x64Pair: launch_small<2, 2, 2, 2, 5, 2>(st, epi, a); return hipGetLastError();
    case kT64x128: launch_small<2, 2, 2, 4, 3, 2>(st, epi, a); return hipGetLastError();
    case kT128x128: launch_small<2, 4, 4, 2, 5, 1>(st, epi, a); return hipGetLastError();
    default: break;
  }
  const bool rf = a.res_f32, of = a.y_f32;
#define ARDIT_INT_GEMM(E, R, O) launch_t<E, R, O>(st, tile, a)
#define ARDIT_INT_RES(E)                                  \
  if (rf && of) ARDIT_INT_GEMM(E, float, float);          \
  else if (rf) ARDIT_INT_GEMM(E, float, bf16_t);          \
  else if (of) ARDIT_INT_GEMM(E, bf16_t, float);          \
  else ARDIT_INT_GEMM(E, bf16_t, bf16_t);
  switch (epi) {
    case kEpiBias:
      if (of) ARDIT_INT_GEMM(kEpiBias, bf16_t, float);
      else ARDIT_INT_GEMM(kEpiBias, bf16_t, bf16_t);
      break;
    case kEpiBiasGelu: ARDIT_INT_GEMM(kEpiBiasGelu, bf16_t, bf16_t); break;
    case kEpiBiasGateRes: ARDIT_INT_RES(kEpiBiasGateRes) break;
    case kEpiBiasRes: ARDIT_INT_RES(kEpiBiasRes) break;
    default: return hipErrorInvalidValue;
  }
#undef ARDIT_INT_RES
#undef ARDIT_INT_GEMM
  return hipGetLastError();
}

}  // namespace ardit
