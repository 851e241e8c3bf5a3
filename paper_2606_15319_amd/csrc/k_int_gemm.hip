// Linear layers over 8-bit integer codes: y = epilogue(sx_i sw_j sum_k X_ik W_jk).
//
// X [M][K] and W [N][K] are both K-contiguous.  v_mfma_i32_16x16x64_i8 sums exactly in 32 bits
// (|sum| <= 2^30 at K = 65536), at twice the bf16 rate per operand byte.  The MFMA computes
// C^T = W X^T: W rows feed the A operand and X rows the B operand, so a lane ends with one row i
// and four consecutive columns j of every 16 x 16 block.
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

// Four consecutive elements from n on, those before `end`; whole where `vec`.
template <typename T>
__device__ __forceinline__ void load4(const T* p, int left, bool vec, float* f) {
  if (vec && left >= 4) {
    if constexpr (sizeof(T) == 4) {
      const float4 r = *reinterpret_cast<const float4*>(p);
      f[0] = r.x; f[1] = r.y; f[2] = r.z; f[3] = r.w;
    } else {
      const uint2 r = *reinterpret_cast<const uint2*>(p);
      f[0] = __uint_as_float(r.x << 16); f[1] = __uint_as_float(r.x & 0xffff0000u);
      f[2] = __uint_as_float(r.y << 16); f[3] = __uint_as_float(r.y & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = e < left ? as_float(p[e]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store4(T* p, int left, bool vec, const float* y) {
  if (vec && left >= 4) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(p) = make_float4(y[0], y[1], y[2], y[3]);
    else *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
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
  Scale s[NB_][4];
  float bias[NB_][4];
};
template <int NB_>
__device__ __forceinline__ void load_columns(const IntGemmArgs& p, int n0, Columns<NB_>& c) {
#pragma unroll
  for (int b = 0; b < NB_; ++b) {
    const int n = n0 + 16 * b, left = p.N - n;
    float sw[4];
    load4(p.sw + n, left, p.vec_cols, sw);
#pragma unroll
    for (int e = 0; e < 4; ++e) c.s[b][e] = split_scale(sw[e]), c.bias[b][e] = 0.f;
    if (p.bias) load4(p.bias + n, left, p.vec_cols, c.bias[b]);
  }
}

// Row m of a lane's columns: epilogue and store.
template <int EPI, typename ResT, typename OutT, int NB_>
__device__ __forceinline__ void finish_row(const IntGemmArgs& p, int m, int n0, const i32x4 (&acc)[NB_],
                                           const Columns<NB_>& c) {
  const Scale sx = split_scale(p.sx[m]);
  OutT* o = static_cast<OutT*>(p.y) + m * p.ldy;
  const float* mod = nullptr;
  const float* tab = nullptr;
  if (EPI == kEpiBiasGateRes) {
    mod = p.mod + (static_cast<size_t>(fdiv(m, p.rows_per_stream)) * 6 + p.gate_row) * p.N;
    if (p.table) tab = p.table + static_cast<size_t>(p.gate_row) * p.N;
  }
  float res[NB_][4], gate[NB_][4];
#pragma unroll
  for (int b = 0; b < NB_; ++b) {
    const int n = n0 + 16 * b, left = p.N - n;
    if (EPI == kEpiBiasRes || EPI == kEpiBiasGateRes)
      load4(static_cast<const ResT*>(p.res) + m * p.ldr + n, left, p.vec_res, res[b]);
    if (EPI == kEpiBiasGateRes) {
      load4(mod + n, left, p.vec_cols, gate[b]);
      if (tab) {
        float t[4];
        load4(tab + n, left, p.vec_cols, t);
#pragma unroll
        for (int e = 0; e < 4; ++e) gate[b][e] += t[e];
      }
    }
  }
#pragma unroll
  for (int b = 0; b < NB_; ++b) {
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      y[e] = finish<EPI>(acc[b][e], sx, c.s[b][e], c.bias[b][e], EPI >= kEpiBiasGateRes ? res[b][e] : 0.f,
                         EPI == kEpiBiasGateRes ? gate[b][e] : 0.f);
    store4(o + n0 + 16 * b, p.N - n0 - 16 * b, p.vec_y, y);
  }
}

// ------------------------------------------------------------------ large tiles
constexpr int BN = 256, BK = 128, NT = 512, NWAVES = 8;   // (a K step is 128 bytes of every row)
constexpr int WN = 64, NB = WN / 16, NWN = BN / WN;
constexpr int W_INS = BN * BK / 1024 / NWAVES;
constexpr int GROUP_M = 8;   // m-tiles per raster group (L2 reuse of W columns)
// LDS: a ring of five places, each for one operand of a step (X0 W0 X1 W1 X2 ...)
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

  const int n0 = tn * BN + WN * wn + 4 * g;
  Columns<NB> col;
  load_columns<NB>(p, n0, col);
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) {
    const int m = tm * BM + WM * wm + 16 * mb + l16;
    if (m < p.M) finish_row<EPI, ResT, OutT, NB>(p, m, n0, acc[mb], col);
  }
}


// ------------------------------------------------------------------ small tiles
// Tiles of 16 MB WM_ x 16 NB WN_ on WM_ x WN_ waves for products too small to give every CU a
// large tile.  S - 1 K steps are under way through a ring of S stages in LDS; one barrier a step
// publishes stage kt and closes the reads of stage kt - 1, into which step kt + S - 1 is requested.
template <int WM_, int WN_, int MB, int NB_, int S, int EPI, typename ResT, typename OutT>
__global__ __launch_bounds__(64 * WM_ * WN_, 1) void int_gemm_small(const IntGemmArgs p, int tiles_m, int tiles_n) {
  constexpr int NW = WM_ * WN_, BM = 16 * MB * WM_, BNS = 16 * NB_ * WN_;
  constexpr int AB = BM * BK, WB = BNS * BK, STAGE = AB + WB;
  constexpr int A_INS = AB / 1024 / NW, WI = WB / 1024 / NW, INS = A_INS + WI;
  static_assert(A_INS * NW * 1024 == AB && WI * NW * 1024 == WB, "whole loads per wave");
  static_assert(S * STAGE <= 160 * 1024 && S >= 3 && (S - 2) * INS < 64, "LDS, counter");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[S * STAGE];
  // XCD-aware order: each XCD takes a run of column tiles with all their row tiles
  const int total = tiles_m * tiles_n, per_xcd = (total + kNumXcd - 1) / kNumXcd;
  const int L = static_cast<int>(blockIdx.x % kNumXcd) * per_xcd + static_cast<int>(blockIdx.x / kNumXcd);
  if (L >= total) return;
  const int tm = L % tiles_m, tn = L / tiles_m;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
  const uint32_t lds_a = lds_address(smem) + 1024u * (wave * A_INS), lds_w = lds_address(smem) + AB + 1024u * (wave * WI);
  const int chunks = (p.K + 15) / 16, nk = (chunks + 7) / 8, last = chunks - 8 * (nk - 1);
  auto issue = [&](int kt, int slot) __attribute__((always_inline)) {
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
    if (i < nk) issue(i, i);
  int slot = 0;
  for (int kt = 0; kt < nk; ++kt) {
    if (kt + S - 1 <= nk) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 2) * INS));
    else asm volatile("s_waitcnt vmcnt(0)");
    __syncthreads();
    if (kt + S - 1 < nk) issue(kt + S - 1, slot == 0 ? S - 1 : slot - 1);
    const unsigned char* sa = smem + slot * STAGE + (16 * MB * wm + l16) * BK;
    const unsigned char* sw = smem + slot * STAGE + AB + (16 * NB_ * wn + l16) * BK;
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
    slot = slot == S - 1 ? 0 : slot + 1;
  }
  const int n0 = tn * BNS + 16 * NB_ * wn + 4 * g;
  Columns<NB_> col;
  load_columns<NB_>(p, n0, col);
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) {
    const int m = tm * BM + 16 * (MB * wm + mb) + l16;
    if (m < p.M) finish_row<EPI, ResT, OutT, NB_>(p, m, n0, acc[mb], col);
  }
}

// -------------------------------------------------------------------- few rows
// 16 MB rows at most: the weights are read once, straight into registers, 16 NBW columns to a
// workgroup whose eight waves take every eighth step of 128 bytes of K and are joined in LDS.
// Lane (l16, g) holds bytes 32 g .. 32 g + 31 of a step of its row (both operands alike), so that
// the two loads of a step cover whole lines.  U steps are requested together.
template <int MB, int NBW, int U, int EPI, typename ResT, typename OutT>
__global__ __launch_bounds__(512) void int_gemm_rows(const IntGemmArgs p) {
  __shared__ __attribute__((aligned(16))) i32x4 part[8][MB * NBW][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int nt = blockIdx.x * 16 * NBW;
  const int8_t* xr[MB];
  const int8_t* wr[NBW];
#pragma unroll
  for (int a = 0; a < MB; ++a) xr[a] = p.x + static_cast<int64_t>(min(16 * a + l16, p.M - 1)) * p.ldx;
#pragma unroll
  for (int b = 0; b < NBW; ++b) wr[b] = p.w + static_cast<int64_t>(min(nt + 16 * b + l16, p.N - 1)) * p.ldw;
  i32x4 acc[MB][NBW];
#pragma unroll
  for (int a = 0; a < MB; ++a)
#pragma unroll
    for (int b = 0; b < NBW; ++b) acc[a][b] = i32x4{0, 0, 0, 0};
  const int chunks = (p.K + 15) / 16, nk = (chunks + 7) / 8;
  for (int t0 = wave; t0 < nk; t0 += 8 * U) {
    i32x4 fw[U][2][NBW], fx[U][2][MB];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int c = 8 * (t0 + 8 * u) + 2 * g + h;
        const bool in = c < chunks;
#pragma unroll
        for (int b = 0; b < NBW; ++b) {
          fw[u][h][b] = i32x4{0, 0, 0, 0};
          if (in) fw[u][h][b] = *reinterpret_cast<const i32x4*>(wr[b] + 16 * c);
        }
#pragma unroll
        for (int a = 0; a < MB; ++a) {
          fx[u][h][a] = i32x4{0, 0, 0, 0};
          if (in) fx[u][h][a] = *reinterpret_cast<const i32x4*>(xr[a] + 16 * c);
        }
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int a = 0; a < MB; ++a)
#pragma unroll
          for (int b = 0; b < NBW; ++b)
            acc[a][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[u][h][b], fx[u][h][a], acc[a][b], 0, 0, 0);
  }
#pragma unroll
  for (int a = 0; a < MB; ++a)
#pragma unroll
    for (int b = 0; b < NBW; ++b) part[wave][a * NBW + b][lane] = acc[a][b];
  __syncthreads();
  // wave w ends blocks w, w + 8, ...
  for (int i = wave; i < MB * NBW; i += 8) {
    i32x4 sum[1] = {part[0][i][lane]};
#pragma unroll
    for (int w = 1; w < 8; ++w) sum[0] += part[w][i][lane];
    const int n0 = nt + 16 * (i % NBW) + 4 * g, m = 16 * (i / NBW) + l16;
    Columns<1> col;
    load_columns<1>(p, n0, col);
    if (m < p.M) finish_row<EPI, ResT, OutT, 1>(p, m, n0, sum, col);
  }
}

}  // namespace

template <int BM, int EPI, typename ResT, typename OutT>
static void launch_tile(hipStream_t st, const IntGemmArgs& a) {
  const int tiles_m = (a.M + BM - 1) / BM, tiles_n = (a.N + BN - 1) / BN;
  const int per_xcd = (tiles_m * tiles_n + kNumXcd - 1) / kNumXcd;
  hipLaunchKernelGGL((int_gemm_kernel<BM, EPI, ResT, OutT>), dim3(per_xcd * kNumXcd), dim3(NT), 0, st, a, tiles_m,
                     tiles_n, per_xcd);
}

template <int WM_, int WN_, int MB, int NB_, int S, int EPI, typename ResT, typename OutT>
static void launch_small(hipStream_t st, const IntGemmArgs& a) {
  constexpr int BM = 16 * MB * WM_, BNS = 16 * NB_ * WN_;
  const int tiles_m = (a.M + BM - 1) / BM, tiles_n = (a.N + BNS - 1) / BNS;
  const int wgs = (tiles_m * tiles_n + kNumXcd - 1) / kNumXcd * kNumXcd;
  hipLaunchKernelGGL((int_gemm_small<WM_, WN_, MB, NB_, S, EPI, ResT, OutT>), dim3(wgs), dim3(64 * WM_ * WN_), 0, st, a,
                     tiles_m, tiles_n);
}

template <int MB, int NBW, int U, int EPI, typename ResT, typename OutT>
static void launch_rows(hipStream_t st, const IntGemmArgs& a) {
  hipLaunchKernelGGL((int_gemm_rows<MB, NBW, U, EPI, ResT, OutT>), dim3((a.N + 16 * NBW - 1) / (16 * NBW)), dim3(512), 0,
                     st, a);
}

template <int EPI, typename ResT, typename OutT>
static void launch_t(hipStream_t st, const IntGemmArgs& a) {
  const char* force = getenv("ARDIT_LAB_BM");
  const int bm = force ? atoi(force) : a.M <= 32 ? 32 : 64;
  if (bm == 1 && a.M <= 16) return launch_rows<1, 1, 4, EPI, ResT, OutT>(st, a);
  if (bm == 2 && a.M <= 16) return launch_rows<1, 2, 4, EPI, ResT, OutT>(st, a);
  if (bm == 31 && a.M <= 32) return launch_rows<2, 1, 4, EPI, ResT, OutT>(st, a);
  if (bm == 32 && a.M <= 32) return launch_rows<2, 2, 3, EPI, ResT, OutT>(st, a);
  if (bm == 33 && a.M <= 64) return launch_rows<4, 1, 2, EPI, ResT, OutT>(st, a);
  if (bm == 34 && a.M <= 64) return launch_rows<4, 2, 2, EPI, ResT, OutT>(st, a);
  if (bm == 65) return launch_small<2, 2, 1, 2, 6, EPI, ResT, OutT>(st, a);   // 32 x 64
  if (bm == 66) return launch_small<2, 4, 2, 2, 5, EPI, ResT, OutT>(st, a);   // 64 x 128
  if (bm == 67) return launch_small<2, 4, 4, 2, 5, EPI, ResT, OutT>(st, a);   // 128 x 128
  if (bm == 128) return launch_tile<128, EPI, ResT, OutT>(st, a);
  if (bm == 192) return launch_tile<192, EPI, ResT, OutT>(st, a);
  if (bm == 256) return launch_tile<256, EPI, ResT, OutT>(st, a);
  return launch_small<2, 2, 2, 2, 5, EPI, ResT, OutT>(st, a);   // 64 x 64
}

hipError_t launch_int_gemm(hipStream_t st, int epi, const IntGemmArgs& args) {
  if (args.M == 0) return hipSuccess;
  IntGemmArgs a = args;
  auto quads = [](const void* p, int size, int64_t ld) {
    return reinterpret_cast<uintptr_t>(p) % (4 * size) == 0 && ld % 4 == 0;
  };
  a.vec_cols = quads(a.sw, 4, a.N) && (!a.bias || quads(a.bias, 2, a.N)) && quads(a.mod, 4, a.N) &&
               quads(a.table, 4, a.N);
  a.vec_res = quads(a.res, a.res_f32 ? 4 : 2, a.ldr);
  a.vec_y = quads(a.y, a.y_f32 ? 4 : 2, a.ldy);
  const bool rf = a.res_f32, of = a.y_f32;
#define ARDIT_INT_GEMM(E, R, O) launch_t<E, R, O>(st, a)
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
