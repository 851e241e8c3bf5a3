// Rows to 8-bit integer codes and back, and the norm that feeds a linear layer over them.
//
// A row y with m = max|y| takes the scale m / 127 and the codes rint(127 y / m), decided exactly:
// the fp32 estimate t = y (127 / m) is off by a bound that the kernel knows, so only elements
// whose t lies that near to a half (3 in 10^5 when quantised, 2 in 10^4 when normed, so one in most
// rows of 5120) are decided again in fp64, by the sign of 254 |y| - (2 k + 1) m.  Their chunks of 8 are
// read again for that (unrolled over a row in registers the code for it would fill the caches).
//
// Quantising (2 or 4 bytes read an element, 1 written) and reading back are bound by HBM; the norm by its chain
// of dependent steps too (1.9 to 3.5 TB/s).  A row is held in registers, so it is read once: by one wave up
// to 5120 elements when quantised and always when normed, wider or few rows by several.  What a wave does
// once a row (reductions, divisions) costs as much as 30 to 40 elements a lane, and shared by more
// waves it is done more often: 13824 rows of 5120 quantised by five waves each 62 us, by one 53
// (4.0 TB/s; 4680 rows of 13824 by three 50, 3.9).
#include <algorithm>

#include "launch.h"

namespace ardit {

namespace {

// t + kMagic is a whole number in the low mantissa bits, rounded to nearest even (|t| < 2^21)
constexpr float kMagic = 12582912.f;   // 1.5 * 2^23

__device__ __forceinline__ uint32_t abs_bits(float f) { return __float_as_uint(f) & 0x7fffffffu; }

// low bytes of four words
__device__ __forceinline__ uint32_t pack_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x0c0c0400u);
  const uint32_t hi = __builtin_amdgcn_perm(d, c, 0x04000c0cu);
  return lo | hi;
}

// Value of another lane of the same 16, N places round; all lanes then hold a row's reduction after
// N = 8, 4, 2, 1, and the wave's after the two swaps of rows.
template <int N>
__device__ __forceinline__ uint32_t rotated(uint32_t v) {
  return static_cast<uint32_t>(
      __builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x120 + N, 0xf, 0xf, false));
}
template <int N>
__device__ __forceinline__ double rotated(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint64_t lo = rotated<N>(static_cast<uint32_t>(b)), hi = rotated<N>(static_cast<uint32_t>(b >> 32));
  return __builtin_bit_cast(double, hi << 32 | lo);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max(v, rotated<8>(v));
  v = max(v, rotated<4>(v));
  v = max(v, rotated<2>(v));
  v = max(v, rotated<1>(v));
  auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(r[0], r[1]);
  r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(r[0], r[1]);
}
template <typename Op>
__device__ __forceinline__ double wave_join(double v, Op op) {
  v = op(v, rotated<8>(v));
  v = op(v, rotated<4>(v));
  v = op(v, rotated<2>(v));
  v = op(v, rotated<1>(v));
  const double w = op(v, __shfl_xor(v, 16, kWave));
  return op(w, __shfl_xor(w, 32, kWave));
}

__device__ __forceinline__ float load_elem(const void* p, bool f32, size_t at) {
  return f32 ? static_cast<const float*>(p)[at] : bf2f(static_cast<const bf16_t*>(p)[at]);
}

// Elements 8 c .. 8 c + 7 of a row of D as they lie in memory, zero past its end.  kBf16, kF32: the
// row starts on 16 bytes and D is a multiple of 8; kAny: either type from anywhere.
enum : int { kBf16 = 0, kF32 = 1, kAny = 2 };
template <int F>
struct Chunk {
  uint4 v[F == kBf16 ? 1 : 2];
};
template <int F>
__device__ __forceinline__ void load_chunk(const void* row, bool f32, int c, int D, Chunk<F>& q) {
  if constexpr (F == kAny) {
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = 8 * c + e < D ? load_elem(row, f32, 8 * c + e) : 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      q.v[h] = make_uint4(__float_as_uint(f[4 * h]), __float_as_uint(f[4 * h + 1]), __float_as_uint(f[4 * h + 2]),
                          __float_as_uint(f[4 * h + 3]));
  } else {
    const uint4* p = static_cast<const uint4*>(row) + (F == kBf16 ? c : 2 * c);
    q.v[0] = p[0];
    if constexpr (F == kF32) q.v[1] = p[1];
  }
}
template <int F>
__device__ __forceinline__ void clear(Chunk<F>& q) {
#pragma unroll
  for (int h = 0; h < (F == kBf16 ? 1 : 2); ++h) q.v[h] = make_uint4(0, 0, 0, 0);
}
template <int F>
__device__ __forceinline__ void to_floats(const Chunk<F>& q, float* f) {
  if constexpr (F == kBf16) {
    unpack8(q.v[0], f);
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f[4 * h] = __uint_as_float(q.v[h].x);
      f[4 * h + 1] = __uint_as_float(q.v[h].y);
      f[4 * h + 2] = __uint_as_float(q.v[h].z);
      f[4 * h + 3] = __uint_as_float(q.v[h].w);
    }
  }
}

__device__ __forceinline__ const void* row_at(const void* p, bool f32, int64_t elem) {
  return static_cast<const char*>(p) + elem * (f32 ? 4 : 2);
}

// max(a, |b|, |c|) in one instruction; a NaN among them is passed over
__device__ __forceinline__ float max_abs(float a, float b, float c) { return fmaxf(a, fmaxf(fabsf(b), fabsf(c))); }

// Codes of eight estimates t = y inv, and how far the furthest lies from its whole number.
__device__ __forceinline__ uint2 codes8(const float* y, float inv, float* far) {
  uint32_t w[8];
  float d[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float r = fmaf(y[e], inv, kMagic);
    d[e] = fmaf(y[e], inv, kMagic - r);
    w[e] = __float_as_uint(r);
  }
  *far = 0.f;
#pragma unroll
  for (int e = 0; e < 8; e += 2) *far = max_abs(*far, d[e], d[e + 1]);
  return make_uint2(pack_bytes(w[0], w[1], w[2], w[3]), pack_bytes(w[4], w[5], w[6], w[7]));
}

// The code of y in a row whose largest magnitude is m > 0; k_known: a whole number below 127 |y| / m
// that the code is at or one above, or -1 for unknown.
__device__ __forceinline__ int exact_code(double y, double m, float k_known) {
#pragma clang fp contract(off)   // (both products of `side` rounded alike, so that halves of m tie)
  const double a = fabs(y);
  double k = k_known;
  if (k_known < 0.f) k = floor(127.0 * (a / m));   // (or one off: the border decides)
  const double side = 254.0 * a - (2.0 * k + 1.0) * m;
  if (side > 0.0 || (side == 0.0 && (static_cast<int>(k) & 1))) k += 1.0;
  const int q = static_cast<int>(k);
  return y < 0.0 ? -q : q;
}

// codes8 with the open elements (all where inv is no number, and thr -1) decided from exact(e).
template <typename Y>
__device__ __forceinline__ uint2 settled8(const float* y, float inv, float thr, Y exact, double m) {
  uint32_t w[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float r = fmaf(y[e], inv, kMagic);
    w[e] = __float_as_uint(r);
    // (thr >= 0: t is less than a half off, so the code is |t|'s floor or one above)
    if (!(fabsf(fmaf(y[e], inv, kMagic - r)) <= thr))
      w[e] = static_cast<uint32_t>(exact_code(exact(e), m, thr < 0.f ? -1.f : floorf(fabsf(y[e] * inv))));
  }
  return make_uint2(pack_bytes(w[0], w[1], w[2], w[3]), pack_bytes(w[4], w[5], w[6], w[7]));
}

// Results are written past the L2, whose dirty lines a kernel has to flush when it ends: with plain
// stores the norm of 4680 x 5120 from fp32 takes 6.5 us longer, and the fp32 values of
// 4680 x 13824 codes 98 us for 56.  (Rows that are no 16-byte vectors, and bf16 values, take plain stores.)
__device__ __forceinline__ void store_codes(uint2* p, uint2 w) {
  __builtin_nontemporal_store(static_cast<uint64_t>(w.y) << 32 | w.x, reinterpret_cast<uint64_t*>(p));
}

constexpr uint32_t kInfBits = 0x7f800000u;
constexpr uint32_t kWideBits = 0x49800000u;   // 2^20

}  // namespace

// ------------------------------------------------------------------- quantise
// The waves of a workgroup hold a row, up to 512 MAXC elements each; ONE: a row is a wave's, and a
// workgroup's four waves have one each.
template <int MAXC, bool ONE, int F>
__global__ __launch_bounds__(ONE ? 256 : 1024) void int_quantize_kernel(const void* x, int x_f32, int rows, int cols,
                                                                        int64_t ldx, int8_t* codes, int64_t ldc,
                                                                        float* scales) {
  __shared__ uint32_t part[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t0 = ONE ? lane : static_cast<int>(threadIdx.x), stride = ONE ? 64 : static_cast<int>(blockDim.x);
  const int nchunk = 2 * ((cols + 15) / 16);          // (whole 16 bytes of codes)
  const bool f32 = F == kAny ? x_f32 : F == kF32;
  const int row = ONE ? static_cast<int>(blockIdx.x) * 4 + wave : static_cast<int>(blockIdx.x);
  if (ONE && row >= rows) return;
  const void* xr = row_at(x, f32, row * ldx);
  Chunk<F> q[MAXC];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    clear<F>(q[i]);
    const int c = t0 + stride * i;
    if (8 * c < cols) load_chunk<F>(xr, f32, c, cols, q[i]);
  }
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    float v[8];
    to_floats<F>(q[i], v);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, abs_bits(v[e]));
  }
  top = wave_max(top);
  if constexpr (!ONE) {
    if (lane == 0) part[wave] = top;
    __syncthreads();
    top = wave_max(part[lane < static_cast<int>(blockDim.x >> 6) ? lane : 0]);
  }
  const float m = __uint_as_float(top);
  const bool numbers = top < kInfBits && top != 0;
  // t = x inv is within 127 * 2^-23 of 127 x / m, where 127 / m is a number
  const float inv = numbers ? 127.f / m : 0.f;
  const float thr = inv < 3e38f ? 0.5f - 1.6e-5f : -1.f;
  uint2* cr = reinterpret_cast<uint2*>(codes + row * ldc);
  uint32_t open = 0;
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = t0 + stride * i;
    if (c < nchunk) {
      float v[8], far;
      to_floats<F>(q[i], v);
      const uint2 w = codes8(v, inv, &far);
      if (far > thr) open |= 1u << i;
      store_codes(cr + c, numbers ? w : make_uint2(0, 0));
    }
  }
  if (t0 == 0) scales[row] = top < kInfBits ? m / 127.f : __uint_as_float(0x7fc00000u);
  while (open && numbers) {
    const int c = t0 + stride * (__ffs(open) - 1);
    open &= open - 1;
    Chunk<F> again;
    clear<F>(again);
    if (8 * c < cols) load_chunk<F>(xr, f32, c, cols, again);
    float v[8];
    to_floats<F>(again, v);
    cr[c] = settled8(v, inv, thr, [&](int e) { return static_cast<double>(v[e]); }, m);
  }
}

template <int MAXC, bool ONE>
static void launch_q(hipStream_t st, const IntRows& r, int waves, int8_t* codes, int64_t ldc, float* scales, bool vec) {
  const dim3 grid(ONE ? (r.rows + 3) / 4 : r.rows), block(ONE ? 256 : 64 * waves);
#define ARDIT_Q(F)                                                                                                     \
  hipLaunchKernelGGL((int_quantize_kernel<MAXC, ONE, F>), grid, block, 0, st, r.p, r.f32, r.rows, r.cols, r.ld, codes, \
                     ldc, scales)
  if (!vec) ARDIT_Q(kAny);
  else if (r.f32) ARDIT_Q(kF32);
  else ARDIT_Q(kBf16);
#undef ARDIT_Q
}

// rows of 16-byte vectors throughout; others are loaded and stored by elements (us: 4680 bf16 rows of 13821
// quantised 132, of 13824 49; 4680 fp32 rows of 5119 normed 106, of 5120 47)
static bool vec_rows(const void* p, bool f32, int cols, int64_t ld) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && cols % 8 == 0 && ld * (f32 ? 4 : 2) % 16 == 0;
}

hipError_t launch_int_quantize(hipStream_t st, const IntRows& r, int8_t* codes, int64_t ldc, float* scales) {
  if (r.rows == 0) return hipSuccess;
  const bool vec = vec_rows(r.p, r.f32, r.cols, r.ld);
  const int n = (2 * ((r.cols + 15) / 16) + 63) / 64;   // waves' worth of chunks
  // few rows: more waves to a row, for its latency
  if (n > 3 && r.rows < 512 && n <= 48) {
    launch_q<3, false>(st, r, (n + 2) / 3, codes, ldc, scales, vec);
  } else if (n <= 10) {
    if (n <= 1) launch_q<1, true>(st, r, 1, codes, ldc, scales, vec);
    else if (n <= 2) launch_q<2, true>(st, r, 1, codes, ldc, scales, vec);
    else if (n <= 3) launch_q<3, true>(st, r, 1, codes, ldc, scales, vec);
    else if (n <= 5) launch_q<5, true>(st, r, 1, codes, ldc, scales, vec);
    else if (n <= 8) launch_q<8, true>(st, r, 1, codes, ldc, scales, vec);
    else launch_q<10, true>(st, r, 1, codes, ldc, scales, vec);
  } else if (n <= 63 && (n + 8) / 9 * 9 <= (n + 6) / 7 * 7) {
    launch_q<9, false>(st, r, (n + 8) / 9, codes, ldc, scales, vec);
  } else if (n <= 112) {
    launch_q<7, false>(st, r, (n + 6) / 7, codes, ldc, scales, vec);
  } else {
    launch_q<8, false>(st, r, (n + 7) / 8, codes, ldc, scales, vec);
  }
  return hipGetLastError();
}

// ------------------------------------------------------------------ read back
// A workgroup takes `rpg` rows; a lane four codes at a time, neighbours side by side, U of them
// under way.
template <typename T>
__global__ __launch_bounds__(256) void int_dequantize_kernel(const int8_t* __restrict__ codes, int64_t ldc,
                                                             const float* __restrict__ scales, T* __restrict__ y,
                                                             int64_t ldy, int rows, int cols, int rpg, FastDiv fq,
                                                             int vec) {
  constexpr int U = 4;
  const int row0 = blockIdx.x * rpg, quads = static_cast<int>(fq.d);
  const int items = min(rpg, rows - row0) * quads;
  for (int i0 = threadIdx.x; i0 < items; i0 += 256 * U) {
    uint32_t w[U];
    float s[U];
    int64_t at[U];
    int left[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = min(i0 + 256 * u, items - 1);
      const int r = static_cast<int>(fdiv(i, fq)), c = 4 * (i - r * quads);
      w[u] = *reinterpret_cast<const uint32_t*>(codes + (row0 + r) * ldc + c);
      s[u] = scales[row0 + r];
      at[u] = (row0 + r) * ldy + c;
      left[u] = i0 + 256 * u < items ? cols - c : 0;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = static_cast<float>(static_cast<int8_t>(w[u] >> (8 * e))) * s[u];
      T* o = y + at[u];
      if (vec) {
        if (left[u] > 0) {
          if constexpr (sizeof(T) == 4)
            __builtin_nontemporal_store(f32x4{f[0], f[1], f[2], f[3]}, reinterpret_cast<f32x4*>(o));
          else
            *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]));
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < left[u]) {
            if constexpr (sizeof(T) == 4) o[e] = f[e];
            else o[e] = f2bf(f[e]);
          }
      }
    }
  }
}

hipError_t launch_int_dequantize(hipStream_t st, const int8_t* codes, int64_t ldc, const float* scales, void* y,
                                 bool y_f32, int64_t ldy, int rows, int cols) {
  if (rows == 0) return hipSuccess;
  const int quads = (cols + 3) / 4;
  const int rpg = max(1, 2048 / quads);
  const int size = y_f32 ? 4 : 2;
  const bool vec = cols % 4 == 0 && reinterpret_cast<uintptr_t>(y) % (4 * size) == 0 && ldy % 4 == 0;
  const dim3 grid((rows + rpg - 1) / rpg);
  const FastDiv fq = make_fastdiv(quads);
  if (y_f32)
    hipLaunchKernelGGL(int_dequantize_kernel<float>, grid, dim3(256), 0, st, codes, ldc, scales,
                       static_cast<float*>(y), ldy, rows, cols, rpg, fq, vec);
  else
    hipLaunchKernelGGL(int_dequantize_kernel<bf16_t>, grid, dim3(256), 0, st, codes, ldc, scales,
                       static_cast<bf16_t*>(y), ldy, rows, cols, rpg, fq, vec);
  return hipGetLastError();
}

// ----------------------------------------------------------------------- norm
constexpr int kNormRows = 8;   // rows of a workgroup, one a wave

// A workgroup's rows belong to one stream, whose vectors (gate, shift, scale or gain) are staged in
// LDS as fp32 with the halves of every chunk apart, so that a wave's 16-byte reads are
// consecutive.  The mean square is summed in fp64, and the fp32 estimate of
// y = p + shift, p = (h rs) (1 + scale), is within 2^-24 (3 max|p| + max|y|) of the truth, and where
// h rs is subnormal 2^-150 |1 + scale| more, below 2^-129 for scales up to 2^20: that bound says which
// elements may be the largest and which codes are open, and those are computed again in fp64.  With
// larger vectors, or rs below fp32's normal numbers, all are.
// XF, DK: type of x (kBf16, kF32, kAny) and of delta (the same; -1: none).
// (Up to 128 registers two workgroups share a CU; long rows with a branch to add need more, and up to
// 5120 elements run without spills: 9360 rows of 5120 149 us (3.5 TB/s), with spills 18 more.  Its eight waves a CU
// load, sum and store in turn; going from row to row in a loop, with the next row requested ahead or not, spills
// and takes 187 to 195.  Four rows a workgroup take as long, sixteen 20 to 30% longer.  Above 5120 elements
// an fp32 x with an fp32 branch, and rows loaded by elements, spill 55 to 58 registers: 9360 rows of 8192 304 us
// (2.8 TB/s), with the branch in bf16, which spills none, 260 (3.2).)
template <int MAXC, int XF, int DK>
__global__ __launch_bounds__(64 * kNormRows, MAXC > 10 || (MAXC >= 8 && DK >= 0) ? 2 : 4) void int_norm_kernel(const IntNormArgs p) {
  constexpr bool VEC = XF != kAny;
  extern __shared__ float4 lds_vec[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int b = static_cast<int>(fdiv(blockIdx.x, p.groups));
  const int64_t in = static_cast<int64_t>(blockIdx.x - b * p.groups.d) * kNormRows + wave;   // row of the stream
  const int64_t row = b * p.rows_per_stream + in;
  const bool live = in < p.rows_per_stream && row < p.rows;
  const int64_t rd = live ? row : p.rows - 1;
  const int D = p.D, n8 = (D + 7) / 8, nchunk = 2 * ((D + 15) / 16);
  const bool x_f32 = VEC ? XF == kF32 : p.x_f32;
  constexpr int DF = DK < 0 ? static_cast<int>(kBf16) : DK;
  const bool has_d = DK == kAny ? p.dk != 0 : DK >= 0;
  const bool d_f32 = VEC ? DK == kF32 : p.dk == 2;
  const bool has_b = p.shift_row >= 0, has_g = p.gate_row >= 0, gain = p.gain != nullptr, has_a = gain || p.a_row >= 0;
  const void* xr = row_at(p.x, x_f32, rd * p.ldx);
  const void* dr = has_d ? row_at(p.delta, d_f32, rd * p.ldd) : nullptr;

  Chunk<XF> xq[MAXC];
  Chunk<DF> dq[MAXC];
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = lane + 64 * i;
    clear<XF>(xq[i]);
    clear<DF>(dq[i]);
    if (c < n8) {
      load_chunk<XF>(xr, x_f32, c, D, xq[i]);
      if (has_d) load_chunk<DF>(dr, d_f32, c, D, dq[i]);
    }
  }
  // vectors, as many as there are
  float4* lds_a = lds_vec;
  float4* lds_b = lds_a + (has_a ? 2 * n8 : 0);
  float4* lds_g = lds_b + (has_b ? 2 * n8 : 0);
  uint32_t widest = 0;   // bits of the vectors' largest magnitude: an infinity or a NaN is then in every row
  auto stage = [&](float4* to, int r) __attribute__((always_inline)) {
    const float* m = p.mod + (static_cast<int64_t>(b) * 6 + r) * D;
    const float* t = p.table ? p.table + static_cast<int64_t>(r) * D : nullptr;
    for (int k = threadIdx.x; k < 2 * n8; k += 64 * kNormRows) {   // four elements
      float f[4];
      if (VEC && p.vec_mod) {
        const float4 a = reinterpret_cast<const float4*>(m)[k];
        const float4 c = t ? reinterpret_cast<const float4*>(t)[k] : make_float4(0.f, 0.f, 0.f, 0.f);
        f[0] = a.x + c.x; f[1] = a.y + c.y; f[2] = a.z + c.z; f[3] = a.w + c.w;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = 4 * k + e < D ? (t ? m[4 * k + e] + t[4 * k + e] : m[4 * k + e]) : 0.f;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) widest = max(widest, abs_bits(f[e]));
      to[(k & 1) * n8 + (k >> 1)] = make_float4(f[0], f[1], f[2], f[3]);
    }
  };
  if (gain) {
    for (int k = threadIdx.x; k < 2 * n8; k += 64 * kNormRows) {
      float f[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = 4 * k + e < D ? bf2f(p.gain[4 * k + e]) : 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) widest = max(widest, abs_bits(f[e]));
      lds_a[(k & 1) * n8 + (k >> 1)] = make_float4(f[0], f[1], f[2], f[3]);
    }
  } else if (has_a) {
    stage(lds_a, p.a_row);
  }
  if (has_b) stage(lds_b, p.shift_row);
  if (has_g) stage(lds_g, p.gate_row);
  const bool wide = __syncthreads_or(widest >= kWideBits);
  const bool spoilt = wide && __syncthreads_or(widest >= kInfBits);
  if (!live) return;
  auto vec8 = [&](const float4* v, int c, float* f) __attribute__((always_inline)) {
    const float4 lo = v[c], hi = v[n8 + c];
    f[0] = lo.x; f[1] = lo.y; f[2] = lo.z; f[3] = lo.w;
    f[4] = hi.x; f[5] = hi.y; f[6] = hi.z; f[7] = hi.w;
  };
  // h of a chunk from what memory holds
  auto sum8 = [&](const Chunk<XF>& x, const Chunk<DF>& d, int c, float* h) __attribute__((always_inline)) {
    to_floats<XF>(x, h);
    if (has_d) {
      float f[8], g[8];
      to_floats<DF>(d, f);
      if (has_g) vec8(lds_g, c, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = has_g ? fmaf(g[e], f[e], h[e]) : h[e] + f[e];
    }
  };

  float v[MAXC][8];
  double ss = 0.0;
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = lane + 64 * i;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
    if (c < n8) {
      sum8(xq[i], dq[i], c, v[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double z = v[i][e];
        ss = fma(z, z, ss);
      }
      if (p.h) {
        float* hr = p.h + row * p.ldh + 8 * c;
        if (VEC) {
          f32x4* ho = reinterpret_cast<f32x4*>(hr);
          __builtin_nontemporal_store(f32x4{v[i][0], v[i][1], v[i][2], v[i][3]}, ho);
          __builtin_nontemporal_store(f32x4{v[i][4], v[i][5], v[i][6], v[i][7]}, ho + 1);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (8 * c + e < D) hr[e] = v[i][e];
        }
      }
    }
  }
  ss = wave_join(ss, [](double a, double c) { return a + c; });
  const double rs = 1.0 / sqrt(ss / D + p.eps);
  const float rs32 = static_cast<float>(rs);

  // y of a chunk of h in fp32, and the largest |p|
  auto form = [&](const float* h, int c, float* y, float* pm) __attribute__((always_inline)) {
    float a[8], s[8];
    if (has_a) vec8(lds_a, c, a);
    if (has_b) vec8(lds_b, c, s);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float u = h[e] * rs32;
      y[e] = gain ? u * a[e] : has_a ? fmaf(u, a[e], u) : u;
    }
    if (has_b) {
      if (pm)
#pragma unroll
        for (int e = 0; e < 8; e += 2) *pm = max_abs(*pm, y[e], y[e + 1]);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] += s[e];
    }
  };
  // and in fp64; without scale and shift in units of 1 / rms, which the codes do not depend on:
  // h gain is exact, and so are its halves of the largest
  const bool in_units = !has_b && (gain || !has_a);
  auto exact = [&](float h, int c, int e) __attribute__((always_inline)) {
    const int at = (e >> 2) * 4 * n8 + 4 * c + (e & 3);
    const double a = has_a ? reinterpret_cast<const float*>(lds_a)[at] : 0.f;
    double y = h;
    if (!in_units) y *= rs;
    if (has_a) y *= gain ? a : 1.0 + a;
    if (has_b) y += static_cast<double>(reinterpret_cast<const float*>(lds_b)[at]);
    return y;
  };
  // this lane's largest chunk, and the largest of its others
  float most = 0.f, next = 0.f, pm = 0.f;
  int at = 0;
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = lane + 64 * i;
    if (c < n8) {
      float y[8], cm = 0.f;
      form(v[i], c, y, &pm);
#pragma unroll
      for (int e = 0; e < 8; e += 2) cm = max_abs(cm, y[e], y[e + 1]);
      next = fmaxf(next, fminf(cm, most));
      if (cm > most) most = cm, at = i;
    }
  }
  // (maxima of non-negative numbers as those of their bits; a NaN in h shows in the sum)
  const float ym = __uint_as_float(wave_max(__float_as_uint(most)));
  pm = has_b ? __uint_as_float(wave_max(__float_as_uint(pm))) : ym;
  const bool known = !wide && rs32 > 3e-38f;   // else nothing is known of y
  const float err = 5.97e-8f * (3.25f * pm + 1.25f * ym) + 3e-39f;
  // (p of known rows stays far below fp32's end, so y passes it where its estimate does)
  bool finite = !spoilt && (!known || ym <= 3.4028235e38f) && ss <= 1.7e308;

  // the largest magnitude, from the chunks that may hold it
  double m = 0.0;
  if (finite && (ym != 0.f || ss != 0.0)) {   // (y is 0 throughout where both are)
    const float low = known ? ym - 2.f * err : -1.f;
    if (most >= low) {
#pragma unroll
      for (int i = 0; i < MAXC; ++i) {
        const int c = lane + 64 * i;
        if (c < n8 && (i == at || next >= low))
#pragma unroll
          for (int e = 0; e < 8; ++e) m = fmax(m, fabs(exact(v[i][e], c, e)));
      }
    }
    m = wave_join(m, [](double a, double c) { return fmax(a, c); });
    finite = known || static_cast<float>(in_units ? m * rs : m) <= 3.4028235e38f;
  }
  const bool numbers = finite && m > 0.0;
  const float inv = numbers ? 127.f / ym : 0.f;
  const float thr = known && inv < 3e38f ? 0.5f - 1.1f * (2.f * err * inv + 1.6e-5f) : -1.f;
  uint2* cr = reinterpret_cast<uint2*>(p.codes + row * p.ldc);
  uint32_t open = 0;
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = lane + 64 * i;
    if (c < nchunk) {
      uint2 w = make_uint2(0, 0);
      if (numbers && c < n8) {
        float y[8], far;
        form(v[i], c, y, nullptr);
        w = codes8(y, inv, &far);
        if (far > thr) open |= 1u << i;
      }
      store_codes(cr + c, w);
    }
  }
  if (lane == 0) p.scales[row] = finite ? static_cast<float>((in_units ? m * rs : m) / 127.0) : __uint_as_float(0x7fc00000u);
  while (open) {
    const int c = lane + 64 * (__ffs(open) - 1);
    open &= open - 1;
    float h[8];
    if (p.h) {          // (x or delta may be under it)
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = 8 * c + e < D ? p.h[row * p.ldh + 8 * c + e] : 0.f;
    } else {
      Chunk<XF> x;
      Chunk<DF> d;
      load_chunk<XF>(xr, x_f32, c, D, x);
      if (has_d) load_chunk<DF>(dr, d_f32, c, D, d);
      sum8(x, d, c, h);
    }
    float y[8];
    form(h, c, y, nullptr);
    cr[c] = settled8(y, inv, thr, [&](int e) { return exact(h[e], c, e); }, m);
  }
}

template <int MAXC>
static void launch_norm_t(hipStream_t st, const IntNormArgs& a, int grid, size_t lds, bool vec) {
#define ARDIT_NORM(XF, DK) \
  hipLaunchKernelGGL((int_norm_kernel<MAXC, XF, DK>), dim3(grid), dim3(64 * kNormRows), lds, st, a)
  if (!vec) {
    ARDIT_NORM(kAny, kAny);
  } else if (a.x_f32) {
    if (a.dk == 0) ARDIT_NORM(kF32, -1);
    else if (a.dk == 1) ARDIT_NORM(kF32, kBf16);
    else ARDIT_NORM(kF32, kF32);
  } else {
    if (a.dk == 0) ARDIT_NORM(kBf16, -1);
    else if (a.dk == 1) ARDIT_NORM(kBf16, kBf16);
    else ARDIT_NORM(kBf16, kF32);
  }
#undef ARDIT_NORM
}

hipError_t launch_int_norm(hipStream_t st, IntNormArgs a) {
  if (a.rows == 0) return hipSuccess;
  const int64_t per = std::min<int64_t>(a.rows_per_stream, a.rows);
  a.rows_per_stream = per;
  const int64_t streams = (a.rows + per - 1) / per, groups = (per + kNormRows - 1) / kNormRows;
  a.groups = make_fastdiv(static_cast<uint32_t>(groups));
  const int vectors = (a.a_row >= 0 || a.gain) + (a.shift_row >= 0) + (a.gate_row >= 0);
  const size_t lds = static_cast<size_t>(vectors) * ((a.D + 7) / 8) * 32;
  const int grid = static_cast<int>(streams * groups);
  const bool vec = vec_rows(a.x, a.x_f32, a.D, a.ldx) && (!a.dk || vec_rows(a.delta, a.dk == 2, a.D, a.ldd)) &&
                   (!a.h || vec_rows(a.h, true, a.D, a.ldh));
  a.vec_mod = vec_rows(a.mod, true, a.D, 8) && vec_rows(a.table, true, a.D, 8);
  const int n = (2 * ((a.D + 15) / 16) + 63) / 64;   // waves' worth of chunks
  if (n <= 1) launch_norm_t<1>(st, a, grid, lds, vec);
  else if (n <= 2) launch_norm_t<2>(st, a, grid, lds, vec);
  else if (n <= 3) launch_norm_t<3>(st, a, grid, lds, vec);
  else if (n <= 5) launch_norm_t<5>(st, a, grid, lds, vec);
  else if (n <= 8) launch_norm_t<8>(st, a, grid, lds, vec);
  else if (n <= 10) launch_norm_t<10>(st, a, grid, lds, vec);
  else launch_norm_t<16>(st, a, grid, lds, vec);
  return hipGetLastError();
}

}  // namespace ardit
