// Rows to 8-bit integer codes and back, and the norm that feeds a linear layer over them.
//
// A row y with m = max|y| takes the scale m / 127 and the codes rint(127 y / m), decided exactly:
// the fp32 estimate t = y (127 / m) is off by a bound that the kernel knows, so only elements
// whose t lies that near to a half (a few in 10^5) are decided again in fp64, by the sign of
// 254 |y| - (2 k + 1) m.  Chunks of 8 elements that hold one are marked, and rewritten by one
// loop at the end that reads its elements again.
//
// All are bound by HBM (quantising reads 2 or 4 bytes an element and writes 1): a row is held in
// registers by one wave, or by the waves of a workgroup where it is wide, so it is read once and
// all its loads are under way together.
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

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), s, kWave)));
  return v;
}
__device__ __forceinline__ double wave_max(double v) {
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) v = fmax(v, __shfl_xor(v, s, kWave));
  return v;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) v += __shfl_xor(v, s, kWave);
  return v;
}

__device__ __forceinline__ float load_elem(const void* p, bool f32, size_t at) {
  return f32 ? static_cast<const float*>(p)[at] : bf2f(static_cast<const bf16_t*>(p)[at]);
}

// Elements 8 c .. 8 c + 7 of a row of D, zero past its end.  VEC: the row starts on 16 bytes and
// D is a multiple of 8.
template <bool VEC>
__device__ __forceinline__ void load_chunk(const void* row, bool f32, int c, int D, float* f) {
  if constexpr (VEC) {
    if (f32) {
      const float4* p = static_cast<const float4*>(row) + 2 * c;
      const float4 a = p[0], b = p[1];
      f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
      f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    } else {
      unpack8(static_cast<const uint4*>(row)[c], f);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = 8 * c + e < D ? load_elem(row, f32, 8 * c + e) : 0.f;
  }
}

__device__ __forceinline__ const void* row_at(const void* p, bool f32, int64_t elem) {
  return static_cast<const char*>(p) + elem * (f32 ? 4 : 2);
}

// Codes of eight estimates t = y inv; true when one lies further than thr from its whole number
// (or is no number): its code is not decided.
__device__ __forceinline__ bool codes8(const float* y, float inv, float thr, uint2* out) {
  uint32_t w[8];
  bool open = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float t = y[e] * inv;
    const float r = t + kMagic;
    open |= !(fabsf(t - (r - kMagic)) <= thr);
    w[e] = __float_as_uint(r);
  }
  *out = make_uint2(pack_bytes(w[0], w[1], w[2], w[3]), pack_bytes(w[4], w[5], w[6], w[7]));
  return open;
}

// The code of y in a row whose largest magnitude is m > 0.
__device__ __forceinline__ int exact_code(double y, double m) {
#pragma clang fp contract(off)   // (both products of `side` rounded alike, so that halves of m tie)
  const double a = fabs(y);
  double k = floor(127.0 * (a / m));   // (or one off: the border decides)
  const double side = 254.0 * a - (2.0 * k + 1.0) * m;
  if (side > 0.0 || (side == 0.0 && (static_cast<int>(k) & 1))) k += 1.0;
  const int q = static_cast<int>(k);
  return y < 0.0 ? -q : q;
}

constexpr uint32_t kInfBits = 0x7f800000u;

}  // namespace

// ------------------------------------------------------------------- quantise
// WPR waves hold a row of up to 512 MAXC WPR elements; a workgroup has four waves, or WPR.
template <int MAXC, int WPR, bool VEC>
__global__ __launch_bounds__(WPR < 4 ? 256 : 64 * WPR) void int_quantize_kernel(
    const void* x, int x_f32, int rows, int cols, int64_t ldx, int8_t* codes, int64_t ldc, float* scales) {
  constexpr int NW = WPR < 4 ? 4 : WPR, RPG = NW / WPR;
  __shared__ uint32_t part[NW];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = blockIdx.x * RPG + wave / WPR;
  const int t0 = (wave % WPR) * 64 + lane;            // this lane's place among the row's
  const int nchunk = 2 * ((cols + 15) / 16);          // (whole 16 bytes of codes)
  const bool live = row < rows;
  const void* xr = row_at(x, x_f32, static_cast<int64_t>(min(row, rows - 1)) * ldx);
  float v[MAXC][8];
  uint32_t top = 0;
  auto load_all = [&](bool f32) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
      const int c = t0 + 64 * WPR * i;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
      if (8 * c < cols) load_chunk<VEC>(xr, f32, c, cols, v[i]);
    }
  };
  if (x_f32) load_all(true);
  else load_all(false);
#pragma unroll
  for (int i = 0; i < MAXC; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, abs_bits(v[i][e]));
  top = wave_max(top);
  if constexpr (WPR > 1) {
    if (lane == 0) part[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WPR; ++w) top = max(top, part[wave / WPR * WPR + w]);
  }
  if (!live) return;
  const float m = __uint_as_float(top);
  const bool numbers = top < kInfBits && top != 0;
  // t = x inv is within 127 * 2^-23 of 127 x / m, where 127 / m is a number
  const float inv = numbers ? 127.f / m : 0.f;
  const float thr = 0.5f - 1.6e-5f;
  uint2* cr = reinterpret_cast<uint2*>(codes + static_cast<int64_t>(row) * ldc);
  uint32_t open = 0;
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = t0 + 64 * WPR * i;
    if (c < nchunk) {
      uint2 q = make_uint2(0, 0);
      if (numbers && codes8(v[i], inv, thr, &q)) open |= 1u << i;
      cr[c] = q;
    }
  }
  if (t0 == 0) scales[row] = top < kInfBits ? m / 127.f : __uint_as_float(0x7fc00000u);
  while (open) {
    const int c = t0 + 64 * WPR * (__ffs(open) - 1);
    open &= open - 1;
    for (int j = 8 * c; j < min(8 * c + 8, cols); ++j)
      codes[static_cast<int64_t>(row) * ldc + j] = static_cast<int8_t>(exact_code(load_elem(xr, x_f32, j), m));
  }
}

template <int MAXC, int WPR>
static void launch_q(hipStream_t st, const IntRows& r, int8_t* codes, int64_t ldc, float* scales, bool vec) {
  constexpr int NW = WPR < 4 ? 4 : WPR, RPG = NW / WPR;
  const dim3 grid((r.rows + RPG - 1) / RPG), block(64 * NW);
  if (vec)
    hipLaunchKernelGGL((int_quantize_kernel<MAXC, WPR, true>), grid, block, 0, st, r.p, r.f32, r.rows, r.cols, r.ld,
                       codes, ldc, scales);
  else
    hipLaunchKernelGGL((int_quantize_kernel<MAXC, WPR, false>), grid, block, 0, st, r.p, r.f32, r.rows, r.cols, r.ld,
                       codes, ldc, scales);
}

// rows of 16-byte vectors throughout
static bool vec_rows(const void* p, bool f32, int cols, int64_t ld) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && cols % 8 == 0 && ld * (f32 ? 4 : 2) % 16 == 0;
}

hipError_t launch_int_quantize(hipStream_t st, const IntRows& r, int8_t* codes, int64_t ldc, float* scales) {
  if (r.rows == 0) return hipSuccess;
  const bool vec = vec_rows(r.p, r.f32, r.cols, r.ld);
  const int n = (2 * ((r.cols + 15) / 16) + 63) / 64;   // waves' worth of chunks
  if (n <= 1) launch_q<1, 1>(st, r, codes, ldc, scales, vec);
  else if (n <= 2) launch_q<2, 1>(st, r, codes, ldc, scales, vec);
  else if (n <= 4) launch_q<4, 1>(st, r, codes, ldc, scales, vec);
  else if (n <= 8) launch_q<2, 4>(st, r, codes, ldc, scales, vec);
  else if (n <= 16) launch_q<4, 4>(st, r, codes, ldc, scales, vec);
  else if (n <= 32) launch_q<4, 8>(st, r, codes, ldc, scales, vec);
  else launch_q<8, 16>(st, r, codes, ldc, scales, vec);
  return hipGetLastError();
}

// ------------------------------------------------------------------ read back
// A workgroup takes `rpg` rows; a lane four codes at a time, neighbours side by side.
template <typename T>
__global__ __launch_bounds__(256) void int_dequantize_kernel(const int8_t* __restrict__ codes, int64_t ldc,
                                                             const float* __restrict__ scales, T* __restrict__ y,
                                                             int64_t ldy, int rows, int cols, int rpg, FastDiv fq,
                                                             int vec) {
  const int row0 = blockIdx.x * rpg;
  const int items = min(rpg, rows - row0) * static_cast<int>(fq.d);
  for (int i = threadIdx.x; i < items; i += 256) {
    const int r = static_cast<int>(fdiv(i, fq)), c = 4 * (i - r * static_cast<int>(fq.d));
    const int64_t row = row0 + r;
    const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + row * ldc + c);
    const float s = scales[row];
    float f[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = static_cast<float>(static_cast<int8_t>(w >> (8 * e))) * s;
    T* o = y + row * ldy + c;
    if (vec) {
      if constexpr (sizeof(T) == 4)
        *reinterpret_cast<float4*>(o) = make_float4(f[0], f[1], f[2], f[3]);
      else
        *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < cols) {
          if constexpr (sizeof(T) == 4) o[e] = f[e];
          else o[e] = f2bf(f[e]);
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

// A workgroup's rows belong to one stream, whose vectors (scale or gain, shift, gate) are staged
// in LDS as fp32 with the halves of every chunk apart, so that a wave's 16-byte reads are
// consecutive.  The mean square is summed in fp64, and the fp32 estimate of
// y = p + shift, p = (h rs) (1 + scale), is within 2^-24 (3 max|p| + max|y|) of the truth: that
// bound says which elements may be the largest and which codes are open, and those are computed
// again in fp64.
// XF, DK: type of x (0 bf16, 1 fp32) and of delta (0 none, 1 bf16, 2 fp32); VEC false: as
// IntNormArgs says.
template <int MAXC, int XF, int DK, bool VEC>
__global__ __launch_bounds__(64 * kNormRows) void int_norm_kernel(const IntNormArgs p) {
  extern __shared__ float4 lds_vec[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int b = static_cast<int>(fdiv(blockIdx.x, p.groups));
  const int64_t in = static_cast<int64_t>(blockIdx.x - b * p.groups.d) * kNormRows + wave;   // row of the stream
  const int64_t row = b * p.rows_per_stream + in;
  const bool live = in < p.rows_per_stream && row < p.rows;
  const int64_t rd = live ? row : p.rows - 1;
  const int D = p.D, n8 = (D + 7) / 8, nchunk = 2 * ((D + 15) / 16);
  const bool x_f32 = VEC ? XF == 1 : p.x_f32;
  const int dk = VEC ? DK : p.dk;
  const void* xr = row_at(p.x, x_f32, rd * p.ldx);
  const void* dr = dk ? row_at(p.delta, dk == 2, rd * p.ldd) : nullptr;

  float h[MAXC][8], d[MAXC][8];
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = lane + 64 * i;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[i][e] = d[i][e] = 0.f;
    if (c < n8) {
      load_chunk<VEC>(xr, x_f32, c, D, h[i]);
      if (dk) load_chunk<VEC>(dr, dk == 2, c, D, d[i]);
    }
  }
  // vectors: a (gain or scale), then shift, then gate, as many as there are
  float4* lds_a = lds_vec;
  float4* lds_b = lds_a + (p.a_row >= 0 || p.gain ? 2 * n8 : 0);
  float4* lds_g = lds_b + (p.shift_row >= 0 ? 2 * n8 : 0);
  auto stage = [&](float4* to, int r) {
    const float* m = p.mod + (static_cast<int64_t>(b) * 6 + r) * D;
    const float* t = p.table ? p.table + static_cast<int64_t>(r) * D : nullptr;
    float* f = reinterpret_cast<float*>(to);
    for (int j = threadIdx.x; j < 8 * n8; j += 64 * kNormRows) {
      const float z = j < D ? (t ? m[j] + t[j] : m[j]) : 0.f;
      f[(j & 4) * n8 + 4 * (j >> 3) + (j & 3)] = z;
    }
  };
  if (p.gain) {
    float* f = reinterpret_cast<float*>(lds_a);
    for (int j = threadIdx.x; j < 8 * n8; j += 64 * kNormRows)
      f[(j & 4) * n8 + 4 * (j >> 3) + (j & 3)] = j < D ? bf2f(p.gain[j]) : 0.f;
  } else if (p.a_row >= 0) {
    stage(lds_a, p.a_row);
  }
  if (p.shift_row >= 0) stage(lds_b, p.shift_row);
  if (p.gate_row >= 0) stage(lds_g, p.gate_row);
  __syncthreads();
  if (!live) return;
  const bool has_a = p.a_row >= 0 || p.gain, has_b = p.shift_row >= 0, has_g = p.gate_row >= 0;
  const float base = p.gain ? 0.f : 1.f;   // p = u a + u base
  auto vec8 = [&](const float4* v, int c, float* f) __attribute__((always_inline)) {
    const float4 lo = v[c], hi = v[n8 + c];
    f[0] = lo.x; f[1] = lo.y; f[2] = lo.z; f[3] = lo.w;
    f[4] = hi.x; f[5] = hi.y; f[6] = hi.z; f[7] = hi.w;
  };

  double ss = 0.0;
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = lane + 64 * i;
    if (c < n8) {
      if (dk) {
        float g[8];
        if (has_g) vec8(lds_g, c, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[i][e] = has_g ? fmaf(g[e], d[i][e], h[i][e]) : h[i][e] + d[i][e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double z = h[i][e];
        ss = fma(z, z, ss);
      }
      if (p.h) {
        float* hr = p.h + row * p.ldh + 8 * c;
        if (VEC) {
          reinterpret_cast<float4*>(hr)[0] = make_float4(h[i][0], h[i][1], h[i][2], h[i][3]);
          reinterpret_cast<float4*>(hr)[1] = make_float4(h[i][4], h[i][5], h[i][6], h[i][7]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (8 * c + e < D) hr[e] = h[i][e];
        }
      }
    }
  }
  const double rs = 1.0 / sqrt(wave_sum(ss) / D + p.eps);
  const float rs32 = static_cast<float>(rs);

  // y of chunk i in fp32; pm takes the largest |p|
  auto form = [&](int i, float* y, float* pm) __attribute__((always_inline)) {
    const int c = lane + 64 * i;
    float a[8], s[8];
    if (has_a) vec8(lds_a, c, a);
    if (has_b) vec8(lds_b, c, s);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float u = h[i][e] * rs32;
      const float q = has_a ? fmaf(u, a[e], u * base) : u;
      if (pm) *pm = fmaxf(*pm, fabsf(q));
      y[e] = has_b ? q + s[e] : q;
    }
  };
  uint32_t top = 0;
  float pm = 0.f;
#pragma unroll
  for (int i = 0; i < MAXC; ++i)
    if (lane + 64 * i < n8) {
      float y[8];
      form(i, y, &pm);
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, abs_bits(y[e]));
    }
  top = wave_max(top);
  pm = __uint_as_float(wave_max(__float_as_uint(pm)));
  const float ym = __uint_as_float(top);
  // error of y; of a subnormal 1 / rms nothing is known
  float err = 5.97e-8f * (3.25f * pm + 1.25f * ym) + 1e-44f;
  if (!(rs32 > 3e-38f)) err = ym + 1.f;
  const bool finite = top < kInfBits;
  // (where ym is 0 the largest |y| is below 2^-149, and its scale rounds to 0)

  // element j of the row again, in fp64; without scale and shift in units of 1 / rms, which the
  // codes do not depend on: h gain is exact, and so are its halves of the largest
  const bool in_units = !has_b && p.a_row < 0;
  auto again = [&](int j) -> double {
    float z;
    if (p.h) {
      z = p.h[row * p.ldh + j];
    } else {
      z = load_elem(xr, x_f32, j);
      const int at = (j & 4) * n8 + 4 * (j >> 3) + (j & 3);
      if (dk) {
        const float dd = load_elem(dr, dk == 2, j);
        z = has_g ? fmaf(reinterpret_cast<const float*>(lds_g)[at], dd, z) : z + dd;
      }
    }
    const int at = (j & 4) * n8 + 4 * (j >> 3) + (j & 3);
    double y = in_units ? static_cast<double>(z) : static_cast<double>(z) * rs;
    if (has_a) {
      const double a = reinterpret_cast<const float*>(lds_a)[at];
      y *= p.gain ? a : 1.0 + a;
    }
    if (has_b) y += static_cast<double>(reinterpret_cast<const float*>(lds_b)[at]);
    return y;
  };
  // the largest magnitude: chunks that may hold it
  double m = 0.0;
  if (finite && top != 0) {
    uint32_t near = 0;
    const float low = ym - 2.f * err;
#pragma unroll
    for (int i = 0; i < MAXC; ++i)
      if (lane + 64 * i < n8) {
        float y[8];
        form(i, y, nullptr);
        bool any = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) any |= fabsf(y[e]) >= low;
        if (any) near |= 1u << i;
      }
    while (near) {
      const int c = lane + 64 * (__ffs(near) - 1);
      near &= near - 1;
      for (int j = 8 * c; j < min(8 * c + 8, D); ++j) m = fmax(m, fabs(again(j)));
    }
    m = wave_max(m);
  }
  const bool numbers = finite && m > 0.0;
  const float inv = numbers ? 127.f / ym : 0.f;
  const float thr = 0.5f - 1.1f * (2.f * err * inv + 1.6e-5f);
  uint2* cr = reinterpret_cast<uint2*>(p.codes + row * p.ldc);
  uint32_t open = 0;
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = lane + 64 * i;
    if (c < nchunk) {
      uint2 q = make_uint2(0, 0);
      if (numbers && c < n8) {
        float y[8];
        form(i, y, nullptr);
        if (codes8(y, inv, thr, &q)) open |= 1u << i;
      }
      cr[c] = q;
    }
  }
  if (lane == 0) p.scales[row] = finite ? static_cast<float>((in_units ? m * rs : m) / 127.0) : __uint_as_float(0x7fc00000u);
  while (open) {
    const int c = lane + 64 * (__ffs(open) - 1);
    open &= open - 1;
    for (int j = 8 * c; j < min(8 * c + 8, D); ++j)
      p.codes[row * p.ldc + j] = static_cast<int8_t>(exact_code(again(j), m));
  }
}

template <int MAXC, bool VEC>
static void launch_norm_t(hipStream_t st, const IntNormArgs& a, int grid, size_t lds) {
#define ARDIT_NORM(XF, DK) \
  hipLaunchKernelGGL((int_norm_kernel<MAXC, XF, DK, VEC>), dim3(grid), dim3(64 * kNormRows), lds, st, a)
  if constexpr (!VEC) {
    ARDIT_NORM(0, 0);
  } else if (a.x_f32) {
    if (a.dk == 0) ARDIT_NORM(1, 0);
    else if (a.dk == 1) ARDIT_NORM(1, 1);
    else ARDIT_NORM(1, 2);
  } else {
    if (a.dk == 0) ARDIT_NORM(0, 0);
    else if (a.dk == 1) ARDIT_NORM(0, 1);
    else ARDIT_NORM(0, 2);
  }
#undef ARDIT_NORM
}

hipError_t launch_int_norm(hipStream_t st, IntNormArgs a) {
  if (a.rows == 0) return hipSuccess;
  const int64_t per = a.rows_per_stream < a.rows ? a.rows_per_stream : a.rows;
  a.rows_per_stream = per;
  const int64_t streams = (a.rows + per - 1) / per, groups = (per + kNormRows - 1) / kNormRows;
  a.groups = make_fastdiv(static_cast<uint32_t>(groups));
  const int vectors = (a.a_row >= 0 || a.gain) + (a.shift_row >= 0) + (a.gate_row >= 0);
  const size_t lds = static_cast<size_t>(vectors) * ((a.D + 7) / 8) * 32;
  const int grid = static_cast<int>(streams * groups);
  const bool vec = vec_rows(a.x, a.x_f32, a.D, a.ldx) && (!a.dk || vec_rows(a.delta, a.dk == 2, a.D, a.ldd)) &&
                   (!a.h || vec_rows(a.h, true, a.D, a.ldh));
  const int n = (2 * ((a.D + 15) / 16) + 63) / 64;
#define ARDIT_NORM_C(C)                                  \
  if (n <= C) {                                          \
    if (vec) launch_norm_t<C, true>(st, a, grid, lds);   \
    else launch_norm_t<C, false>(st, a, grid, lds);      \
    return hipGetLastError();                            \
  }
  ARDIT_NORM_C(1)
  ARDIT_NORM_C(3)
  ARDIT_NORM_C(6)
  ARDIT_NORM_C(10)
  ARDIT_NORM_C(16)
#undef ARDIT_NORM_C
  return hipErrorInvalidValue;
}

}  // namespace ardit
