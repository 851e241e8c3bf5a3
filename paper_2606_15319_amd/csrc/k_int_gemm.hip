// Linear layers over 8-bit integer codes: y = epilogue(sx_i sw_j sum_k X_ik W_jk).
//
// X [M][K] and W [N][K] are both K-contiguous.  v_mfma_i32_16x16x64_i8 sums exactly in 32 bits
// (|sum| <= 2^30 at K = 65536), at twice the bf16 rate per operand byte.  The MFMA computes
// C^T = W X^T: W rows feed the A operand and X rows the B operand, so a lane ends with one row i
// and four consecutive columns j of every 16 x 16 block.
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

__device__ __forceinline__ float gate_at(const IntGemmArgs& p, int row, int n) {
  const size_t at = (static_cast<size_t>(fdiv(row, p.rows_per_stream)) * 6 + p.gate_row) * p.N + n;
  const float g = p.mod[at];
  return p.table ? g + p.table[static_cast<size_t>(p.gate_row) * p.N + n] : g;
}

// A wave takes 32 rows and 64 columns, its fragments straight from memory.
template <int EPI, typename ResT, typename OutT>
__global__ __launch_bounds__(256) void int_gemm_simple(const IntGemmArgs p, uint32_t tiles_m) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int l16 = lane & 15, g = lane >> 4;
  const uint32_t tile = blockIdx.x * 4 + wave;   // (below 2^31: M / 32 * N / 64)
  const int m0 = tile % tiles_m * 32, n0 = tile / tiles_m * 64;
  if (n0 >= p.N) return;
  const int8_t* xr[2];
  const int8_t* wr[4];
#pragma unroll
  for (int a = 0; a < 2; ++a) xr[a] = p.x + static_cast<int64_t>(min(m0 + 16 * a + l16, p.M - 1)) * p.ldx;
#pragma unroll
  for (int b = 0; b < 4; ++b) wr[b] = p.w + static_cast<int64_t>(min(n0 + 16 * b + l16, p.N - 1)) * p.ldw;
  i32x4 acc[2][4];
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < 4; ++b) acc[a][b] = i32x4{0, 0, 0, 0};
  for (int k = 16 * g; k - 16 * g < p.K; k += 64) {
    i32x4 fx[2], fw[4];
    const bool in = k < p.K;   // (rows go on to the next multiple of 16)
#pragma unroll
    for (int a = 0; a < 2; ++a) fx[a] = in ? *reinterpret_cast<const i32x4*>(xr[a] + k) : i32x4{0, 0, 0, 0};
#pragma unroll
    for (int b = 0; b < 4; ++b) fw[b] = in ? *reinterpret_cast<const i32x4*>(wr[b] + k) : i32x4{0, 0, 0, 0};
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int b = 0; b < 4; ++b) acc[a][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[b], fx[a], acc[a][b], 0, 0, 0);
  }
#pragma unroll
  for (int a = 0; a < 2; ++a) {
    const int m = m0 + 16 * a + l16;
    if (m >= p.M) continue;
    const Scale sx = split_scale(p.sx[m]);
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int n = n0 + 16 * b + 4 * g + e;
        if (n >= p.N) continue;
        float res = 0.f, gate = 0.f;
        if (EPI == kEpiBiasRes || EPI == kEpiBiasGateRes)
          res = as_float(static_cast<const ResT*>(p.res)[m * p.ldr + n]);
        if (EPI == kEpiBiasGateRes) gate = gate_at(p, m, n);
        const float y = finish<EPI>(acc[a][b][e], sx, split_scale(p.sw[n]), p.bias ? bf2f(p.bias[n]) : 0.f, res, gate);
        OutT* o = static_cast<OutT*>(p.y) + m * p.ldy + n;
        if constexpr (sizeof(OutT) == 4) *o = y;
        else *o = f2bf(y);
      }
  }
}

}  // namespace

template <int EPI, typename ResT, typename OutT>
static void launch_t(hipStream_t st, const IntGemmArgs& a) {
  const uint32_t tiles_m = (a.M + 31) / 32, tiles_n = (a.N + 63) / 64;
  const int64_t tiles = static_cast<int64_t>(tiles_m) * tiles_n;
  hipLaunchKernelGGL((int_gemm_simple<EPI, ResT, OutT>), dim3(static_cast<uint32_t>((tiles + 3) / 4)), dim3(256), 0, st,
                     a, tiles_m);
}

hipError_t launch_int_gemm(hipStream_t st, int epi, const IntGemmArgs& a) {
  if (a.M == 0) return hipSuccess;
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
