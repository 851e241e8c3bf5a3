// Microscaled blocks on gfx950: scales and codes of 32 values, and the pages
// that hold them (internal to libardit).
//
// A block of 32 values holds codes of 8 bits (E4M3) or 4 bits (E2M1) and one
// scale byte s = e + 127 for the power of two 2^e: the value of a code is
// code 2^e.  e is the smallest exponent, at least -117, with max|x| / 2^e below
// 256 (E4M3) or at most 6 (E2M1), so that no code saturates (E4M3 then may round
// up to 256); codes are rounded to nearest, ties to even.  A block with an
// infinity or NaN takes the scale byte 255, under which every code reads as NaN.
// From e >= -117 every code's value is a normal bf16 number or zero (the least
// is 2^-9 2^-117), so it is exact in bf16.
#pragma once

#include "launch.h"

namespace ardit {

constexpr int kMxMinScale = 10;   // scale byte of e = -117

// Scale byte of a block whose largest |x| has the bits m (no sign).
template <int BITS>
__device__ __forceinline__ int mx_scale_byte(uint32_t m) {
  const int E = static_cast<int>(m >> 23);   // 0 for subnormals: below the least exponent in any case
  int s;
  if constexpr (BITS == 8) s = E - 7;
  else s = min(E - 2 + ((m & 0x7fffffu) > 0x400000u ? 1 : 0), 252);   // (252: 6 2^125 is still a bf16 number)
  s = max(s, kMxMinScale);
  return m >= 0x7f800000u ? 255 : s;
}
// 2^-e for a scale byte (255: any number will do, the scale makes the block NaN)
__device__ __forceinline__ float mx_inverse(int s) {
  return __uint_as_float(static_cast<uint32_t>(254 - min(s, 253)) << 23);
}
// 2^e as the conversions take it (255 gives their NaN)
__device__ __forceinline__ float mx_scale(uint32_t s) { return __uint_as_float(s << 23); }

// Codes of 8 values scaled by inv = 2^-e: two words of E4M3, or one of E2M1 (in x).
template <int BITS>
__device__ __forceinline__ uint2 mx_encode8(const float* f, float inv) {
  uint2 r = make_uint2(0u, 0u);
  if constexpr (BITS == 8) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[0] * inv, f[1] * inv, 0, false);
    r.x = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(f[2] * inv, f[3] * inv, w, true));
    w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4] * inv, f[5] * inv, 0, false);
    r.y = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(f[6] * inv, f[7] * inv, w, true));
  } else {
    uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, f[0] * inv, f[1] * inv, 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2] * inv, f[3] * inv, 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4] * inv, f[5] * inv, 1.0f, 2);
    r.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6] * inv, f[7] * inv, 1.0f, 3);
  }
  return r;
}

// bf16 values of 8 codes: words a, b of E4M3, or word a of E2M1.
template <int BITS>
__device__ __forceinline__ u32x4 mx_decode8(uint32_t a, uint32_t b, float scale) {
  u32x4 r;
  if constexpr (BITS == 8) {
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true));
  } else {
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a, scale, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a, scale, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a, scale, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a, scale, 3));
  }
  return r;
}

// keys [0, left) of 8 bf16 values kept, the others zero
__device__ __forceinline__ u32x4 keep_first(u32x4 x, int left) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = 2 * i + 1 < left ? x[i] : (2 * i < left ? x[i] & 0xffffu : 0u);
  return x;
}

// Bytes of a tile of 64 keys of one head.
__host__ __device__ constexpr int mx_tile_bytes(int hd, int bits) { return 64 * hd * bits / 8; }
__host__ __device__ constexpr int mx_scale_bytes(int hd) { return 2 * hd; }   // 64 keys x hd / 32, and 2 x hd

// Tile index of (page, head, tile of the page): code tiles and scale tiles alike.
__device__ __forceinline__ size_t mx_tile(const MxPages& p, int page, int h, int ti) {
  return (static_cast<size_t>(page) * p.H + h) * p.nt + ti;
}
// Page of frame f of table row `row`, clamped into the pool (reads)
__device__ __forceinline__ int mx_read_page(const MxPages& p, int row, int f) {
  const int g = p.page_table[static_cast<size_t>(row) * p.max_frames + f];
  return min(max(g, 0), p.n_pages - 1);
}

}  // namespace ardit
