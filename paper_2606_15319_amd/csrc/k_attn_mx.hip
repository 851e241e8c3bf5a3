// Attention over microscaled key/value pages on gfx950.
//
// o = softmax(q K^T / sqrt(d)) V per (stream, head) over keys [0, kv_len), K and
// V the values that the pages' codes stand for (mx.h), q and o bf16.
//
// Scores.  Keys go into the matrix cores as they lie in the pages: the scaled
// product v_mfma_scale_f32_32x32x64_f8f6f4 takes E4M3 or E2M1 codes and applies a
// scale byte per 32 of its 64 steps.  The queries keep their 8 bits: a bf16 number
// is hi + lo with hi its four leading significant bits and lo the rest, both E4M3
// (hi with the block's scale, lo with one 2^-4 smaller; below 2^-13 of the block's
// largest element lo runs out of bits, an error of 2^-21 of that element).  Two
// products at twice bf16's rate, so the time of one in bf16, and the keys are never
// converted nor stored twice as wide.
//   S^T = K Q_hi^T + K Q_lo^T (32 keys x 32 queries a product).
// Weights.  exp2 in fp32 against a running maximum, rounded to bf16 (2^-9 of a
// weight at most, errors of both signs: about 1e-3 of an output), summed as rounded.
//   O^T += V^T P^T on v_mfma_f32_32x32x16_bf16, V converted to bf16 (exact).
//
// Operand layouts (measured): of the scaled product, lane m + 32 h holds row m and,
// of E4M3, steps 16 h .. + 16 and 32 + 16 h .. + 16; of E2M1 steps 32 h .. + 32; and
// supplies the scale of steps 32 h .. + 32.  Results: lane n + 32 h holds in register
// i row 8 (i / 4) + 4 h + i % 4 of column n.  Row r of key block b is key
// row_key(b, r), so that a lane's 32 scores are those of keys 32 h .. 32 h + 31 in
// order: step k of the second product (16 keys) takes from lane half h keys 32 h +
// 8 k .. + 8, so the weights need no exchange, and the value codes a lane of that
// product takes are 32 consecutive ones.
#include <math.h>
#include <string.h>

#include <algorithm>
#include <type_traits>

#include "mx.h"

namespace ardit {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Key of row r of key block b (32 rows each) of a tile.
__device__ __forceinline__ constexpr int row_key(int b, int r) {
  return 32 * ((r >> 2) & 1) + 16 * b + 4 * (r >> 3) + (r & 3);
}

// Lane id, formed where it is called for (two instructions) and held in no register.
__device__ __forceinline__ uint32_t lane_anew() {
  uint32_t zero = 0;
  asm volatile("" : "+s"(zero));
  return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, zero));
}

// max / sum over lanes l and l ^ 32
__device__ __forceinline__ float pair_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A query row's operands: hi and lo codes of 64 dims a step, and their scales: byte
// 2 ks hi's of step ks, byte 2 ks + 1 lo's (4 less).
template <int HD>
struct Query {
  i32x8 hi[HD / 64], lo[HD / 64];
  int sc;
};

// 16 dims of a block (the lane 32 on has its other 16) into words w0 .. w0 + 3
__device__ __forceinline__ void split_query(const uint4 (&raw)[2], i32x8& hi, i32x8& lo, int w0, int& sb) {
  float f[16];
  unpack8(raw[0], f);
  unpack8(raw[1], f + 8);
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(f[i]));
  m = pair_max(m);
  // max / 2^e in [128, 256); at least 2^-113, so that lo's scale stays a byte
  sb = max(static_cast<int>(__float_as_uint(m) >> 23) - 7, 14);
  const float inv = __uint_as_float(static_cast<uint32_t>(254 - sb) << 23);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float a = f[4 * w] * inv, b = f[4 * w + 1] * inv, c = f[4 * w + 2] * inv, d = f[4 * w + 3] * inv;
    int h = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    h = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, h, true);
    const auto p = __builtin_amdgcn_cvt_pk_f32_fp8(h, false), q = __builtin_amdgcn_cvt_pk_f32_fp8(h, true);
    int l = __builtin_amdgcn_cvt_pk_fp8_f32((a - p[0]) * 16.f, (b - p[1]) * 16.f, 0, false);
    l = __builtin_amdgcn_cvt_pk_fp8_f32((c - q[0]) * 16.f, (d - q[1]) * 16.f, l, true);
    hi[w0 + w] = h;
    lo[w0 + w] = l;
  }
}

// Query row at qp (its head's first dim); hh: lane / 32
template <int HD>
__device__ __forceinline__ void read_query(const bf16_t* qp, int hh, uint4 (&raw)[HD / 64][2][2]) {
#pragma unroll
  for (int ks = 0; ks < HD / 64; ++ks)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        raw[ks][b][i] = *reinterpret_cast<const uint4*>(qp + 64 * ks + 32 * b + 16 * hh + 8 * i);
}
template <int HD>
__device__ __forceinline__ void split_row(const uint4 (&raw)[HD / 64][2][2], int hh, Query<HD>& q) {
#pragma unroll
  for (int ks = 0; ks < HD / 64; ++ks) {
    int s0, s1;
    split_query(raw[ks][0], q.hi[ks], q.lo[ks], 0, s0);
    split_query(raw[ks][1], q.hi[ks], q.lo[ks], 4, s1);
    const int s = hh ? s1 : s0;
    q.sc = ks == 0 ? s + ((s - 4) << 8) : q.sc + (s << 16) + ((s - 4) << 24);
  }
}

// Key fragment of the 64-dim step ks from the rows at tk; at: byte offsets of this lane's
// 16-byte chunks.
template <int BITS>
__device__ __forceinline__ i32x8 key_fragment(const uint8_t* tk, const uint32_t* at, int ks) {
  if constexpr (BITS == 8) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(tk + at[2 * ks]), y = *reinterpret_cast<const u32x4*>(tk + at[2 * ks + 1]);
    return i32x8{static_cast<int>(x[0]), static_cast<int>(x[1]), static_cast<int>(x[2]), static_cast<int>(x[3]),
                 static_cast<int>(y[0]), static_cast<int>(y[1]), static_cast<int>(y[2]), static_cast<int>(y[3])};
  } else {
    const u32x4 x = *reinterpret_cast<const u32x4*>(tk + at[ks]);
    return i32x8{static_cast<int>(x[0]), static_cast<int>(x[1]), static_cast<int>(x[2]), static_cast<int>(x[3]), 0, 0, 0, 0};
  }
}

// S^T of a tile's two 32-key blocks; sk: each key's scale bytes, shifted by the lane's
// half, so that byte 2 ks is that of the 64-dim step ks.
template <int HD, int BITS>
__device__ __forceinline__ void scores(const i32x8 (&k)[2][HD / 64], const uint32_t (&sk)[2], const Query<HD>& q,
                                       f32x16 (&s)[2]) {
  constexpr int FMT = BITS == 8 ? 0 : 4;
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
  // (which byte of a scale operand: an immediate of the instruction)
#pragma unroll
  for (int b = 0; b < 2; ++b)
    s[b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k[b][0], q.hi[0], s[b], FMT, 0, 0, static_cast<int>(sk[b]), 0, q.sc);
#pragma unroll
  for (int b = 0; b < 2; ++b)
    s[b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k[b][0], q.lo[0], s[b], FMT, 0, 0, static_cast<int>(sk[b]), 1, q.sc);
  if constexpr (HD == 128) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
      s[b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k[b][1], q.hi[1], s[b], FMT, 0, 2, static_cast<int>(sk[b]), 2, q.sc);
#pragma unroll
    for (int b = 0; b < 2; ++b)
      s[b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k[b][1], q.lo[1], s[b], FMT, 0, 2, static_cast<int>(sk[b]), 3, q.sc);
  }
}

// Weights p[i0 .. i0 + 8) as one operand of the value product; sum: their sum as rounded.
__device__ __forceinline__ bf16x8 pack_weights(const f32x16& p, int i0, float& sum) {
  const bf16x2 one2 = {static_cast<__bf16>(1.0f), static_cast<__bf16>(1.0f)};
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    w[j] = pack_bf16x2(p[i0 + 2 * j], p[i0 + 2 * j + 1]);
    sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[j]), one2, sum, false);
  }
  return __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
}

// 16-byte chunk c of an LDS row of ROWB bytes sits at chunk c ^ swz(r): 16 rows then
// cover every bank for a fixed c.
template <int ROWB>
__device__ __forceinline__ int swz(int r) { return (r / (256 / ROWB)) & (ROWB / 16 - 1); }

// ------------------------------------------------------------- few queries
// A workgroup takes 32 rows of one (stream, head) and a cut of its key tiles, each of
// its eight waves every eighth tile; the waves meet in LDS.  A wave's tiles are its own:
// they come by direct loads into a ring of 16 KB a wave, 1 to 4 tiles, so that a CU
// has 128 KB under way whatever the format, and nobody waits for another wave.  A tile's
// bytes go to registers at once and its place in the ring to the next one.  Cuts of
// one row tile leave partial results (unnormalised o, running maximum, denominator)
// that a second kernel joins.  Spans of few tiles are solo: a cut is one wave's, and
// the eight waves of a workgroup are on their own.
// What bounds it: the cache's bytes.  Eight tokens over 9 to 21 frames each, 12 heads of
// 128, in 8 bits 106 to 110 us with the join's 5, 5 TB/s (in 4 bits 58); as first built,
// with four waves and rings of 32 KB 117 for 113 (in 4 bits 86 for 66).
constexpr int SM_BQ = 32;
constexpr int SM_WAVES = 8;

template <int HD, int BITS>
struct Ring {
  static constexpr int TILES = 16384 / (2 * mx_tile_bytes(HD, BITS));
  struct Tile {
    uint8_t k[mx_tile_bytes(HD, BITS)];     // row R = 32 b + r: key row_key(b, r), chunks swizzled
    uint8_t v[mx_tile_bytes(HD, BITS)];     // row: dim, chunks swizzled
    uint8_t ks[mx_scale_bytes(HD)], vs[mx_scale_bytes(HD)];
  };
  Tile t[SM_WAVES][TILES];
};
template <int HD>
struct Meeting {
  float o[SM_WAVES][SM_BQ][HD];
  float m[SM_WAVES][SM_BQ], l[SM_WAVES][SM_BQ];
};

template <int HD, int BITS>
__global__ __launch_bounds__(64 * SM_WAVES, 1) void attn_mx_small_kernel(const MxSmallArgs a) {
  constexpr int DB = HD / 32, KS = HD / 64;
  constexpr int TB = mx_tile_bytes(HD, BITS), SB = mx_scale_bytes(HD);
  constexpr int NL = TB / 1024;                        // loads of a tile of keys, and of values
  constexpr int KROW = HD * BITS / 8, VROW = 8 * BITS;   // bytes of a key, and of a dim's 64 keys
  constexpr int NT = Ring<HD, BITS>::TILES;
  constexpr int LOADS = 2 * NL + 2;
  static_assert((NT - 1) * LOADS < 64, "the counter of loads under way has six bits");
  __shared__ union __attribute__((aligned(1024))) Lds {
    Ring<HD, BITS> ring;
    Meeting<HD> part;
  } lds;
  const MxPages& p = a.p;
  const int xcd = static_cast<int>(blockIdx.x) % kNumXcd, j = static_cast<int>(blockIdx.x) / kNumXcd;
  // first of a run's workgroups in the XCD's list
  auto first = [&](const MxRun& r) { return r.eighths + r.rest / kNumXcd + (xcd < r.rest % kNumXcd ? 1 : 0); };
  if (j >= first(a.run[a.n_runs])) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // the last run that begins at or before the workgroup, and of solo spans the last that
  // begins at or before the wave: a lane looks at one of the others (one after the other
  // they cost a scalar load and a wait each)
  const int e = __builtin_popcountll(__ballot(lane + 1 < a.n_runs && j >= first(a.run[min(lane + 1, a.n_runs)])));
  const MxRun R = a.run[e], next = a.run[e + 1];
  const int turn = (xcd - R.rest) & (kNumXcd - 1);   // the run's pieces begin with the XCD whose turn it is
  int it = j - first(R) + turn * (next.eighths - R.eighths) + min(turn, next.rest - R.rest);
  int si = a.run_span[e];
  const bool solo = si >= a.solo_span;
  if (solo) {
    it = it * SM_WAVES + wave;
    if (it >= a.solo_waves) return;
    si += __builtin_popcountll(__ballot(si + lane + 1 < a.n_spans &&
                                        it >= a.s[min(si + lane + 1, kMaxStreams)].wave_begin));
  }
  const MxSpan S = a.s[__builtin_amdgcn_readfirstlane(si)];
  if (solo) it -= S.wave_begin;
  const int hp = it / S.n_qtiles, qt = it - hp * S.n_qtiles;
  const int h = hp / S.pieces, piece = hp - h * S.pieces;
  const int tb = S.tile0 + piece * S.per_piece, te = min(S.tile1, tb + S.per_piece);
  const int t0 = solo ? tb : tb + wave, stride = solo ? 1 : SM_WAVES;   // the wave's tiles
  const int n = lane & 31, hh = lane >> 5;
  const float c = a.scale_log2;

  // pages of 64 frames, a lane each, from the frame of the next tile requested on
  const int last_frame = static_cast<int>(fdiv(static_cast<uint32_t>(S.kv_len - 1), p.fT));
  const int32_t* pt = p.page_table + static_cast<size_t>(S.row) * p.max_frames;
  auto page_window = [&](int f0) __attribute__((always_inline)) {
    return min(max(pt[min(f0 + lane, last_frame)], 0), p.n_pages - 1);
  };
  int pw0 = static_cast<int>(fdiv(static_cast<uint32_t>(min(t0, te - 1)), p.fnt));
  int pw = page_window(pw0);
  const bf16_t* qp = a.q + static_cast<size_t>(S.q_off + min(qt * SM_BQ + n, S.q_len - 1)) * a.ld + h * HD;
  uint4 raw[KS][2][2];
  read_query<HD>(qp, hh, raw);
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)   // the row and the pages have landed before the first direct load
    asm volatile("" : "+v"(raw[ks][0][0].x), "+v"(raw[ks][0][1].x), "+v"(raw[ks][1][0].x), "+v"(raw[ks][1][1].x),
                 "+v"(pw));

  // direct loads.  Load j of the keys fills LDS rows j (1024 / KROW) ..; of the values alike.
  uint32_t k_off[NL], v_off[NL];
#pragma unroll
  for (int j = 0; j < NL; ++j) {
    const int R = j * (1024 / KROW) + lane / (KROW / 16), D = j * (1024 / VROW) + lane / (VROW / 16);
    k_off[j] = static_cast<uint32_t>(row_key(R >> 5, R & 31) * KROW + (((lane % (KROW / 16)) ^ swz<KROW>(R)) << 4));
    v_off[j] = static_cast<uint32_t>(D * VROW + (((lane % (VROW / 16)) ^ swz<VROW>(D)) << 4));
  }
  const uint32_t s_off = static_cast<uint32_t>(lane * 4);
  typename Ring<HD, BITS>::Tile* ring = lds.ring.t[wave];
  const uint32_t lds_ring = lds_address(ring);
  auto fetch = [&](int t, int slot) __attribute__((always_inline)) {
    const int f = static_cast<int>(fdiv(static_cast<uint32_t>(t), p.fnt));
    if (f - pw0 >= 64) {
      pw0 = f;
      pw = page_window(f);
      asm volatile("" : "+v"(pw));
    }
    const size_t tile = mx_tile(p, __builtin_amdgcn_readlane(pw, f - pw0), h, t - f * p.nt);
    const uint32_t at = lds_ring + static_cast<uint32_t>(slot) * sizeof(typename Ring<HD, BITS>::Tile);
    const char* kc = reinterpret_cast<const char*>(p.k) + tile * TB;
    const char* vc = reinterpret_cast<const char*>(p.v) + tile * TB;
#pragma unroll
    for (int j = 0; j < NL; ++j) lds_dma16(kc, k_off[j], at + 1024u * j);
#pragma unroll
    for (int j = 0; j < NL; ++j) lds_dma16(vc, v_off[j], at + TB + 1024u * j);
    if (lane < SB / 4) {
      lds_dma4(reinterpret_cast<const char*>(p.ks) + tile * SB, s_off, at + 2 * TB);
      lds_dma4(reinterpret_cast<const char*>(p.vs) + tile * SB, s_off, at + 2 * TB + SB);
    }
  };
#pragma unroll 1
  for (int i = 0; i < NT; ++i)
    if (t0 + stride * i < te) fetch(t0 + stride * i, i);

  Query<HD> q;
  split_row<HD>(raw, hh, q);
  // byte offsets of this lane's fragments in a tile
  uint32_t k_at[KS * BITS / 4];
  int ks_at[2], v_at[BITS / 4];
#pragma unroll
  for (int i = 0; i < KS * BITS / 4; ++i) k_at[i] = static_cast<uint32_t>(n * KROW + (((2 * i + hh) ^ swz<KROW>(n)) << 4));
#pragma unroll
  for (int b = 0; b < 2; ++b) ks_at[b] = row_key(b, n) * (HD / 32);
#pragma unroll
  for (int i = 0; i < BITS / 4; ++i) v_at[i] = n * VROW + (((hh * (BITS / 4) + i) ^ swz<VROW>(n)) << 4);

  f32x16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  // (it starts finite, so that scores that all overflowed to -inf weigh nothing)
  float m_run = kNoMax, l_run = 0.f;
  int slot = 0;
#pragma unroll 1
  for (int t = t0; t < te; t += stride) {
    // this tile has landed: those after it are under way, NT - 1 of them but at the end
    if (t + stride * (NT - 1) < te) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NT - 1) * LOADS) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const typename Ring<HD, BITS>::Tile& tile = ring[slot];
    i32x8 kf[2][KS];
    uint32_t sk[2], vsb[DB];
    u32x4 vw[DB][BITS / 4];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      if constexpr (HD == 128) sk[b] = *reinterpret_cast<const uint32_t*>(tile.ks + ks_at[b]);
      else sk[b] = *reinterpret_cast<const uint16_t*>(tile.ks + ks_at[b]);
      sk[b] >>= 8 * hh;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) kf[b][ks] = key_fragment<BITS>(tile.k + 32 * KROW * b, k_at, ks);
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) {
#pragma unroll
      for (int i = 0; i < BITS / 4; ++i) vw[db][i] = *reinterpret_cast<const u32x4*>(tile.v + 32 * VROW * db + v_at[i]);
      vsb[db] = tile.vs[hh * HD + 32 * db + n];
    }
    // everything read: the slot takes the tile after those under way
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (t + stride * NT < te) fetch(t + stride * NT, slot);
    slot = slot + 1 == NT ? 0 : slot + 1;
    const int f = static_cast<int>(fdiv(static_cast<uint32_t>(t), p.fnt));
    const int keys = min(64, min(p.T, S.kv_len - f * p.T) - 64 * (t - f * p.nt));
    f32x16 s[2];
    scores<HD, BITS>(kf, sk, q, s);
    if (keys < 64) {
      const int left = keys - 32 * hh;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[b][i] = 16 * b + i < left ? s[b][i] : -INFINITY;
      // Values past the end are zero: whatever the page holds there would meet a zero
      // weight.  Codes are cut with one mask a word for all dims of a lane (six ragged
      // streams over pages of 72 keys 66 us with their bf16 values cut, 53 so).  A block
      // without keys may hold any scale.
      constexpr int PER = 32 / BITS;   // codes of a word
#pragma unroll
      for (int w = 0; w < BITS; ++w) {
        const int n_in = left - PER * w;
        const uint32_t mask = n_in >= PER ? ~0u : (n_in <= 0 ? 0u : (1u << (BITS * n_in)) - 1u);
#pragma unroll
        for (int db = 0; db < DB; ++db) vw[db][w >> 2][w & 3] &= mask;
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) vsb[db] = left > 0 ? vsb[db] : 127u;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[b][i]);
    mx = pair_max(mx) * c;
    // raised only when a tile's maximum exceeds it by more than 8 (weights stay below
    // 2^8), so that o is seldom rescaled
    if (__any(mx > m_run + 8.0f)) {
      const float m_new = fmaxf(m_run, mx);
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
    }
    bf16x8 pf[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      f32x16 w;
#pragma unroll
      for (int i = 8 * (k & 1); i < 8 * (k & 1) + 8; ++i) w[i] = __builtin_amdgcn_exp2f(fmaf(s[k >> 1][i], c, -m_run));
      pf[k] = pack_weights(w, 8 * (k & 1), l_run);
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const float sc = mx_scale(vsb[db]);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        u32x4 x;
        if constexpr (BITS == 8) x = mx_decode8<8>(vw[db][k >> 1][2 * (k & 1)], vw[db][k >> 1][2 * (k & 1) + 1], sc);
        else x = mx_decode8<4>(vw[db][0][k], 0u, sc);
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), pf[k], o[db], 0, 0, 0);
      }
    }
  }
  const float l_tot = pair_sum(l_run);
  if (solo) {   // lane n + 32 hh holds dims 32 db + 8 g + 4 hh .. + 4 of its query
    const int ql = qt * SM_BQ + n;
    if (ql >= S.q_len) return;
    if (S.part_begin < 0) {
      const float inv = 1.0f / l_tot;
      bf16_t* op = a.o + static_cast<size_t>(S.q_off + ql) * a.ld + h * HD;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          uint2 w;
          w.x = pack_bf16x2(o[db][4 * g] * inv, o[db][4 * g + 1] * inv);
          w.y = pack_bf16x2(o[db][4 * g + 2] * inv, o[db][4 * g + 3] * inv);
          *reinterpret_cast<uint2*>(op + 32 * db + 8 * g + 4 * hh) = w;
        }
    } else {
      const size_t at = S.part_begin + static_cast<size_t>(hp) * S.q_len + ql;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<float4*>(a.part_o + at * HD + 32 * db + 8 * g + 4 * hh) =
              make_float4(o[db][4 * g], o[db][4 * g + 1], o[db][4 * g + 2], o[db][4 * g + 3]);
      if (hh == 0) a.part_ml[at] = make_float2(m_run, l_tot);
    }
    return;
  }
  __syncthreads();   // the rings make room for the results

  // the waves' results meet: o = sum_w 2^(m_w - M) o_w (a wave without tiles adds nothing)
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {   // dims 32 db + 8 g + 4 hh .. + 4; 16-byte chunks XOR-swizzled by row
      const int ch = 8 * db + 2 * g + hh;
      *reinterpret_cast<float4*>(&lds.part.o[wave][n][4 * (ch ^ (n & 15))]) =
          make_float4(o[db][4 * g], o[db][4 * g + 1], o[db][4 * g + 2], o[db][4 * g + 3]);
    }
  if (hh == 0) {
    lds.part.m[wave][n] = m_run;
    lds.part.l[wave][n] = l_tot;
  }
  __syncthreads();
  constexpr int TPR = HD / 4;
  for (int i = tid; i < SM_BQ * TPR; i += 64 * SM_WAVES) {
    const int row = i / TPR, c4 = i % TPR;
    const int ql = qt * SM_BQ + row;
    if (ql >= S.q_len) break;
    float M = lds.part.m[0][row];
#pragma unroll
    for (int w = 1; w < SM_WAVES; ++w) M = fmaxf(M, lds.part.m[w][row]);
    float l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < SM_WAVES; ++w) {
      if (tb + w >= te) break;
      const float wgt = __builtin_amdgcn_exp2f(lds.part.m[w][row] - M);
      const float4 x = *reinterpret_cast<const float4*>(&lds.part.o[w][row][4 * (c4 ^ (row & 15))]);
      l += wgt * lds.part.l[w][row];
      acc.x += wgt * x.x;
      acc.y += wgt * x.y;
      acc.z += wgt * x.z;
      acc.w += wgt * x.w;
    }
    if (S.part_begin < 0) {
      const float inv = 1.0f / l;
      uint2 w;
      w.x = pack_bf16x2(acc.x * inv, acc.y * inv);
      w.y = pack_bf16x2(acc.z * inv, acc.w * inv);
      *reinterpret_cast<uint2*>(a.o + static_cast<size_t>(S.q_off + ql) * a.ld + h * HD + 4 * c4) = w;
    } else {
      const size_t slot = S.part_begin + static_cast<size_t>(hp) * S.q_len + ql;
      *reinterpret_cast<float4*>(a.part_o + slot * HD + 4 * c4) = acc;
      if (c4 == 0) a.part_ml[slot] = make_float2(M, l);
    }
  }
}

// Joins the partial results of a row: those of its stream's cuts and, when the batch
// shares a prefix, of the prefix's.  Rows that were written whole, or that are the other
// kernel's, are not counted.  HD / 4 lanes hold a row; a.groups such groups, at
// least a wave, take the cuts in turn and meet in LDS: one token over 32760 keys, one head,
// 14 us for 16 with the groups of a wave (27 cuts: one group of lanes took 16 us for the
// join alone, one trip to memory after the other, a wave of them 5).
template <int HD>
__global__ __launch_bounds__(256) void attn_mx_join_kernel(const MxSmallArgs a) {
  constexpr int TPR = HD / 4, NG = 256 / TPR;
  __shared__ float4 part_o[NG][TPR];
  __shared__ float2 part_ml[NG];
  const int grp = static_cast<int>(threadIdx.x) / TPR, c4 = threadIdx.x % TPR, lane = threadIdx.x & 63;
  const int sub = grp & (a.groups - 1);
  const int i = (static_cast<int>(blockIdx.x) * NG + grp) / a.groups;   // head-major rows, one to a wave
  const int h = __builtin_amdgcn_readfirstlane(i / a.join_rows), jr = __builtin_amdgcn_readfirstlane(i - h * a.join_rows);
  // the stream's span (in any order; each holds its rows once)
  const MxSpan& mine = a.s[min(a.shared + lane, kMaxStreams)];
  const uint64_t hit = __ballot(a.shared + lane < a.n_spans && mine.part_begin >= 0 && jr >= mine.join_begin &&
                                jr - mine.join_begin < mine.q_len);
  const int si = a.shared + (hit ? __builtin_ctzll(hit) : 0);
  const MxSpan S = a.s[__builtin_amdgcn_readfirstlane(si)];
  const int r = S.q_off + jr - S.join_begin;
  const bool join = h < a.p.H && hit != 0;
  const MxSpan& P = a.s[0];
  const int own = S.pieces, all = join ? own + (a.shared ? P.pieces : 0) : 0;
  float M = kNoMax, l = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int j = sub; j < all; j += a.groups) {
    const size_t at = j < own ? S.part_begin + (static_cast<size_t>(h) * own + j) * S.q_len + (r - S.q_off)
                              : P.part_begin + (static_cast<size_t>(h) * P.pieces + j - own) * P.q_len + r;
    const float2 ml = a.part_ml[at];
    const float4 x = *reinterpret_cast<const float4*>(a.part_o + at * HD + 4 * c4);
    const float m_new = fmaxf(M, ml.x);
    const float keep = __builtin_amdgcn_exp2f(M - m_new), wgt = __builtin_amdgcn_exp2f(ml.x - m_new);
    M = m_new;
    l = l * keep + wgt * ml.y;
    acc.x = acc.x * keep + wgt * x.x;
    acc.y = acc.y * keep + wgt * x.y;
    acc.z = acc.z * keep + wgt * x.z;
    acc.w = acc.w * keep + wgt * x.w;
  }
  part_o[grp][c4] = acc;
  if (c4 == 0) part_ml[grp] = make_float2(M, l);
  __syncthreads();
  if (sub != 0 || !join) return;
  const float own_m = M;
  for (int g = 1; g < a.groups; ++g) M = fmaxf(M, part_ml[grp + g].x);
  const float first = __builtin_amdgcn_exp2f(own_m - M);
  l *= first;
  acc.x *= first;
  acc.y *= first;
  acc.z *= first;
  acc.w *= first;
  for (int g = 1; g < a.groups; ++g) {
    const float2 ml = part_ml[grp + g];
    const float wgt = __builtin_amdgcn_exp2f(ml.x - M);
    const float4 x = part_o[grp + g][c4];
    l += wgt * ml.y;
    acc.x += wgt * x.x;
    acc.y += wgt * x.y;
    acc.z += wgt * x.z;
    acc.w += wgt * x.w;
  }
  const float inv = 1.0f / l;
  uint2 w;
  w.x = pack_bf16x2(acc.x * inv, acc.y * inv);
  w.y = pack_bf16x2(acc.z * inv, acc.w * inv);
  *reinterpret_cast<uint2*>(a.o + static_cast<size_t>(r) * a.ld + h * HD + 4 * c4) = w;
}

// ------------------------------------------------------------ whole chunks
// Items of 256 queries of one (stream, head), eight waves of 32 rows; key tiles are
// shared through LDS.  AttnArgs is planned as for the bf16 attention, with a
// stream's tiles counted page by page; base_off holds its number of keys.
struct MxLargeArgs {
  AttnArgs a;
  MxPages p;
};
static_assert(sizeof(MxLargeArgs) <= 4096, "arguments must fit the kernel-argument buffer");

constexpr int BQ = 256;
constexpr int NTHR = 512;
constexpr int AHEAD = 3;          // tiles requested ahead of the one computed
constexpr int NSLOT = AHEAD + 1;  // tiles of codes in LDS

template <int HD, int BITS>
struct LargeLds {
  uint8_t k[NSLOT][mx_tile_bytes(HD, BITS)];      // row R = 32 b + r: key row_key(b, r)
  uint8_t v[NSLOT][mx_tile_bytes(HD, BITS)];      // as in the page
  bf16_t vb[2][64 * HD];                          // [dim][64 keys]
  uint8_t ks[NSLOT][mx_scale_bytes(HD)];
  uint8_t vs[NSLOT][mx_scale_bytes(HD)];
};

// Runs key tiles [tb, te) of item (S, head h, query tile qt), then writes the
// normalised output (slot < 0) or partial results into slot `slot`.
//
// The two waves of a SIMD run half a tile apart, as in the bf16 attention: a position's
// work is an MFMA phase (O += V P of the position before, S = K Q) and a VALU phase
// (softmax, requests for tiles to come), one barrier a position, group 0 before its
// MFMA phase and group 1 before its VALU phase.  Interval t (after barrier t) reads
// the keys of position t, turns its value codes into bf16 (slot t % 2, each thread
// HD / 8 of them) and reads the bf16 values of position t - 1; it requests the codes
// and scales of position t + 3, whose slots were last read in interval t - 1.
template <int HD, int BITS, bool PAIR>
__device__ __forceinline__ void mx_range(const AttnArgs& a, const MxPages& p, const AttnStream& S, int h, int qt,
                                         int tb, int te, LargeLds<HD, BITS>& lds, int64_t slot) {
  constexpr int KS = HD / 64, DB = HD / 32;
  constexpr int TB = mx_tile_bytes(HD, BITS), SB = mx_scale_bytes(HD);
  constexpr int NL = TB / 1024;            // 1 KB loads of a tile of keys, and of values
  constexpr int KROW = HD * BITS / 8;      // bytes of a key
  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n32 = lane & 31, hh = lane >> 5;
  const int grp = wave >> 2;
  const int n = te - tb;
  const float c = a.scale_log2;
  const int kv_len = S.base_off;

  Query<HD> q;
  {
    uint4 raw[KS][2][2];
    read_query<HD>(a.q + static_cast<size_t>(S.q_off + min(qt * BQ + wave * 32 + n32, S.q_len - 1)) * a.ldq + h * HD,
                   hh, raw);
    split_row<HD>(raw, hh, q);
  }

  // ---- staging by direct loads.  Eight loads a tile: every wave one of keys and one of
  // values; four: waves 0-3 keys, 4-7 values; two: waves 0, 1 and 4, 5.
  constexpr bool BOTH = NL == 8;
  const bool loads_k = BOTH || wave < NL, loads_v = BOTH || (wave >= 4 && wave - 4 < NL);
  const int piece = BOTH ? wave : (wave & 3);
  const int ks_wave = NL == 2 ? 2 : 0, vs_wave = NL == 2 ? 6 : (BOTH ? 1 : 4);
  const int kR = piece * (1024 / KROW) + lane / (KROW / 16);
  const uint32_t k_off = static_cast<uint32_t>(row_key((kR >> 5) & 1, kR & 31) * KROW +
                                               (((lane % (KROW / 16)) ^ swz<KROW>(kR)) << 4));
  const uint32_t lds_k = lds_address(lds.k) + piece * 1024u, lds_v = lds_address(lds.v) + piece * 1024u;
  const uint32_t lds_ks = lds_address(lds.ks), lds_vs = lds_address(lds.vs);

  const int last_frame = static_cast<int>(fdiv(static_cast<uint32_t>(kv_len - 1), p.fT));
  const int32_t* pt = p.page_table + static_cast<size_t>(S.stream) * p.max_frames;
  // lane i: page of frame f0 + i, clamped into the pool
  auto page_window = [&](int f0) __attribute__((always_inline)) {
    return min(max(pt[min(f0 + lane, last_frame)], 0), p.n_pages - 1);
  };
  int fr = static_cast<int>(fdiv(static_cast<uint32_t>(tb), p.fnt));   // frame and tile requested next
  int ti = tb - fr * p.nt;
  int pw0 = fr, pw = page_window(fr);
  size_t tile = mx_tile(p, __builtin_amdgcn_readlane(pw, 0), h, ti);
  // requests position u, the one after those requested (u < n)
  auto stage = [&](int u) __attribute__((always_inline)) {
    const uint32_t sl = static_cast<uint32_t>(u % NSLOT);
    const char* kc = reinterpret_cast<const char*>(p.k) + tile * TB;
    const char* vc = reinterpret_cast<const char*>(p.v) + tile * TB + piece * 1024;
    const uint32_t ln = PAIR ? lane_anew() : lane, v_off = ln * 16u, s_off = ln * 4u;
    if (loads_k) lds_dma16(kc, k_off, lds_k + sl * TB);
    if (loads_v) lds_dma16(vc, v_off, lds_v + sl * TB);
    if (wave == ks_wave && ln < SB / 4)
      lds_dma4(reinterpret_cast<const char*>(p.ks) + tile * SB, s_off, lds_ks + sl * SB);
    if (wave == vs_wave && ln < SB / 4)
      lds_dma4(reinterpret_cast<const char*>(p.vs) + tile * SB, s_off, lds_vs + sl * SB);
    ++tile;
    if (++ti == p.nt) {
      ti = 0;
      ++fr;
      if (fr - pw0 >= 64) {
        pw0 = fr;
        pw = page_window(fr);
        asm volatile("" : "+v"(pw));   // waited for here, so no later wait has to
      }
      if (u + 1 < n) tile = mx_tile(p, __builtin_amdgcn_readlane(pw, fr - pw0), h, 0);
    }
  };
  const int per_pair = (loads_k ? 1 : 0) + (loads_v ? 1 : 0) + (wave == ks_wave ? 1 : 0) + (wave == vs_wave ? 1 : 0);
  // all but the last P positions requested by this wave have landed
  auto wait_pairs = [&](auto pairs_c) __attribute__((always_inline)) {
    constexpr int P = decltype(pairs_c)::value;
    if (per_pair == 3) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * P) : "memory");
    else if (per_pair == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * P) : "memory");
    else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(P) : "memory");
  };
  const std::integral_constant<int, 0> w0;
  const std::integral_constant<int, 2> w2;
  const std::integral_constant<int, 3> w3;
  // keys of position t's tile
  auto keys_of = [&](int t) __attribute__((always_inline)) {
    const int f = static_cast<int>(fdiv(static_cast<uint32_t>(tb + t), p.fnt));
    return min(64, min(p.T, kv_len - f * p.T) - 64 * (tb + t - f * p.nt));
  };

  // byte offsets of this lane's fragments in a tile
  // (of keys 16-byte chunk 2 i + hh of row n32, row 32 + n32 32 KROW on; of values chunk
  // 4 hh + k.  PAIR: from the first, of which the others are an XOR away)
  constexpr int NK = KS * BITS / 4;
  uint32_t k_at[NK], v_at[4];
#pragma unroll
  for (int i = 0; i < NK; ++i) k_at[i] = static_cast<uint32_t>(n32 * KROW + (((2 * i + hh) ^ swz<KROW>(n32)) << 4));
#pragma unroll
  for (int k = 0; k < 4; ++k) v_at[k] = static_cast<uint32_t>(n32 * 128 + (((4 * hh + k) ^ swz<128>(n32)) << 4));
  const uint32_t ks_at = static_cast<uint32_t>(row_key(0, n32) * (HD / 32));
  static_assert(row_key(1, 0) == 16 && row_key(1, 31) == row_key(0, 31) + 16, "block 1's keys are 16 on");

  f32x16 o[DB], s[2];
  bf16x8 pf[4];                // weights as the products take them
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  float m_run = kNoMax, l_run = 0.f;

  // value codes of position t to bf16: this thread HD / 8 keys of one dim
  auto convert = [&](int t, auto cut_c, int keys) __attribute__((always_inline)) {
    constexpr int E = HD / 8;
    const int dim = tid / (64 / E), k0 = E * (tid % (64 / E));
    const uint8_t* src = lds.v[t % NSLOT] + tid * (E * BITS / 8);
    const float sc = mx_scale(lds.vs[t % NSLOT][(k0 >> 5) * HD + dim]);
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    if constexpr (E * BITS == 128) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(src);
      w[0] = x[0]; w[1] = x[1]; w[2] = x[2]; w[3] = x[3];
    } else if constexpr (E * BITS == 64) {
      const uint2 x = *reinterpret_cast<const uint2*>(src);
      w[0] = x.x; w[1] = x.y;
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(src);
    }
    bf16_t* dst = lds.vb[t & 1] + dim * 64;
#pragma unroll
    for (int i = 0; i < E / 8; ++i) {
      u32x4 x = BITS == 8 ? mx_decode8<BITS>(w[2 * i], w[2 * i + 1], sc) : mx_decode8<BITS>(w[i], 0u, sc);
      if constexpr (decltype(cut_c)::value) x = keep_first(x, keys - k0 - 8 * i);
      *reinterpret_cast<u32x4*>(dst + 8 * ((k0 / 8 + i) ^ swz<128>(dim))) = x;
    }
  };
  const std::true_type yes;
  const std::false_type no;
  // (a tile that is not whole is written again with zeros past its keys)
  auto trim = [&](int t) __attribute__((always_inline)) {
    const int keys = keys_of(t);
    if (keys < 64) convert(t, yes, keys);
  };
  auto mfma_phase = [&](int t, auto pv_c, auto qk_c) __attribute__((always_inline)) {
    constexpr bool PV = decltype(pv_c)::value, QK = decltype(qk_c)::value;
    __builtin_amdgcn_s_setprio(1);
    bf16x8 vf[4][DB];
    if constexpr (QK) {
      const uint32_t slot_at = static_cast<uint32_t>((t % NSLOT) * TB);
      uint32_t at[NK];
#pragma unroll
      for (int i = 0; i < NK; ++i) at[i] = PAIR ? (slot_at + k_at[0]) ^ (32u * i) : slot_at + k_at[i];
      const uint8_t* tks = lds.ks[t % NSLOT] + ks_at;
      i32x8 kf[2][KS];
      uint32_t sk[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        if constexpr (HD == 128) sk[b] = *reinterpret_cast<const uint32_t*>(tks + 16 * b * (HD / 32));
        else sk[b] = *reinterpret_cast<const uint16_t*>(tks + 16 * b * (HD / 32));
        sk[b] >>= 8 * hh;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[b][ks] = key_fragment<BITS>(lds.k[0] + 32 * KROW * b, at, ks);
      }
      scores<HD, BITS>(kf, sk, q, s);
    }
    if constexpr (PV) {
      const uint8_t* tv = reinterpret_cast<const uint8_t*>(&lds.vb[0][0]);
      const uint32_t tile_at = static_cast<uint32_t>(((t - 1) & 1) * (128 * HD));
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t at = PAIR ? (tile_at + v_at[0]) ^ (16u * k) : tile_at + v_at[k];
#pragma unroll
        for (int db = 0; db < DB; ++db) vf[k][db] = *reinterpret_cast<const bf16x8*>(tv + at + 4096 * db);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int db = 0; db < DB; ++db)
          o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[k][db], pf[k], o[db], 0, 0, 0);
    }
    if constexpr (QK) convert(t, no, 64);
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
  };

  // VALU phase: the weights of the scores, against the running maximum as it is, and
  // their sum.  A row whose weights sum to more than 2^14 (or to no number) raises the
  // maximum and forms them again; a tile's maximum is seldom taken.  (Taken for every
  // tile, 4680 queries over 37440 keys, 20 heads of 128, 8 bits 1523 us for 1511, 4 bits
  // 1475 for 1450; at d = 64 as fast, but in more registers than two on a CU have.)
  auto softmax = [&](int keys) __attribute__((always_inline)) {
    if (keys < 64) {
      const int left = keys - (PAIR ? static_cast<int>(lane_anew() & 32u) : 32 * hh);
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[b][i] = 16 * b + i < left ? s[b][i] : -INFINITY;
    }
    float s0 = 0.f, s1 = 0.f;
    auto weigh = [&]() __attribute__((always_inline)) {
      s0 = s1 = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        f32x16 p;
#pragma unroll
        for (int i = 8 * (k & 1); i < 8 * (k & 1) + 8; ++i)
          p[i] = __builtin_amdgcn_exp2f(fmaf(s[k >> 1][i], c, -m_run));
        pf[k] = pack_weights(p, 8 * (k & 1), k & 1 ? s1 : s0);
      }
    };
    weigh();
    if (__any(!(s0 + s1 <= 16384.f))) {
      float top = -INFINITY;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
      const float m_new = fmaxf(m_run, pair_max(top) * c);
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
      weigh();
    }
    l_run += s0 + s1;
    asm volatile("" : "+v"(pf[0]), "+v"(pf[1]), "+v"(pf[2]), "+v"(pf[3]), "+v"(l_run));
  };

  // ---- prologue: the positions ahead of the group's first VALU phase
#pragma unroll 1
  for (int u = 0; u < AHEAD + grp; ++u)
    if (u < n) stage(u);
  if (AHEAD + grp > n) wait_pairs(w0);
  else if (grp == 0) wait_pairs(w2);
  else wait_pairs(w3);
  __syncthreads();
  auto wait_next = [&](int u) __attribute__((always_inline)) {   // u: the last position requested
    if (u < n) wait_pairs(w2);
    else wait_pairs(w0);
  };
  if (qt * BQ + wave * 32 < S.q_len) {
    mfma_phase(0, no, yes);
    trim(0);
#pragma unroll 1
    for (int t = 0; t + 1 < n; ++t) {
      if (grp == 1) {
        wait_next(t + AHEAD);
        __syncthreads();
      }
      if (t + AHEAD + grp < n) stage(t + AHEAD + grp);
      softmax(keys_of(t));
      if (grp == 0) {
        wait_next(t + AHEAD);
        __syncthreads();
      }
      mfma_phase(t + 1, yes, yes);
      trim(t + 1);
    }
    // the last position: nothing is left to request, and no scores follow
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (grp == 1) __syncthreads();
    softmax(keys_of(n - 1));
    if (grp == 0) __syncthreads();
    mfma_phase(n, yes, no);
  } else {   // no query of this wave exists: it only stages and converts
    convert(0, yes, keys_of(0));
#pragma unroll 1
    for (int t = 0; t < n; ++t) {
      if (grp == 0 && t + AHEAD < n) stage(t + AHEAD);
      wait_next(t + AHEAD);
      __syncthreads();
      if (grp == 1 && t + AHEAD + 1 < n) stage(t + AHEAD + 1);
      if (t + 1 < n) convert(t + 1, yes, keys_of(t + 1));
    }
  }

  // ---- lane n + 32 hh holds dims 32 db + 8 g + 4 hh .. + 4 of its query
  const int end_lane = PAIR ? static_cast<int>(lane_anew()) : lane, half = end_lane >> 5;
  const float l_tot = pair_sum(l_run);
  const int row = wave * 32 + (end_lane & 31), ql = qt * BQ + row;
  if (slot < 0) {
    const float inv = 1.0f / l_tot;
    if (ql < S.q_len) {
      bf16_t* op = a.o + static_cast<size_t>(S.q_off + ql) * a.ldo + h * HD;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          uint2 w;
          w.x = pack_bf16x2(o[db][4 * g] * inv, o[db][4 * g + 1] * inv);
          w.y = pack_bf16x2(o[db][4 * g + 2] * inv, o[db][4 * g + 3] * inv);
          *reinterpret_cast<uint2*>(op + 32 * db + 8 * g + 4 * half) = w;
        }
    }
  } else {
    float* po = a.part_o + (static_cast<size_t>(slot) * BQ + row) * HD;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<float4*>(po + 32 * db + 8 * g + 4 * half) =
            make_float4(o[db][4 * g], o[db][4 * g + 1], o[db][4 * g + 2], o[db][4 * g + 3]);
    if (half == 0) {
      a.part_ml[static_cast<size_t>(slot) * 2 * BQ + row] = m_run;
      a.part_ml[static_cast<size_t>(slot) * 2 * BQ + BQ + row] = l_tot;
    }
    __syncthreads();   // a following range reuses the tiles
  }
}

__device__ __forceinline__ int item_stream(const AttnArgs& a, int item) {
  int si = 0;
  for (int i = 1; i < a.n_streams; ++i)
    if (item >= a.s[i].item_begin) si = i;
  return si;
}

// One workgroup per item, each XCD a contiguous range of them.  PAIR: two on a CU, in 128
// registers (some offsets are formed anew instead of kept, which takes 2% where a CU has
// one workgroup).
template <int HD, int BITS, bool PAIR>
__global__ __launch_bounds__(NTHR, PAIR ? 4 : 2) void attn_mx_kernel(const MxLargeArgs x) {
  __shared__ __attribute__((aligned(1024))) LargeLds<HD, BITS> lds;
  const AttnArgs& a = x.a;
  const int xcd = blockIdx.x % kNumXcd;
  const int L = a.xcd_begin[xcd] + blockIdx.x / kNumXcd;
  if (L >= a.xcd_begin[xcd + 1]) return;
  const AttnStream S = a.s[item_stream(a, L)];
  const int it = L - S.item_begin, h = it / S.n_qtiles;
  mx_range<HD, BITS, PAIR>(a, x.p, S, h, it - h * S.n_qtiles, 0, S.n_tiles, lds, -1);
}

// The split schedule of plan_attention: main parts of the items from item0 on, then
// equal ranges of their concatenated tails (slots as attn_merge_kernel reads them).
template <int HD, int BITS>
__global__ __launch_bounds__(NTHR, 1) void attn_mx_split_kernel(const MxLargeArgs x) {
  __shared__ __attribute__((aligned(1024))) LargeLds<HD, BITS> lds;
  const AttnArgs& a = x.a;
  const int xcd = blockIdx.x % kNumXcd, j = blockIdx.x / kNumXcd;
  const int items = a.total_items - a.item0;
  const int ipx = items / kNumXcd, irem = items % kNumXcd;
  const int nx = ipx + (xcd < irem ? 1 : 0), pre = xcd * ipx + min(xcd, irem);
  if (j < nx) {
    const int gi = a.item0 + pre + j;
    const AttnStream S = a.s[item_stream(a, gi)];
    const int item = gi - S.item_begin, h = item / S.n_qtiles;
    mx_range<HD, BITS, false>(a, x.p, S, h, item - h * S.n_qtiles, 0, S.main_tiles, lds,
                       S.main_tiles == S.n_tiles ? -1 : gi - a.item0);
    return;
  }
  const int r = a.per_xcd * xcd + j - (pre + nx);
  if (r >= a.split_blocks - items) return;
  int pos = r * a.split_tiles;
  const int end = min(pos + a.split_tiles, a.total_tiles);
  while (pos < end) {
    int si = 0;
    for (int i = 1; i < a.n_streams; ++i)
      if (pos >= a.s[i].tail_begin) si = i;
    const AttnStream S = a.s[si];
    const int tl = S.n_tiles - S.main_tiles, rel = pos - S.tail_begin;
    const int item = max(0, a.item0 - S.item_begin) + rel / tl;
    const int tb = S.main_tiles + rel % tl, te = min(S.n_tiles, tb + (end - pos));
    pos += te - tb;
    const int h = item / S.n_qtiles;
    mx_range<HD, BITS, false>(a, x.p, S, h, item - h * S.n_qtiles, tb, te, lds,
                       static_cast<int64_t>(items) + S.item_begin + item - a.item0 + r);
  }
}

constexpr size_t kMoreThanHalf = 82 * 1024;   // of a CU's 160 KB of LDS: room for one workgroup

// More items than CUs run in pairs at d = 64, unless they end sooner alone (plan_attention's
// estimate).  us alone and in pairs: streams of 1560 and 4680 queries over 6240 and 18720
// keys, 20 heads, 638 / 551 (4 bits 634 / 537); 4680 over 37440, 40 heads, 1937 / 1756; 4608
// over 32256, 32 heads, 1242 / 1143; two streams of 4608 over 32256 and 13824, 8 heads, 522 /
// 630, which the rule would leave alone (the few rows' kernel has them, see below).
template <int HD, int BITS>
hipError_t launch_items(hipStream_t st, const MxLargeArgs& x, int grid, int items) {
  size_t more = 0;
  if constexpr (HD == 64) {
    if (items > kAttnSplitBlocks && !x.a.alone) {
      hipLaunchKernelGGL((attn_mx_kernel<HD, BITS, true>), dim3(grid), dim3(NTHR), 0, st, x);
      return hipGetLastError();
    }
    if (x.a.alone) more = kMoreThanHalf - sizeof(LargeLds<HD, BITS>);
  }
  hipLaunchKernelGGL((attn_mx_kernel<HD, BITS, false>), dim3(grid), dim3(NTHR), more, st, x);
  return hipGetLastError();
}

template <int HD, int BITS>
hipError_t launch_large(hipStream_t st, const MxLargeArgs& x) {
  const AttnArgs& a = x.a;
  if (!a.split_blocks)
    return launch_items<HD, BITS>(st, x, a.per_xcd * kNumXcd, a.total_items);
  if (a.item0 > 0) {
    const hipError_t e = launch_items<HD, BITS>(st, x, a.item0, a.item0);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((attn_mx_split_kernel<HD, BITS>), dim3(a.per_xcd * kNumXcd), dim3(NTHR), 0, st, x);
  return launch_attention_merge(st, a, HD);
}

// A round of equal items that leaves fewer CUs idle than plan_attention splits for: each
// idle one takes the last tiles of k items, so many that it ends with the items; a piece
// costs it `piece` 128ths of a tile more, all of them the merge (plan_attention's figures).
// Taken where the tiles say 6% or more: the clock falls as more CUs are busy, and it gains
// half of that or less.  us whole and so: d = 128, 8 heads of 6240 queries (200 items, 319
// tiles) 490 / 434, 11 of 4680 (209, 299) 449 / 434, 12 (228, 524) 796 / 792; d = 64, 12
// heads (228, 524) 555 / 526.  Not taken: 12 heads of 128 (228, 299; 4%) 461 / 465 to 482 /
// 470 by the values held, 13 (247, 524) 830 / 847.
void shed_tails(AttnArgs& a, int head_dim, float* part) {
  const int items = a.total_items, spare = kAttnSplitBlocks - items, n = a.s[0].n_tiles;
  if (a.split_blocks || spare <= 0 || a.s[a.n_streams - 1].n_tiles != n) return;
  const bool wide = head_dim == 128;
  const int64_t piece = wide ? 640 : 320, k = (items + spare - 1) / spare;
  const int64_t W = (k * (128 * static_cast<int64_t>(n) + piece) + 128 * (k + 1) - 1) / (128 * (k + 1));
  const int64_t tl = n - W;
  if (tl <= 0 || 128 * W + (wide ? 640 + 4 * items : 384 + 6 * items) >= 120 * static_cast<int64_t>(n)) return;
  if (spare * k * tl > INT32_MAX) return;   // (the kernel counts the tails' tiles in 32 bits)
  int64_t tails = 0;
  for (int i = 0; i < a.n_streams; ++i) {
    a.s[i].main_tiles = static_cast<int32_t>(W);
    a.s[i].tail_begin = static_cast<int32_t>(tails);
    tails += a.s[i].n_qtiles * a.H * tl;
  }
  a.item0 = 0;
  a.split_blocks = kAttnSplitBlocks;
  a.split_tiles = static_cast<int32_t>(k * tl);
  a.total_tiles = static_cast<int32_t>(tails);
  a.part_o = part;
  a.part_ml = part + static_cast<size_t>(2) * kAttnSplitBlocks * BQ * head_dim;
  a.per_xcd = kAttnSplitBlocks / kNumXcd;
}

hipError_t run_large(hipStream_t st, const MxPages& p, const bf16_t* q, bf16_t* o, const RowStreams& rs, int rows_over,
                     float* part) {
  MxLargeArgs x;
  memset(&x, 0, sizeof(x));
  x.p = p;
  AttnArgs& a = x.a;
  a.q = q;
  a.o = o;
  a.ldq = a.ldo = p.H * p.hd;
  a.H = p.H;
  a.scale_log2 = static_cast<float>(1.4426950408889634 / sqrt(static_cast<double>(p.hd)));
  for (int i = 0; i < rs.n; ++i) {
    if (rs.s[i].len <= rows_over) continue;
    AttnStream& s = a.s[a.n_streams++];
    s.q_off = rs.s[i].row_begin;
    s.q_len = rs.s[i].len;
    s.stream = i;
    s.base_off = rs.s[i].cache_len + rs.s[i].len;
    s.kv_len = static_cast<int32_t>(kAttnKTile * mx_tiles(s.base_off, p.T, p.nt));   // as planned: whole tiles
  }
  plan_attention(a, p.hd, part, false);
  shed_tails(a, p.hd, part);
  if (p.hd == 128) return p.bits == 8 ? launch_large<128, 8>(st, x) : launch_large<128, 4>(st, x);
  return p.bits == 8 ? launch_large<64, 8>(st, x) : launch_large<64, 4>(st, x);
}

template <int HD, int BITS>
hipError_t launch_small(hipStream_t st, const MxSmallArgs& a) {
  const MxRun& end = a.run[a.n_runs];
  const int per_xcd = end.eighths + (end.rest + kNumXcd - 1) / kNumXcd;
  hipLaunchKernelGGL((attn_mx_small_kernel<HD, BITS>), dim3(per_xcd * kNumXcd), dim3(64 * SM_WAVES), 0, st, a);
  if (a.join_rows) {
    const int per = 256 / (HD / 4) / a.groups;   // rows of a workgroup
    hipLaunchKernelGGL((attn_mx_join_kernel<HD>), dim3((a.join_rows * a.p.H + per - 1) / per), dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

constexpr int kSmallRound = 256;   // workgroups of one round: one to a CU
// A workgroup's start and end, in tiles of a wave; and the join's launch, and the partial
// rows that it takes as long for as for one, in half tiles.
constexpr int kSmallStart = 3, kSmallJoin = 5, kSmallRows = 4096;
// Most rows and tiles of a solo span.  32 continuations of one history, half of them with
// a frame of their own: 69 us with a workgroup for each, 50 up to 16 tiles, 39 up to 32 or
// 64.  With more rows a wave would write more partial results than it saves (12 and 24, six
// spans of 10 heads of 64, lost 10% to a workgroup when they were joined one by one).
constexpr int kSoloRows = 8, kSoloTiles = 32;

// Cuts the spans' key tiles: the length of a cut with the earliest estimated end among
// a few, such that the partial rows fit max_rows.  Returns that end, in half tiles of a
// wave.  us with one round or more, and the join left out of the estimate, and so: seven
// streams of one token over 32760 keys, 40 heads of 128, 538 / 450; eight tokens over 9 to
// 21 frames, 20 heads of 64, 102 / 94; 192 rows over 6 small frames, 4 heads, 11.7 / 8.
int64_t plan_small(MxSmallArgs& a, int64_t max_rows) {
  // solo spans last: those of one row tile and few key tiles
  auto is_solo = [](const MxSpan& s) { return s.q_len <= kSoloRows && s.tile1 - s.tile0 <= kSoloTiles; };
  MxSpan tmp[kMaxStreams];
  int n_solo = 0, n = a.shared;
  for (int i = a.shared; i < a.n_spans; ++i) {
    if (is_solo(a.s[i])) tmp[n_solo++] = a.s[i];
    else a.s[n++] = a.s[i];
  }
  a.solo_span = n;
  for (int i = 0; i < n_solo; ++i) a.s[n + i] = tmp[i];

  int64_t cost = 0;
  int most = 1;
  for (int i = 0; i < a.n_spans; ++i) {
    MxSpan& s = a.s[i];
    s.n_qtiles = (s.q_len + SM_BQ - 1) / SM_BQ;
    cost += static_cast<int64_t>(s.n_qtiles) * a.p.H * (s.tile1 - s.tile0);
    most = std::max(most, s.tile1 - s.tile0);
  }
  // Cuts of w tiles, of solo spans of a wave's share of them.
  auto cut = [&](const MxSpan& s, int i, int w) {
    const int tiles = s.tile1 - s.tile0;
    const int each = i < a.solo_span ? w : std::max(1, (w + SM_WAVES - 1) / SM_WAVES);
    return std::max(1, (tiles + each - 1) / each);
  };
  // In half tiles of a wave.  The longest workgroups come first: those of a run and of the
  // longer ones take as many rounds as they fill, and what is shorter evens the end out.
  // Partial rows are written, read and joined in a launch of its own.
  auto end = [&](int w) {
    int64_t rows = 0, sum = 0, solo = 0, items = 0;
    int solo_longest = 0, n = 0;
    struct Group {
      int one;
      int64_t wgs;
    } g[kMaxStreams + 1];
    for (int i = 0; i < a.n_spans; ++i) {
      const MxSpan& s = a.s[i];
      const int pieces = cut(s, i, w), each = (s.tile1 - s.tile0 + pieces - 1) / pieces;
      const int64_t c = static_cast<int64_t>(s.n_qtiles) * a.p.H * pieces;
      if (i < a.solo_span) {
        g[n++] = {kSmallStart + (each + SM_WAVES - 1) / SM_WAVES, c};
      } else {
        solo += c;
        solo_longest = std::max(solo_longest, kSmallStart + each);
      }
      if (pieces > 1 || a.shared) rows += static_cast<int64_t>(s.q_len) * pieces * a.p.H;
    }
    if (rows > max_rows) return INT64_MAX;
    if (solo) g[n++] = {solo_longest, (solo + SM_WAVES - 1) / SM_WAVES};
    std::sort(g, g + n, [](const Group& x, const Group& y) { return x.one > y.one; });
    int64_t last = 0;
    for (int i = 0; i < n; ++i) {
      items += g[i].wgs;
      sum += g[i].wgs * g[i].one;
      last = std::max(last, 2 * ((items + kSmallRound - 1) / kSmallRound) * g[i].one);
    }
    if (items > kSmallRound) last = std::max(last, 2 * sum / kSmallRound + g[n - 1].one / 2);
    return last + (rows ? kSmallJoin + rows / kSmallRows : 0);
  };
  // candidates: no span cut, and the shortest cuts whose workgroups fill so many rounds
  const int whole = std::max(most, SM_WAVES * std::min(most, kSoloTiles));
  int W = whole;
  int64_t best = end(whole);
  for (const int rounds : {1, 2, 3, 4, 6, 8}) {
    auto fits = [&](int w) {
      int64_t items = 0, solo = 0;
      for (int i = 0; i < a.n_spans; ++i) {
        const int64_t c = static_cast<int64_t>(a.s[i].n_qtiles) * a.p.H * cut(a.s[i], i, w);
        if (i < a.solo_span) items += c;
        else solo += c;
      }
      return items + (solo + SM_WAVES - 1) / SM_WAVES <= rounds * kSmallRound;
    };
    // (a share of all tiles may pass the longest span, and 32 bits)
    int w = static_cast<int>(std::clamp<int64_t>(cost / (rounds * kSmallRound), SM_WAVES, whole));
    while (w < whole && !fits(w)) w += std::max(1, w / 16);
    if (w >= whole) continue;
    const int64_t e = end(w);
    if (e < best) {
      best = e;
      W = w;
    }
    if (w == SM_WAVES || 4 * e > 5 * best) break;   // (shorter cuts will not do)
  }
  a.join_rows = 0;
  int64_t rows = 0, solo = 0;
  int solo_longest = 0;
  struct Run {
    int span, cost;   // cost of a workgroup
    int64_t wgs;
  } runs[kMaxStreams + 1];
  a.n_runs = 0;
  for (int i = 0; i < a.n_spans; ++i) {
    MxSpan& s = a.s[i];
    const int tiles = s.tile1 - s.tile0;
    s.pieces = cut(s, i, W);
    s.per_piece = (tiles + s.pieces - 1) / s.pieces;
    const int64_t cuts = static_cast<int64_t>(s.n_qtiles) * a.p.H * s.pieces;
    s.wave_begin = static_cast<int32_t>(solo);
    if (i < a.solo_span) {
      runs[a.n_runs++] = {i, kSmallStart + (s.per_piece + SM_WAVES - 1) / SM_WAVES, cuts};
    } else {
      solo += cuts;
      solo_longest = std::max(solo_longest, kSmallStart + s.per_piece);
    }
    s.part_begin = -1;
    if (s.pieces > 1 || a.shared) {
      s.part_begin = static_cast<int32_t>(rows);
      rows += static_cast<int64_t>(a.p.H) * s.pieces * s.q_len;
      s.join_begin = a.join_rows;
      if (i >= a.shared) a.join_rows += s.q_len;
    }
  }
  if (solo) runs[a.n_runs++] = {a.solo_span, solo_longest, (solo + SM_WAVES - 1) / SM_WAVES};
  a.solo_waves = static_cast<int32_t>(solo);
  // Every XCD takes an eighth of each run in one piece (row tiles of the same keys meet in
  // its L2), the longest workgroups first.  (In the batch's order, and each XCD a range of
  // all: streams of 17, 192, 1, 700 and 65 rows over 62 to 404 tiles, 10 heads of 64, 54 us
  // for 46; 32 continuations of one history 39 for 37.)
  std::stable_sort(runs, runs + a.n_runs, [](const Run& x, const Run& y) { return x.cost > y.cost; });
  a.run[0] = {0, 0};
  for (int e = 0; e < a.n_runs; ++e) {
    a.run_span[e] = static_cast<uint8_t>(runs[e].span);
    a.run[e + 1].eighths = a.run[e].eighths + static_cast<int32_t>(runs[e].wgs / kNumXcd);
    a.run[e + 1].rest = a.run[e].rest + static_cast<int32_t>(runs[e].wgs % kNumXcd);
  }
  // groups of the join's lanes: four cuts each, of the row with most
  int cuts = 1;
  for (int i = a.shared; i < a.n_spans; ++i) cuts = std::max(cuts, a.s[i].pieces + (a.shared ? a.s[0].pieces : 0));
  const int lanes = a.p.hd / 4;
  a.groups = kWave / lanes;
  while (a.groups < 256 / lanes && 4 * a.groups < cuts) a.groups *= 2;
  return best;
}

}  // namespace

// Spans of the streams with at most rows_most rows, planned; the estimated end in
// hundredths of a microsecond.
static int64_t plan_few(MxSmallArgs& a, const RowStreams& rs, int rows_most, int shared, int64_t max_rows) {
  const MxPages& p = a.p;
  int first = -1;
  a.n_spans = 0;
  a.shared = shared > 0;
  for (int i = 0; i < rs.n && first < 0; ++i)
    if (rs.s[i].len > 0) first = i;
  const int32_t tile0 = shared * p.nt;
  if (a.shared) {
    MxSpan& s = a.s[a.n_spans++];
    s.q_off = 0;
    s.q_len = a.rows;
    s.kv_len = shared * p.T;
    s.row = first;
    s.tile0 = 0;
    s.tile1 = tile0;
  }
  for (int i = 0; i < rs.n; ++i) {
    if (rs.s[i].len == 0 || rs.s[i].len > rows_most) continue;
    MxSpan& s = a.s[a.n_spans++];
    s.q_off = rs.s[i].row_begin;
    s.q_len = rs.s[i].len;
    s.kv_len = rs.s[i].cache_len + rs.s[i].len;
    s.row = i;
    s.tile0 = tile0;
    s.tile1 = static_cast<int32_t>(mx_tiles(s.kv_len, p.T, p.nt));
  }
  const int64_t end = plan_small(a, max_rows);
  return p.hd == 128 ? 730 + 79 * end : 725 + 57 * end;
}

// The estimated end of whole-chunk items of the streams with more rows, likewise.
static int64_t estimate_many(const MxPages& p, const RowStreams& rs, int rows_over) {
  int64_t items = 0, work = 0, most = 0;
  for (int i = 0; i < rs.n; ++i) {
    if (rs.s[i].len <= rows_over) continue;
    const int64_t tiles = mx_tiles(static_cast<int64_t>(rs.s[i].cache_len) + rs.s[i].len, p.T, p.nt);
    const int64_t n = static_cast<int64_t>((rs.s[i].len + BQ - 1) / BQ) * p.H;
    items += n;
    work += n * tiles;
    most = std::max(most, tiles);
  }
  // (a round that the items leave idle is split; whole items go in rounds)
  const int64_t tiles = items < 3 * kSmallRound / 4 ? work / kSmallRound : std::max(most, work / kSmallRound);
  return p.hd == 128 ? 3250 + 136 * tiles : 2490 + 100 * tiles;
}

// Which kernel takes a stream goes by estimates fitted to 468 calls (1 to 10 streams of
// 20 to 768 rows over 1 to 21 frames of 1560 tokens, 4, 12 and 40 heads of 64 and 128,
// both formats), each timed on both.  The choice loses 0.5% to the better one on average,
// 26% at most (three streams of 300 rows over one frame, 40 heads of 128, 78 us for 62).
// Streams of 780 to 4680 rows in 36 calls that it gives to the few rows' kernel: from half
// the time of whole-chunk items (3120 rows over 3 frames beside 780 over 18, 16 heads of 128,
// 357 / 646) to 14% more (4680 over 21 and 780 over 22, 10 heads of 64, 650 / 568), 2% lost
// on average.
// us of the few rows' kernel and of whole-chunk items, 12 heads of 128 over 32760 tokens:
// 64 rows 31 / 63, 192 56 / 77, 256 74 / 80, 768 209 / 157; four streams of 192 over 14040
// 111 / 94.
hipError_t launch_attention_mx(hipStream_t st, const MxPages& p, const bf16_t* q, bf16_t* o,
                               const RowStreams& rs, int shared, float* part) {
  MxSmallArgs a;
  a.p = p;
  a.q = q;
  a.o = o;
  a.ld = p.H * p.hd;
  a.scale_log2 = static_cast<float>(1.4426950408889634 / sqrt(static_cast<double>(p.hd)));
  a.rows = 0;
  int row_tiles = 0, longest = 0;
  for (int i = 0; i < rs.n; ++i) {
    a.rows += rs.s[i].len;
    row_tiles += (rs.s[i].len + SM_BQ - 1) / SM_BQ;
    longest = std::max(longest, rs.s[i].len);
  }
  if (a.rows == 0) return hipSuccess;
  const int64_t max_rows = static_cast<int64_t>(attention_split_bytes(p.hd) / (sizeof(float) * (p.hd + 2)));
  a.part_o = part;
  a.part_ml = reinterpret_cast<float2*>(part + max_rows * p.hd);
  // The prefix is walked once for all rows where that makes fewer row tiles.
  const bool once = shared > 0 && (a.rows + SM_BQ - 1) / SM_BQ < row_tiles &&
                    static_cast<int64_t>(2) * p.H * a.rows <= max_rows;
  constexpr int kAll = INT32_MAX, kFew = 128;
  int few = kAll;                 // streams of at most this many rows take the few rows' kernel
  const int64_t end = plan_few(a, rs, kAll, once ? shared : 0, max_rows);
  if (longest > SM_BQ) {
    const int64_t many = estimate_many(p, rs, 0);
    if (many < end) few = 0;
    if (longest > kFew) {         // the long streams alone to the other kernel, in a launch before
      MxSmallArgs b = a;
      const int64_t both = plan_few(b, rs, kFew, 0, max_rows) + estimate_many(p, rs, kFew);
      if (b.n_spans > 0 && both < std::min(end, many)) {
        few = kFew;
        a = b;
      }
    }
  }
  if (few != kAll) {
    const hipError_t e = run_large(st, p, q, o, rs, few, part);
    if (e != hipSuccess || few == 0) return e;
  }
  if (p.hd == 128) return p.bits == 8 ? launch_small<128, 8>(st, a) : launch_small<128, 4>(st, a);
  return p.bits == 8 ? launch_small<64, 8>(st, a) : launch_small<64, 4>(st, a);
}

}  // namespace ardit
