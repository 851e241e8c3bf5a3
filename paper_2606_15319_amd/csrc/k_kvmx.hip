// Microscaled key/value pages: a chunk's keys and values quantised as they are
// appended, and pages read back in bf16.
//
// Both move bytes and little else.  An append reads the projections (6 bytes a
// token and dim) and writes the rotated queries (2) and the codes (2 or 1, and
// 1/16 of scales); a read-back reads codes and scales and writes 4.
#include <math.h>

#include <algorithm>

#include "mx.h"

namespace ardit {

namespace {

struct AppendArgs {
  const bf16_t* qkv;
  bf16_t* q_out;
  const bf16_t* g_q;
  const bf16_t* g_k;
  MxPages p;
  int N, D, lat_w;
  int qk_groups, v_tiles;     // workgroups of the rows, and of the value tiles of one head
  FastDiv fT, fW, fnt, fvt;
  float eps;
  int pairs_t, pairs_h;       // pair-index boundaries of the frame and row segments
  double inv_freq[64];        // theta^(-2k/seg) of every pair of a head, in turns (/ 2 pi)
  RowStreams rs;
};
static_assert(sizeof(AppendArgs) <= 4096, "arguments must fit the kernel-argument buffer");

__device__ __forceinline__ int stream_of(const RowStreams& rs, int row) {
  int b = 0;
  for (int i = 1; i < rs.n; ++i)
    if (row >= rs.s[i].row_begin) b = i;
  return b;
}

// -1 for an entry outside the pool: the store is skipped, so a bad table can
// never write into a page another stream owns
__device__ __forceinline__ int write_page(int p, int n_pages) { return p >= 0 && p < n_pages ? p : -1; }

__device__ __forceinline__ void store_stream16(void* p, const uint4& v) {
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), reinterpret_cast<u32x4*>(p));
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m, kWave);
  return v;
}

__device__ __forceinline__ uint32_t quad_max(uint32_t m) {   // over 4 neighbouring lanes
  m = max(m, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(m), 0xB1, 0xf, 0xf, true)));
  return max(m, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(m), 0x4E, 0xf, 0xf, true)));
}

// fp64 to fp32 such that a rounding to fewer bits gives what it gives for x itself: the low
// half of x is cut off and, where it held anything, the last bit that stays is set.  (21
// bits stay, exact in fp32 down to 2^-129.)
__device__ __forceinline__ float to_odd(double x) {
  return static_cast<float>(__hiloint2double(__double2hiint(x) | static_cast<int>(min(static_cast<uint32_t>(__double2loint(x)), 1u)), 0));
}

constexpr uint32_t kSmallKey = 67u << 23;   // bits of 2^-60

// Queries and keys of RPW rows a wave.  Keys are normed and rotated in fp64 up to their
// codes: a code's step is up to an eighth of its value, and with fp32's last bits in doubt 25
// of sixteen million keys lie close enough to the border of two codes to take the farther
// one.  Rounded to fp32 first, a key within 2^-25 of a border would come to lie on it, and 8
// do so and go the wrong way: but all borders end in 19 zero bits, so the lanes that see
// such a key, one in 2^16, form theirs again by to_odd (9360 rows of 5120, E4M3, 104 us for
// 103; all keys by to_odd 112).  Rows of more than 1024 dims go one to a wave and wider ones
// to two or four waves, so that a lane holds three or four pieces: fewer registers, more
// rows under way (with their read-back, 4680 rows of 1536 29 us for 32 with two rows a wave,
// 9360 of 5120 169 for 186 with a wave each).  A lane holds chunks lane + 64 (part + WPR i)
// of 8 dims of a row, so a block of 32 dims is four neighbouring lanes and a head 16 or 8
// of them.
template <int MAXC, int RPW, int WPR, int BITS>
__device__ __forceinline__ void append_rows(const AppendArgs& a, int group, float* lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int set = wave / WPR, part = wave % WPR;   // WPR waves hold the rows of a set
  const int row0 = (group * (4 / WPR) + set) * RPW;
  const int nchunk = a.D >> 3, hd = a.p.hd, lane0 = lane + 64 * part;
  double* lcs = reinterpret_cast<double*>(lds) + set * RPW * 128;   // cos and sin of each row's pairs
  __shared__ double part_sk[4][RPW];
  __shared__ float part_sq[4][RPW];

  uint4 qraw[RPW][MAXC], kraw[RPW][MAXC];
#pragma unroll
  for (int r = 0; r < RPW; ++r) {
    const uint4* qr = reinterpret_cast<const uint4*>(a.qkv + static_cast<size_t>(min(row0 + r, a.N - 1)) * 3 * a.D);
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
      const int c = lane0 + 64 * WPR * i;
      if (c < nchunk) {
        qraw[r][i] = qr[c];
        kraw[r][i] = qr[nchunk + c];
      }
    }
  }
#pragma unroll
  for (int r = 0; r < RPW; ++r) {
    if (WPR > 1 && r % WPR != part) continue;
    const int row = min(row0 + r, a.N - 1);
    const RowStream s = a.rs.s[stream_of(a.rs, row)];
    const int t = row - s.row_begin;
    const int f = static_cast<int>(fdiv(static_cast<uint32_t>(t), a.fT));
    const int rem = t - f * a.p.T;
    const int i = static_cast<int>(fdiv(static_cast<uint32_t>(rem), a.fW));
    const int j = rem - i * a.lat_w;
    double cs = 1.0, sn = 0.0;
    if (lane < (hd >> 1)) {
      // angles in turns
      const int pos = lane < a.pairs_t ? s.frame_pos0 + f : (lane < a.pairs_t + a.pairs_h ? i : j);
      double x = static_cast<double>(pos) * a.inv_freq[lane];
      x -= rint(x);
      sincospi(2.0 * x, &sn, &cs);
    }
    lcs[r * 128 + lane] = cs;
    lcs[r * 128 + 64 + lane] = sn;
  }
#pragma unroll
  for (int r = 0; r < RPW; ++r) {
    float sq = 0.f;
    double sk = 0.0;
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
      if (lane0 + 64 * WPR * i < nchunk) {
        float x[8], y[8];
        unpack8(qraw[r][i], x);
        unpack8(kraw[r][i], y);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          sq += x[e] * x[e];
          sk = fma(static_cast<double>(y[e]), static_cast<double>(y[e]), sk);
        }
      }
    }
    sq = wave_sum(sq);
    sk = wave_sum64(sk);
    if (lane == 0) {
      part_sq[wave][r] = sq;
      part_sk[wave][r] = sk;
    }
  }
  // (a wave's own rows need no barrier: its LDS operations stay in order, the fence
  // keeps the compiler from moving them)
  if constexpr (WPR > 1) __syncthreads();
  else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");

#pragma unroll
  for (int r = 0; r < RPW; ++r) {
    const int row = row0 + r;
    float sq = 0.f;
    double sk = 0.0;
#pragma unroll
    for (int w = 0; w < WPR; ++w) {
      sq += part_sq[set * WPR + w][r];
      sk += part_sk[set * WPR + w][r];
    }
    if (row >= a.N) continue;
    const float rq = 1.0f / sqrtf(sq / static_cast<float>(a.D) + a.eps);
    const double rk = 1.0 / sqrt(sk / static_cast<double>(a.D) + static_cast<double>(a.eps));
    const int b = stream_of(a.rs, row);
    const RowStream s = a.rs.s[b];
    const int slot = s.cache_len + row - s.row_begin;
    const int fr = static_cast<int>(fdiv(static_cast<uint32_t>(slot), a.fT));
    const int page = write_page(a.p.page_table[static_cast<size_t>(b) * a.p.max_frames + fr], a.p.n_pages);
    const int off = slot - fr * a.p.T;
    const double* rcs = lcs + r * 128;
    uint4* qo = reinterpret_cast<uint4*>(a.q_out + static_cast<size_t>(row) * a.D);
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
      const int c = lane0 + 64 * WPR * i;
      if (c < nchunk) {
        const int e0 = (8 * c) & (hd - 1);
        const int h = (8 * c) / hd;
        double cc[4], ss[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          cc[e] = rcs[(e0 >> 1) + e];
          ss[e] = rcs[64 + (e0 >> 1) + e];
        }
        float x[8], y[8], g[8];
        unpack8(reinterpret_cast<const uint4*>(a.g_q)[c], g);
        unpack8(qraw[r][i], x);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x0 = x[2 * e] * rq * g[2 * e], x1 = x[2 * e + 1] * rq * g[2 * e + 1];
          const float co = static_cast<float>(cc[e]), si = static_cast<float>(ss[e]);
          y[2 * e] = x0 * co - x1 * si;
          y[2 * e + 1] = x0 * si + x1 * co;
        }
        store_stream16(qo + c, pack8(y));
        unpack8(reinterpret_cast<const uint4*>(a.g_k)[c], g);
        unpack8(kraw[r][i], x);
        // largest of the lane's keys; least of their last 19 bits
        uint32_t m, low;
        auto turn = [&](auto wide, auto to_fp32) {
          m = 0;
          low = ~0u;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            using P = decltype(wide);
            if constexpr (sizeof(P) == 8) __builtin_amdgcn_sched_barrier(0);   // (one pair's registers at a time)
            const double x0 = static_cast<P>(x[2 * e]) * static_cast<P>(g[2 * e]);
            const double x1 = static_cast<P>(x[2 * e + 1]) * static_cast<P>(g[2 * e + 1]);
            y[2 * e] = to_fp32(rk * fma(x0, cc[e], -x1 * ss[e]));
            y[2 * e + 1] = to_fp32(rk * fma(x0, ss[e], x1 * cc[e]));
            const uint32_t u0 = __float_as_uint(y[2 * e]), u1 = __float_as_uint(y[2 * e + 1]);
            m = max(m, max(u0 & 0x7fffffffu, u1 & 0x7fffffffu));
            low = min(low, min(u0 & 0x7ffffu, u1 & 0x7ffffu));
          }
        };
        // A product of two bf16 numbers is exact in fp32 between its ends: past the upper one a
        // key is an infinity or NaN, which end in 19 zero bits too; below the lower one what is lost,
        // 2^-150 rk, is nothing to keys of 2^-60 and more.
        turn(0.0f, [](double v) { return static_cast<float>(v); });
        if (low == 0 || m < kSmallKey || rk > 1024.0) {   // (on a border: maybe next to it)
          uint4 k = kraw[r][i];
          int again = c;   // (formed anew, so that nothing is held for the few that come here)
          asm volatile("" : "+v"(k.x), "+v"(k.y), "+v"(k.z), "+v"(k.w), "+v"(again));
          unpack8(reinterpret_cast<const uint4*>(a.g_k)[again], g);
          unpack8(k, x);
          turn(0.0, to_odd);
        }
        const int sb = mx_scale_byte<BITS>(quad_max(m));
        const uint2 w = mx_encode8<BITS>(y, mx_inverse(sb));
        // the scale bytes of a head meet in its first lane (a lane's own byte is that of
        // its four neighbours)
        uint32_t sc = static_cast<uint32_t>(sb) << (8 * ((e0 >> 5) & 3));
        if (hd == 128) {
          sc |= static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(sc), 0x124, 0xf, 0xf, true));   // row_ror:4
          sc |= static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(sc), 0x128, 0xf, 0xf, true));   // row_ror:8
        } else {
          sc |= static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(sc), 0x141, 0xf, 0xf, true));   // row_half_mirror
        }
        if (page >= 0) {
          const size_t key = mx_tile(a.p, page, h, 0) * 64 + off;
          uint8_t* kd = a.p.k + (key * hd + e0) * BITS / 8;
          if constexpr (BITS == 8) *reinterpret_cast<uint2*>(kd) = w;
          else *reinterpret_cast<uint32_t*>(kd) = w.x;
          if (e0 == 0) {
            if (hd == 128) *reinterpret_cast<uint32_t*>(a.p.ks + key * 4) = sc;
            else *reinterpret_cast<uint16_t*>(a.p.ks + key * 2) = static_cast<uint16_t>(sc);
          }
        }
      }
    }
  }
}

// One tile of 64 keys of one head's values: rows staged in LDS, then a thread takes
// 16 keys of two neighbouring dims; the lane 32 on holds the block's other 16 keys.
// Keys past the page's end are written as zeros.
template <int BITS>
__device__ __forceinline__ void append_values(const AppendArgs& a, int w, uint32_t* tile) {
  const int hd = a.p.hd, tid = threadIdx.x;
  const int h = static_cast<int>(fdiv(static_cast<uint32_t>(w), a.fvt));
  const int vt = w - h * a.v_tiles;
  const int fg = static_cast<int>(fdiv(static_cast<uint32_t>(vt), a.fnt));   // frame of the batch
  const int ti = vt - fg * a.p.nt;
  const int row0 = fg * a.p.T + 64 * ti;
  const int n = min(64, a.p.T - 64 * ti);
  const int cpr = hd >> 3;
  for (int c = tid; c < 64 * cpr; c += 256) {
    const int r = c / cpr, cc = c - r * cpr;
    uint4 u = make_uint4(0u, 0u, 0u, 0u);
    if (r < n)
      u = *reinterpret_cast<const uint4*>(a.qkv + static_cast<size_t>(row0 + r) * 3 * a.D + 2 * a.D + h * hd + cc * 8);
    *reinterpret_cast<uint4*>(&tile[r * (hd / 2) + cc * 4]) = u;
  }
  __syncthreads();
  const int b = stream_of(a.rs, row0);
  const RowStream s = a.rs.s[b];
  const int fr = static_cast<int>(fdiv(static_cast<uint32_t>(s.cache_len + row0 - s.row_begin), a.fT));
  const int page = write_page(a.p.page_table[static_cast<size_t>(b) * a.p.max_frames + fr], a.p.n_pages);
  if (page < 0) return;
  const int lane = tid & 63, wave = tid >> 6;
  const int half = lane >> 5, kb = wave & 1, dp = (wave >> 1) * 32 + (lane & 31);
  if (2 * dp >= hd) return;
  const int kq = 2 * kb + half;   // 16 keys from 16 kq
  float f[2][16];
  uint32_t m[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t x = tile[(16 * kq + i) * (hd / 2) + dp];
    f[0][i] = __uint_as_float(x << 16);
    f[1][i] = __uint_as_float(x & 0xffff0000u);
    m[0] = max(m[0], __float_as_uint(f[0][i]) & 0x7fffffffu);
    m[1] = max(m[1], __float_as_uint(f[1][i]) & 0x7fffffffu);
  }
  const size_t t = mx_tile(a.p, page, h, ti);
  uint32_t sb[2];
#pragma unroll
  for (int d = 0; d < 2; ++d) {
    const auto sw = __builtin_amdgcn_permlane32_swap(m[d], m[d], false, false);
    sb[d] = static_cast<uint32_t>(mx_scale_byte<BITS>(max(static_cast<uint32_t>(sw[0]), static_cast<uint32_t>(sw[1]))));
    const float inv = mx_inverse(static_cast<int>(sb[d]));
    const uint2 w0 = mx_encode8<BITS>(f[d], inv), w1 = mx_encode8<BITS>(f[d] + 8, inv);
    uint8_t* vd = a.p.v + t * mx_tile_bytes(hd, BITS) + ((2 * dp + d) * 64 + 16 * kq) * BITS / 8;
    if constexpr (BITS == 8) *reinterpret_cast<uint4*>(vd) = make_uint4(w0.x, w0.y, w1.x, w1.y);
    else *reinterpret_cast<uint2*>(vd) = make_uint2(w0.x, w1.x);
  }
  if (half == 0)
    *reinterpret_cast<uint16_t*>(a.p.vs + t * mx_scale_bytes(hd) + kb * hd + 2 * dp) =
        static_cast<uint16_t>(sb[0] | (sb[1] << 8));
}

// Rows and value tiles in one launch, so the two run side by side.
template <int MAXC, int RPW, int WPR, int BITS>
__global__ __launch_bounds__(256) void kv_append_mx_kernel(const AppendArgs a) {
  __shared__ __attribute__((aligned(16))) uint32_t lds[64 * 64];
  const int b = blockIdx.x;
  if (b < a.qk_groups) {
    // each XCD takes a run of row groups, so that neighbouring tokens' scale words
    // (4 bytes each) meet in one L2
    const int per = (a.qk_groups + kNumXcd - 1) / kNumXcd;
    int g = b;
    if (a.qk_groups % kNumXcd == 0) g = (b % kNumXcd) * per + b / kNumXcd;
    append_rows<MAXC, RPW, WPR, BITS>(a, g, reinterpret_cast<float*>(lds));
  } else {
    append_values<BITS>(a, b - a.qk_groups, lds);
  }
}

struct ReadArgs {
  MxPages p;
  bf16_t* k;
  bf16_t* v;
  const int32_t* page_table;
  int max_frames, n_pages;
  int tiles, total;         // tiles of the streams, and of all heads
  FastDiv ftiles;
  RowStreams rs;            // row_begin: first tile of the stream, len and cache_len in tokens
};
static_assert(sizeof(ReadArgs) <= 4096, "arguments must fit the kernel-argument buffer");

// One tile of 64 keys of one head, 8 codes a thread and step, so that every store
// instruction of a wave writes whole runs of lines.
template <int HD, int BITS>
__global__ __launch_bounds__(256) void kv_read_mx_kernel(const ReadArgs a) {
  const MxPages& p = a.p;
  // each XCD takes a run of one head's tiles after the other: the values of neighbouring
  // tiles share lines of dst's transposed rows, which meet in one L2
  const int per = (a.total + kNumXcd - 1) / kNumXcd;
  const int L = static_cast<int>(blockIdx.x % kNumXcd) * per + static_cast<int>(blockIdx.x / kNumXcd);
  if (static_cast<int>(blockIdx.x / kNumXcd) >= per || L >= a.total) return;
  const int h = static_cast<int>(fdiv(static_cast<uint32_t>(L), a.ftiles));
  const int g = L - h * a.tiles;
  const int b = stream_of(a.rs, g);
  const RowStream s = a.rs.s[b];
  const int t = g - s.row_begin;                  // tile of the stream's range
  const int fo = static_cast<int>(fdiv(static_cast<uint32_t>(t), p.fnt));
  const int ti = t - fo * p.nt;
  const int n = min(min(64, p.T - 64 * ti), s.len - fo * p.T - 64 * ti);   // tokens of the tile
  const int fr = static_cast<int>(fdiv(static_cast<uint32_t>(s.cache_len), p.fT)) + fo;
  const int src = mx_read_page(p, b, fr);
  const int dst = write_page(a.page_table[static_cast<size_t>(b) * a.max_frames + fr], a.n_pages);
  if (dst < 0) return;
  const size_t tile = mx_tile(p, src, h, ti);
  constexpr int STEPS = HD / 32;                  // 64 HD values: 8 a thread and step
  const uint8_t* kc = p.k + tile * mx_tile_bytes(HD, BITS);
  const uint8_t* vc = p.v + tile * mx_tile_bytes(HD, BITS);
  uint2 kw[STEPS], vw[STEPS];
  uint32_t ksb[STEPS], vsb[STEPS];
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int c = threadIdx.x + 256 * i;
    if constexpr (BITS == 8) {
      kw[i] = *reinterpret_cast<const uint2*>(kc + c * 8);
      vw[i] = *reinterpret_cast<const uint2*>(vc + c * 8);
    } else {
      kw[i] = make_uint2(*reinterpret_cast<const uint32_t*>(kc + c * 4), 0u);
      vw[i] = make_uint2(*reinterpret_cast<const uint32_t*>(vc + c * 4), 0u);
    }
    ksb[i] = p.ks[tile * mx_scale_bytes(HD) + c / 4];                                 // 32 dims of a key: 4 threads
    vsb[i] = p.vs[tile * mx_scale_bytes(HD) + ((c & 7) >> 2) * HD + (c >> 3)];       // 32 keys of a dim
  }
  const size_t head = (static_cast<size_t>(dst) * p.H + h) * p.T * HD;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int c = threadIdx.x + 256 * i;
    const int key = c / (HD / 8), e0 = 8 * (c % (HD / 8));
    if (key < n)
      store_stream16(a.k + head + static_cast<size_t>(64 * ti + key) * HD + e0,
                     __builtin_bit_cast(uint4, mx_decode8<BITS>(kw[i].x, kw[i].y, mx_scale(ksb[i]))));
    const int dim = c >> 3, j0 = 8 * (c & 7);
    const u32x4 x = mx_decode8<BITS>(vw[i].x, vw[i].y, mx_scale(vsb[i]));
    bf16_t* d = a.v + head + static_cast<size_t>(dim) * p.T + 64 * ti + j0;
    const int left = n - j0;
    if (left >= 8) {
      *reinterpret_cast<uint4*>(d) = __builtin_bit_cast(uint4, x);
    } else {   // the tokens behind the last stay as they were
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) d[e] = static_cast<bf16_t>(x[e >> 1] >> (16 * (e & 1)));
    }
  }
}

}  // namespace

hipError_t launch_kv_append_mx(hipStream_t st, const bf16_t* qkv, int N, const RopeGeom& g,
                               const bf16_t* g_q, const bf16_t* g_k, bf16_t* q_out,
                               const MxPages& pages, const RowStreams& rs) {
  if (N == 0) return hipSuccess;
  AppendArgs a;
  a.qkv = qkv;
  a.q_out = q_out;
  a.g_q = g_q;
  a.g_k = g_k;
  a.p = pages;
  a.N = N;
  a.D = g.D;
  a.lat_w = g.lat_w;
  a.fT = pages.fT;
  a.fW = make_fastdiv(g.lat_w);
  a.fnt = pages.fnt;
  a.v_tiles = N / g.T * pages.nt;
  a.fvt = make_fastdiv(a.v_tiles);
  a.eps = g.eps;
  const int seg_hw = 2 * (g.hd / 6), seg_t = g.hd - 2 * seg_hw;
  a.pairs_t = seg_t / 2;
  a.pairs_h = seg_hw / 2;
  int pair = 0;
  for (int k = 0; k < 64; ++k) a.inv_freq[k] = 0.0;
  for (const int seg : {seg_t, seg_hw, seg_hw})
    for (int k = 0; k < seg / 2; ++k)
      a.inv_freq[pair++] = pow(static_cast<double>(g.theta), -2.0 * k / seg) / 6.283185307179586;
  a.rs = rs;
  // chunks of a lane, rows of a wave and waves of a row by the row's width
  const int chunks = (g.D / 8 + 63) / 64;
  int rows = 0;   // of a workgroup
#define ARDIT_APPEND_CASE(C, R, W)                                                                   \
  do {                                                                                               \
    rows = 4 / W * R;                                                                                \
    a.qk_groups = (N + rows - 1) / rows;                                                             \
    const dim3 grid(a.qk_groups + a.v_tiles * g.H);                                                  \
    if (pages.bits == 8) hipLaunchKernelGGL((kv_append_mx_kernel<C, R, W, 8>), grid, dim3(256), 0, st, a); \
    else hipLaunchKernelGGL((kv_append_mx_kernel<C, R, W, 4>), grid, dim3(256), 0, st, a);           \
  } while (0)
  if (chunks <= 1) ARDIT_APPEND_CASE(1, 2, 1);
  else if (chunks <= 2) ARDIT_APPEND_CASE(2, 2, 1);
  else if (chunks <= 3) ARDIT_APPEND_CASE(3, 1, 1);
  else if (chunks <= 4) ARDIT_APPEND_CASE(4, 1, 1);
  else if (chunks <= 6) ARDIT_APPEND_CASE(3, 1, 2);
  else if (chunks <= 8) ARDIT_APPEND_CASE(4, 1, 2);
  else if (chunks <= 12) ARDIT_APPEND_CASE(3, 1, 4);
  else ARDIT_APPEND_CASE(4, 1, 4);
#undef ARDIT_APPEND_CASE
  return hipGetLastError();
}

hipError_t launch_kv_read_mx(hipStream_t st, const MxPages& p, bf16_t* k_pages, bf16_t* v_pages,
                             const int32_t* page_table, int max_frames, int n_pages,
                             const RowStreams& rs) {
  ReadArgs a;
  a.p = p;
  a.k = k_pages;
  a.v = v_pages;
  a.page_table = page_table;
  a.max_frames = max_frames;
  a.n_pages = n_pages;
  a.rs = rs;
  int64_t tiles = 0;
  for (int i = 0; i < rs.n; ++i) {
    a.rs.s[i].row_begin = static_cast<int32_t>(tiles);
    tiles += mx_tiles(rs.s[i].len, p.T, p.nt);
  }
  if (tiles == 0) return hipSuccess;
  a.tiles = static_cast<int>(tiles);
  a.total = static_cast<int>(tiles * p.H);
  a.ftiles = make_fastdiv(static_cast<uint32_t>(tiles));
  const dim3 grid(static_cast<unsigned>((a.total + kNumXcd - 1) / kNumXcd * kNumXcd));
  if (p.hd == 128) {
    if (p.bits == 8) hipLaunchKernelGGL((kv_read_mx_kernel<128, 8>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((kv_read_mx_kernel<128, 4>), grid, dim3(256), 0, st, a);
  } else {
    if (p.bits == 8) hipLaunchKernelGGL((kv_read_mx_kernel<64, 8>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((kv_read_mx_kernel<64, 4>), grid, dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace ardit
