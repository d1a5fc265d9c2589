// Linear layer over a few rows with 4-bit weights in groups along K:
//   out[m, n] = f(bias[n] + add[m, n] + sum_g s[n, g] sum_{k in g} x[m, k] (q[n, k] - z[n, g])).
//
// Bound by the bytes of the codes, so they are read once, in their own
// layout, 16 bytes a lane, and the arithmetic on them is kept to a few
// instructions per 8 codes:
//  * The products run on bf16 MFMAs (16 rows of x by 16 weight rows, 32 k).
//    A code as a byte is the e4m3 number q * 2^-9 (subnormals and the first
//    binade are one even ladder), so 8 codes become fp32 with two masks, a
//    shift and four conversions; the zero point is taken off there, and the
//    differences, whole numbers below 16, are bf16 exactly.  (Taken off the
//    sums, as z sum x, it costs ten instructions less, 14.1 us in place of 14.7
//    for 16 rows of 8192 x 8192, but then an outlier of x that meets a weight of
//    zero swamps the rest of its group.)
//  * The differences are held 2^11 times too small, so that their products with
//    a group's 128 finite x add up to a finite sum (128 * 15 < 2^11).  The
//    group's scale, 2^11 times as large, multiplies that sum in fp32: the
//    weights are never rounded.
//  * fp32 x is cut into three bf16 parts of 8 bits each (their sum is x
//    exactly), so its products are exact as well; the small parts are summed
//    first, where fp32 rounds least.
//  * A lane's 16 bytes are 32 consecutive k of one weight row, while one MFMA
//    takes 8 k from each of four lane groups: a 4 x 4 transpose of dwords
//    between the groups (four lane swaps) makes every MFMA cover 32
//    consecutive k, which lie in one group.
// The waves of a block split K in chunks of 128 and are summed through LDS in
// order.  The split depends on K and N, never on M: a row's bits do not
// depend on the rows beside it.
#include <type_traits>

#include "device_common.h"
#include "kernels.h"

namespace sd {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr int KC = 128;  // k per chunk: 16 bytes of codes a lane

// d + A B over 32 k for a 16 x 16 tile: A rows m, B columns n, lane l holds 8
// k from 8 (l / 16) on of row / column l % 16; D rows 4 (l / 16) + i, column l % 16.
__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
#else
  return c;
#endif
}

// r[i] of lane group g <-> r[g] of lane group i.
__device__ __forceinline__ void transpose_groups(u32x4& r) {
#if defined(__HIP_DEVICE_COMPILE__)
  auto a = __builtin_amdgcn_permlane32_swap(r[0], r[2], false, false);
  auto b = __builtin_amdgcn_permlane32_swap(r[1], r[3], false, false);
  auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
  auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
  r[0] = c[0]; r[1] = c[1]; r[2] = d[0]; r[3] = d[1];
#endif
}

// The high halves of a (first) and b as one dword.
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

constexpr float DOWN = 1.0f / 2048;  // codes and zero points are held this much smaller

// (code - zero point) * DOWN of 8 codes -> bf16, in the order of k; z: the zero point * DOWN.
__device__ __forceinline__ u32x4 codes_bf16(uint32_t w, float z) {
  u32x4 r = {0, 0, 0, 0};
#if defined(__HIP_DEVICE_COMPILE__)
  const uint32_t even = w & 0x0F0F0F0Fu, odd = (w >> 4) & 0x0F0F0F0Fu;
  const auto put = [&](auto e, auto o, int i) __attribute__((always_inline)) {
    r[i] = high_halves(__float_as_uint(e[0] - z), __float_as_uint(o[0] - z));
    r[i + 1] = high_halves(__float_as_uint(e[1] - z), __float_as_uint(o[1] - z));
  };
  put(__builtin_amdgcn_cvt_scalef32_pk_f32_fp8(even, 512.f * DOWN, false), __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(odd, 512.f * DOWN, false), 0);
  put(__builtin_amdgcn_cvt_scalef32_pk_f32_fp8(even, 512.f * DOWN, true), __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(odd, 512.f * DOWN, true), 2);
#endif
  return r;
}

// SiLU where asked: one branch around all 8 (value by value the compiler
// computes it always and picks: fp32, 16 rows of 4096 x 4096 12.0 us, as under
// SiLU, against 9.0).
__device__ __forceinline__ void silu_if(int on, float (&v)[8]) {
  if (__builtin_amdgcn_readfirstlane(on)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = silu_f(v[e]);
    asm volatile("" : "+v"(v[0]));  // (and keeps the branch)
  }
}

// A wave's work in order: chunks wave, wave + nw, ... of the block's tiles of
// weight rows (blockIdx.x, + gridDim.x, ...), one sequence, so that loads run
// ahead across tiles.
struct Item {
  int tile, c;
  __device__ __forceinline__ void next(int wave, int nw, int chunks, int stride) {
    c += nw;
    if (c >= chunks) {
      c = wave;
      tile += stride;
    }
  }
};

// Codes, scales and zero points of T x 16 weight rows.  Codes: four lanes a
// row, 16 bytes each.  Scales: lane (col, g) loads those of row col and the
// chunk's group g, and every lane of the column asks it.  (Offsets past a
// resource's end, of rows past N, read as zero.)
template <int T, int G>
struct Weights {
  static constexpr int GC = KC / G;
  int woff, col, grp;
  __device__ __forceinline__ Weights(const LinearW4Args& a, int lane) : col(lane & 15), grp(lane >> 4) {
    woff = (lane >> 2) * (a.K >> 1) + (lane & 3) * 16;
  }
  __device__ __forceinline__ void codes(const LinearW4Args& a, const Item& it, u32x4 (&w)[T]) const {
    const int n0 = it.tile * 16 * T, rowb = a.K >> 1;
    const __amdgpu_buffer_rsrc_t r = make_rsrc(a.w + (long)n0 * rowb, (long)min(16 * T, a.N - n0) * rowb);
#pragma unroll
    for (int t = 0; t < T; ++t)
      w[t] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, woff + 16 * t * rowb, it.c * (KC / 2), 0));
  }
  __device__ __forceinline__ void scales(const LinearW4Args& a, const Item& it, float (&s)[T], int (&z)[T]) const {
    const int n0 = it.tile * 16 * T;
    const long first = (long)n0 * a.groups, count = (long)min(16 * T, a.N - n0) * a.groups;
    if (grp < GC) {
      const int g = min(it.c * GC + grp, a.groups - 1);
#pragma unroll
      for (int t = 0; t < T; ++t) {
        const int i = (16 * t + col) * a.groups + g;
        if (a.scale_f32)
          s[t] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(make_rsrc((const float*)a.scale + first, count * 4), i * 4, 0, 0));
        else
          s[t] = __uint_as_float((uint32_t)__builtin_amdgcn_raw_buffer_load_b16(make_rsrc((const bf16*)a.scale + first, count * 2), i * 2, 0, 0) << 16);
        if (a.zero) z[t] = __builtin_amdgcn_raw_buffer_load_b8(make_rsrc(a.zero + first, count), i, 0, 0);
      }
    }
  }
  // what the products take of them: the scale / DOWN, the zero point * DOWN
  __device__ __forceinline__ static float scale_up(float s) { return s * (1.0f / DOWN); }
  __device__ __forceinline__ static float zero_down(const LinearW4Args& a, int z) { return (a.zero ? (float)(z & 15) : 8.0f) * DOWN; }
  __device__ __forceinline__ float at(float v, int g) const { return __shfl(v, col + 16 * g, 64); }
};

// The sum of nw waves' tiles ([T][MT][4][64] accumulators, `apart` floats apart)
// in order, and the epilogue, on rows of 16 T columns.
template <int T, int MT>
__device__ __forceinline__ void finish(const LinearW4Args& a, const float* red, int apart, int nw, int n0, int m0, int tid, int nt,
                                       bool row_scale) {
  constexpr int TILE = T * MT * 256;
  for (int e = tid; e < TILE; e += nt) {
    const int nl = e % (16 * T), ml = e / (16 * T);
    const int n = n0 + nl, m = m0 + ml;
    if (n >= a.N || m >= a.M) continue;
    const int at = (((nl >> 4) * MT + (ml >> 4)) * 4 + (ml & 3)) * 64 + ((ml & 15) >> 2) * 16 + (nl & 15);
    const float b = a.bias ? a.bias[n] : 0.f, ad = a.add ? a.add[(long)m * a.N + n] : 0.f, xs = row_scale ? a.x_scale[m] : 1.f;
    float v = red[at];
    for (int u = 1; u < nw; ++u) v += red[u * apart + at];
    v = fmaf(v, xs, b) + ad;
    if (a.silu_out) v = silu_f(v);
    if (a.out_f32)
      ((float*)a.out)[m * a.out_ld + n] = v;
    else
      ((bf16*)a.out)[m * a.out_ld + n] = (bf16)v;
  }
}

}  // namespace

// bf16 (E8 = 0) and e4m3 (E8 = 1) x, for MT tiles of 16 rows and T of 16 weight
// rows.  Neighbouring lanes load neighbouring bytes of a row (a lane per row,
// as the MFMA wants it, takes the L1 one cycle per lane: 8192 x 8192, 16 rows
// 18.8 us); a wave's own piece of LDS turns them into operands, without a
// barrier: 14.7 us, 2.4 TB/s of codes.  Loading alone takes 7; the turn, the
// scales and the waves' sums are the rest.
template <bool E8, int MT, int T>
__host__ __device__ constexpr int w4_wave_bytes() { return T * 16 * 80 + MT * 16 * 17 * (E8 ? 8 : 16); }
template <int T>
__host__ __device__ constexpr int w4_f32_wave_bytes() { return T * 16 * 80 + 3 * 16 * (KC + 16); }

template <bool E8, int MT, int T, int G>
__global__ __launch_bounds__(1024) void linear_w4_kernel(LinearW4Args a) {
  constexpr int GC = KC / G, JG = G / 32;  // groups per chunk; MFMA steps per group
  constexpr int PF = 2;                    // chunks whose codes are in flight
  constexpr int XB = E8 ? 8 : 16;          // bytes of 8 k of x
  constexpr int WROW = 80, XROW = 16 * XB + XB;  // LDS rows of codes and x: padded against bank conflicts
  constexpr int WAVE = w4_wave_bytes<E8, MT, T>();
  typedef typename std::conditional<E8, uint2, u32x4>::type XPiece;
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
  const int m0 = blockIdx.y * 16 * MT, tiles = (a.N + 16 * T - 1) / (16 * T);
  const int col = lane & 15, grp = lane >> 4;
  uint8_t* wl = smem + wave * WAVE;
  uint8_t* xl = wl + T * 16 * WROW;
  const int wput = (lane >> 2) * WROW + (lane & 3) * 16, wget = col * WROW + grp * 16;
  const int xput = grp * XROW + col * XB, xget = col * XROW + grp * XB;
  const int ldb = (int)a.x_ld * (XB / 8), chunks = (a.K + KC - 1) / KC, rows = min(16 * MT, a.M - m0);
  const __amdgpu_buffer_rsrc_t xr = make_rsrc((const uint8_t*)a.x + (long)m0 * ldb, (long)(rows - 1) * ldb + a.K * (XB / 8));
  const Weights<T, G> wt(a, lane);
  // x: piece i of a lane is row 4 i + lane / 16, 8 k from 8 (lane % 16) on
  const int xoff = grp * ldb + col * XB;
  const bool xblocks = E8 && a.x_blocks > 1;

  float sn[T], xsn[MT];  // (xsn: row col of each tile of x)
  int zn[T];
#pragma unroll
  for (int i = 0; i < MT; ++i) xsn[i] = 1.0f;
  auto load_x = [&](int c, XPiece (&x)[4 * MT]) __attribute__((always_inline)) {
    // (K is a multiple of 8: a lane's 8 k are all in or all out)
    const int at = c * KC + 8 * col < a.K ? xoff : OOB;
#pragma unroll
    for (int i = 0; i < 4 * MT; ++i) {
      if (4 * i >= rows) break;  // (rows past M hold anything: they reach only their own results)
      const int soff = c * 16 * XB;
      if constexpr (E8)
        x[i] = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(xr, at + i * 4 * ldb, soff, 0));
      else
        x[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(xr, at + i * 4 * ldb, soff, 0));
    }
    if (xblocks)
#pragma unroll
      for (int i = 0; i < MT; ++i) xsn[i] = a.x_scale[(long)min(m0 + 16 * i + col, a.M - 1) * a.x_blocks + c];
  };

  f32x4 acc[T][MT];
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 w[PF][T];
  XPiece xn[4 * MT] = {};
  Item it = {(int)blockIdx.x, wave}, it1 = it, itw;  // this chunk, the next, the one whose codes are loaded next
  it1.next(wave, nw, chunks, gridDim.x);
  itw = it1;
  wt.codes(a, it, w[0]);  // (nw <= chunks: every wave has a chunk of every tile)
  load_x(it.c, xn);
  wt.scales(a, it, sn, zn);
#pragma unroll
  for (int u = 1; u < PF; ++u) {
    if (itw.tile < tiles) wt.codes(a, itw, w[u]);
    itw.next(wave, nw, chunks, gridDim.x);
  }
  auto chunk = [&](u32x4 (&w)[T]) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < T; ++t) *(u32x4*)(wl + t * 16 * WROW + wput) = w[t];
#pragma unroll
    for (int i = 0; i < 4 * MT; ++i) *(XPiece*)(xl + i * 4 * XROW + xput) = xn[i];
    float s[T], z[T], xs[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) xs[i] = xsn[i];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      s[t] = wt.scale_up(sn[t]);
      z[t] = wt.zero_down(a, zn[t]);
    }
    asm volatile("" ::: "memory");  // (one wave's LDS accesses complete in order)
    u32x4 q[T];
#pragma unroll
    for (int t = 0; t < T; ++t) q[t] = *(const u32x4*)(wl + t * 16 * WROW + wget);
    XPiece xp[MT][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) xp[i][j] = *(const XPiece*)(xl + i * 16 * XROW + j * 4 * XB + xget);
    if (it1.tile < tiles) {
      load_x(it1.c, xn);
      wt.scales(a, it1, sn, zn);
    }
    if (itw.tile < tiles) wt.codes(a, itw, w);
#pragma unroll
    for (int t = 0; t < T; ++t) transpose_groups(q[t]);

    f32x4 part[T][MT];  // e4m3: the chunk's sums, until its scale of x multiplies them
#pragma unroll
    for (int g = 0; g < GC; ++g) {
      f32x4 d[T][MT];
      const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
      float zg[T];
#pragma unroll
      for (int t = 0; t < T; ++t) zg[t] = wt.at(z[t], g);
#pragma unroll
      for (int j = g * JG; j < (g + 1) * JG; ++j) {
        const bool first = j == g * JG;
        u32x4 b[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          if constexpr (E8) {
#if defined(__HIP_DEVICE_COMPILE__)
            b[i][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(xp[i][j].x, 1.f, false));
            b[i][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(xp[i][j].x, 1.f, true));
            b[i][2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(xp[i][j].y, 1.f, false));
            b[i][3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(xp[i][j].y, 1.f, true));
#else
            b[i] = u32x4{0, 0, 0, 0};
#endif
          } else {
            b[i] = xp[i][j];
          }
        }
#pragma unroll
        for (int t = 0; t < T; ++t) {
          const u32x4 qb = codes_bf16(q[t][j], zg[t]);
#pragma unroll
          for (int i = 0; i < MT; ++i) d[t][i] = mfma(b[i], qb, first ? zero : d[t][i]);
        }
      }
#pragma unroll
      for (int t = 0; t < T; ++t) {
        const float sg = wt.at(s[t], g);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if constexpr (E8)
              part[t][i][e] = g == 0 ? sg * d[t][i][e] : fmaf(sg, d[t][i][e], part[t][i][e]);
            else
              acc[t][i][e] = fmaf(sg, d[t][i][e], acc[t][i][e]);
          }
      }
    }
    if constexpr (E8) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = __shfl(xs[i], 4 * grp + e, 64);
#pragma unroll
          for (int t = 0; t < T; ++t) acc[t][i][e] = fmaf(x, part[t][i][e], acc[t][i][e]);
        }
    }
    if (it1.tile != it.tile) {  // the tile's last chunk
      float* red = (float*)wl;  // (the wave's own operands are used up)
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            red[(t * MT + i) * 256 + e * 64 + lane] = acc[t][i][e];
            acc[t][i][e] = 0.f;
          }
      __syncthreads();
      finish<T, MT>(a, (const float*)smem, WAVE / 4, nw, it.tile * 16 * T, m0, threadIdx.x, blockDim.x, E8 && !xblocks);
      __syncthreads();
    }
    it = it1;
    it1.next(wave, nw, chunks, gridDim.x);
    itw.next(wave, nw, chunks, gridDim.x);
  };
  while (it.tile < tiles)
#pragma unroll
    for (int u = 0; u < PF; ++u)
      if (it.tile < tiles) chunk(w[u]);
}

// fp32 x, and any x under SiLU, for 16 rows and T tiles of 16 weight rows.  As
// above, but x goes through LDS half a chunk at a time, cut into its parts on
// the way.  (Sharing that pass among 2 to 8 waves side by side left too few
// waves along K and made all of them wait for it: 8192 x 8192, 1 row 40 us.)
template <int T, int G>
__global__ __launch_bounds__(1024) void linear_w4_f32_kernel(LinearW4Args a) {
  constexpr int GC = KC / G, HC = KC / 2, WROW = 80, XROW = HC * 2 + 16, PART = 16 * XROW;
  constexpr int WAVE = w4_f32_wave_bytes<T>();
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
  const int m0 = blockIdx.y * 16, tiles = (a.N + 16 * T - 1) / (16 * T);
  const int col = lane & 15, grp = lane >> 4;
  uint8_t* wl = smem + wave * WAVE;
  uint8_t* xl = wl + T * 16 * WROW;  // [3][16] rows
  const int wput = (lane >> 2) * WROW + (lane & 3) * 16, wget = col * WROW + grp * 16;
  const int xput = (lane >> 3) * XROW + (lane & 7) * 16, xget = col * XROW + grp * 16;
  const int xs = a.x_type == 0 ? 4 : 2, ldb = (int)a.x_ld * xs;
  const int chunks = (a.K + KC - 1) / KC, rows = min(16, a.M - m0);
  const __amdgpu_buffer_rsrc_t xr = make_rsrc((const uint8_t*)a.x + (long)m0 * ldb, (long)(rows - 1) * ldb + a.K * xs);
  const Weights<T, G> wt(a, lane);
  const int xoff = (lane >> 3) * ldb + (lane & 7) * 8 * xs;  // 8 lanes a row, 8 rows a load

  // half h of chunk c
  auto load_x = [&](int c, int h, u32x4 (&x)[2][2]) __attribute__((always_inline)) {
    const int k = c * KC + h * HC;
    if (k >= a.K) {  // (no offset past the rows, not even with lanes switched off)
#pragma unroll
      for (int i = 0; i < 2; ++i) x[i][0] = x[i][1] = u32x4{0, 0, 0, 0};
      return;
    }
    const int at = k + 8 * (lane & 7) < a.K ? xoff : OOB;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (8 * i >= rows) break;
      const int off = at + i * 8 * ldb;
      x[i][0] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(xr, off, k * xs, 0));
      if (a.x_type == 0) x[i][1] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(xr, off + 16, k * xs, 0));
    }
  };
  auto put_x = [&](const u32x4 (&x)[2][2]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (8 * i >= rows) break;
      uint32_t part[3][8];
      float xv[8];
      if (a.x_type == 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) xv[e] = __uint_as_float(x[i][e >> 2][e & 3]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) xv[e] = __uint_as_float(e & 1 ? x[i][0][e >> 1] & 0xFFFF0000u : x[i][0][e >> 1] << 16);
      }
      silu_if(a.silu_in, xv);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float v = xv[e];
        // (an infinity or NaN leaves a NaN in the second part)
        part[0][e] = __float_as_uint(v);
        v -= __uint_as_float(part[0][e] & 0xFFFF0000u);
        part[1][e] = __float_as_uint(v);
        v -= __uint_as_float(part[1][e] & 0xFFFF0000u);
        part[2][e] = __float_as_uint(v);
      }
#pragma unroll
      for (int u = 0; u < 3; ++u) {
        u32x4 b;
#pragma unroll
        for (int e = 0; e < 4; ++e) b[e] = high_halves(part[u][2 * e], part[u][2 * e + 1]);
        *(u32x4*)(xl + u * PART + i * 8 * XROW + xput) = b;
      }
    }
  };

  f32x4 acc[T];
#pragma unroll
  for (int t = 0; t < T; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 wn[T], xn[2][2] = {};
  float sn[T];
  int zn[T];
  Item it = {(int)blockIdx.x, wave};
  wt.codes(a, it, wn);  // (nw <= chunks: every wave has a chunk of every tile)
  load_x(it.c, 0, xn);
  wt.scales(a, it, sn, zn);
  while (it.tile < tiles) {
    Item it1 = it;
    it1.next(wave, nw, chunks, gridDim.x);
    float s[T], z[T], zg[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      *(u32x4*)(wl + t * 16 * WROW + wput) = wn[t];
      s[t] = wt.scale_up(sn[t]);
      z[t] = wt.zero_down(a, zn[t]);
    }
    u32x4 q[T];
    f32x4 d[T], e[T];  // products: of the first part, of the others
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      put_x(xn);
      asm volatile("" ::: "memory");  // (one wave's LDS accesses complete in order)
      if (h == 0) {
#pragma unroll
        for (int t = 0; t < T; ++t) q[t] = *(const u32x4*)(wl + t * 16 * WROW + wget);
        load_x(it.c, 1, xn);
        if (it1.tile < tiles) wt.codes(a, it1, wn);
      } else if (it1.tile < tiles) {
        load_x(it1.c, 0, xn);
        wt.scales(a, it1, sn, zn);
      }
      if (h == 0)
#pragma unroll
        for (int t = 0; t < T; ++t) transpose_groups(q[t]);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int jc = 2 * h + j, g = jc * 32 / G;  // step and group within the chunk
        u32x4 x[3];
#pragma unroll
        for (int u = 0; u < 3; ++u) x[u] = *(const u32x4*)(xl + u * PART + j * 64 + xget);
        if (jc * 32 % G == 0)
#pragma unroll
          for (int t = 0; t < T; ++t) {
            d[t] = e[t] = zero;
            zg[t] = wt.at(z[t], g);
          }
#pragma unroll
        for (int t = 0; t < T; ++t) {
          const u32x4 b = codes_bf16(q[t][jc], zg[t]);
          e[t] = mfma(x[1], b, mfma(x[2], b, e[t]));
          d[t] = mfma(x[0], b, d[t]);
        }
        if ((jc + 1) * 32 % G == 0)
#pragma unroll
          for (int t = 0; t < T; ++t) {
            const float sg = wt.at(s[t], g);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[t][i] = fmaf(sg, d[t][i] + e[t][i], acc[t][i]);
          }
      }
      asm volatile("" ::: "memory");
    }
    if (it1.tile != it.tile) {  // the tile's last chunk
      float* red = (float*)wl;  // (the wave's own operands are used up)
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          red[t * 256 + i * 64 + lane] = acc[t][i];
          acc[t][i] = 0.f;
        }
      __syncthreads();
      finish<T, 1>(a, (const float*)smem, WAVE / 4, nw, it.tile * 16 * T, m0, threadIdx.x, blockDim.x, false);
      __syncthreads();
    }
    it = it1;
  }
}

// The same for wide layers: WN waves side by side (16 weight rows each) share
// one pass of x through LDS, wave rows wk split K.  (20160 x 1280, fp32 under
// SiLU: 1 row 11.3 us against 13.6 above, 32 rows 17.9 against 27.9; narrower
// layers leave it too few waves: 8192 x 8192, 1 row 61 us against 20.)  Bound by
// bringing x in, activated and cut, once per block, and its LDS reads.
template <int MT, int G>
__global__ __launch_bounds__(1024) void linear_w4_wide_kernel(LinearW4Args a) {
  constexpr int WN = 8, GC = KC / G, JG = G / 32, LD = KC + 8;  // LDS rows 272 bytes apart: no bank conflicts over 16 rows
  constexpr int ROWS = 16 * MT, NT = 64 * WN, PIECES = ROWS * (KC / 8), PPT = (PIECES + NT - 1) / NT;
  constexpr int XB = 3 * ROWS * LD;  // bf16 of one wave row's chunk
  extern __shared__ float lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nwk = blockDim.x / NT;
  const int wn = wave % WN, wk = wave / WN, tid = threadIdx.x % NT;
  bf16* xs = (bf16*)lds + wk * XB;  // [3][ROWS][LD]
  const int n0 = blockIdx.x * 16 * WN, m0 = blockIdx.y * ROWS;
  const int col = lane & 15, grp = lane >> 4;
  const bool tile_on = n0 + 16 * wn < a.N;
  const int tile = tile_on ? n0 / 16 + wn : n0 / 16;
  const int rowb = a.K >> 1;
  const __amdgpu_buffer_rsrc_t wr = make_rsrc(a.w + (long)tile * 16 * rowb, (long)min(16, a.N - 16 * tile) * rowb);
  const int woff = col * rowb + grp * 16;
  const long sat = (long)min(16 * tile + col, a.N - 1) * a.groups;
  const int chunks = (a.K + KC - 1) / KC;

  // A thread stages 8 k of a row at a time, 16 threads a row.
  float xr[PPT][8];
  auto fetch = [&](int c) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < PPT; ++p) {
      const int idx = tid + p * NT, m = m0 + idx / 16, k = c * KC + 8 * (idx % 16);
#pragma unroll
      for (int e = 0; e < 8; ++e) xr[p][e] = 0.f;
      if (idx < PIECES && m < a.M && k < a.K) {
        if (a.x_type == 0)
          load8f((const float*)a.x + (long)m * a.x_ld + k, xr[p]);
        else
          load8f((const bf16*)a.x + (long)m * a.x_ld + k, xr[p]);
      }
    }
  };
  auto stage = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < PPT; ++p) {
      const int idx = tid + p * NT, row = idx / 16;
      if (idx >= PIECES || m0 + row >= a.M) continue;  // (whole groups of 16 lanes)
      uint32_t part[3][8];
      silu_if(a.silu_in, xr[p]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float v = xr[p][e];
        // (an infinity or NaN leaves a NaN in the second part)
        part[0][e] = __float_as_uint(v);
        v -= __uint_as_float(part[0][e] & 0xFFFF0000u);
        part[1][e] = __float_as_uint(v);
        v -= __uint_as_float(part[1][e] & 0xFFFF0000u);
        part[2][e] = __float_as_uint(v);
      }
#pragma unroll
      for (int u = 0; u < 3; ++u) {
        u32x4 b;
#pragma unroll
        for (int e = 0; e < 4; ++e) b[e] = high_halves(part[u][2 * e], part[u][2 * e + 1]);
        *(u32x4*)(xs + (u * ROWS + row) * LD + 8 * (idx % 16)) = b;
      }
    }
  };

  f32x4 acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  fetch(wk);  // (nwk <= chunks)
  // (codes and scales: a lane per row.  The turn through LDS of the kernels
  // above, and scales a round ahead, cost these barriers 2 us.)
  u32x4 wnext = __builtin_bit_cast(u32x4, buf_load16(wr, woff + wk * (KC / 2)));
  const int rounds = (chunks + nwk - 1) / nwk;
  for (int r = 0; r < rounds; ++r) {
    const int c = r * nwk + wk;
    if (r) __syncthreads();  // the last round's operands have been read
    if (c < chunks) stage();
    __syncthreads();
    u32x4 w = wnext;
    float s[GC], z[GC];
#pragma unroll
    for (int g = 0; g < GC; ++g) {
      const long i = sat + min(c * GC + g, a.groups - 1);
      s[g] = (a.scale_f32 ? ((const float*)a.scale)[i] : (float)((const bf16*)a.scale)[i]) * (1.0f / DOWN);
      z[g] = (a.zero ? (float)(a.zero[i] & 15) : 8.0f) * DOWN;
    }
    if (c + nwk < chunks) {
      fetch(c + nwk);
      wnext = __builtin_bit_cast(u32x4, buf_load16(wr, woff + (c + nwk) * (KC / 2)));
    }
    if (c >= chunks) continue;  // (the last round)
    transpose_groups(w);
#pragma unroll
    for (int g = 0; g < GC; ++g) {
      u32x4 q[JG];
#pragma unroll
      for (int j = 0; j < JG; ++j) q[j] = codes_bf16(w[g * JG + j], z[g]);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 2; u >= 0; --u)
#pragma unroll
          for (int j = 0; j < JG; ++j)
            d = mfma(*(const u32x4*)(xs + (u * ROWS + 16 * i + col) * LD + 32 * (g * JG + j) + 8 * grp), q[j], d);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][e] = fmaf(s[g], d[e], acc[i][e]);
      }
    }
  }
  // [wn][wk][MT][4][64]
  __syncthreads();
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) lds[((wn * nwk + wk) * MT + i) * 256 + e * 64 + lane] = acc[i][e];
  __syncthreads();
  // wave row wk finishes what it can of its column's tile
  if (tile_on) finish<1, MT>(a, lds + wn * nwk * MT * 256, MT * 256, nwk, n0 + 16 * wn, m0, wk * 64 + lane, nwk * 64, false);
}

// Blocks: as many as run at once (16 waves a CU at up to 128 registers), each
// over several tiles where there are more (bf16, 16 rows, 20160 x 1280: 12.9 ->
// 11.6 us; 64 rows 33.5 -> 27.3).  A wave's sums take the place of its operands in LDS.
static dim3 w4_grid(int tiles, int rows, int nw) {
  const int once = 256 * (16 / nw);
  return dim3((unsigned)(tiles < once ? tiles : once), (unsigned)rows);
}

template <bool E8, int MT, int T, int G>
static void launch_tile(const LinearW4Args& a, hipStream_t s) {
  constexpr int MOST = 16;
  constexpr size_t wave = w4_wave_bytes<E8, MT, T>();
  static_assert(MOST * wave <= 160 * 1024 && wave >= T * MT * 1024, "the LDS holds 16 waves");
  const int chunks = (a.K + KC - 1) / KC, nw = chunks < MOST ? chunks : MOST;
  const dim3 grid = w4_grid((a.N + 16 * T - 1) / (16 * T), (a.M + 16 * MT - 1) / (16 * MT), nw);
  linear_w4_kernel<E8, MT, T, G><<<grid, 64 * nw, nw * wave, s>>>(a);
}

// Two tiles of x rows past 16 rows, two of weight rows where a block would have
// more than one anyway (6144 x 2048, 16 rows of bf16: 7.1 -> 5.8 us), as far as
// 128 registers hold them: groups of 32 take one by one, e4m3 in groups of 64
// one tile of x.
template <bool E8, int G>
static void launch_x(const LinearW4Args& a, hipStream_t s) {
  constexpr int MT = G == 128 || (G == 64 && !E8) ? 2 : 1, T = G == 32 ? 1 : 2;
  if (MT == 2 && a.M > 16)
    launch_tile<E8, MT, 1, G>(a, s);
  else if (T == 2 && a.N > 4096)
    launch_tile<E8, 1, T, G>(a, s);
  else
    launch_tile<E8, 1, 1, G>(a, s);
}

template <int T, int G>
static void launch_f32_tile(const LinearW4Args& a, hipStream_t s) {
  constexpr int MOST = 16;
  constexpr size_t wave = w4_f32_wave_bytes<T>();
  static_assert(MOST * wave <= 160 * 1024 && wave >= T * 1024, "the LDS holds 16 waves");
  const int chunks = (a.K + KC - 1) / KC, nw = chunks < MOST ? chunks : MOST;
  const dim3 grid = w4_grid((a.N + 16 * T - 1) / (16 * T), (a.M + 15) / 16, nw);
  linear_w4_f32_kernel<T, G><<<grid, 64 * nw, nw * wave, s>>>(a);
}

template <int MT, int G>
static void launch_wide(const LinearW4Args& a, hipStream_t s) {
  constexpr int WN = 8, MOST = 2;
  const int chunks = (a.K + KC - 1) / KC, nwk = chunks < MOST ? chunks : MOST;
  const dim3 grid((unsigned)((a.N + 16 * WN - 1) / (16 * WN)), (unsigned)((a.M + 16 * MT - 1) / (16 * MT)));
  // operands of x; the waves' sums take their place
  constexpr size_t row = 3 * 16 * MT * (KC + 8) * 2;
  static_assert(row >= WN * MT * 1024 && MOST * row <= 160 * 1024, "the sums fit, and all of it the LDS");
  linear_w4_wide_kernel<MT, G><<<grid, 64 * WN * nwk, nwk * row, s>>>(a);
}

// The kernel follows N alone, so that a row's bits do not depend on M: a
// compromise between few rows and many.  From 16384 outputs on the wide one is
// ahead at 64 rows, about level or ahead at 32 and for one row of a short K, and
// behind for one row of a long K (us, this one against the one above it, at
// 1 / 32 / 64 rows: 20160 x 1280 10 / 16 / 30 against 12 / 22 / 42, 16384 x 4000
// 29 / 42 / 45 against 17 / 39 / 75; at 12288 x 4096 28 / 42 / 43 against 17 / 31 / 58).
template <int G>
static void launch_f32(const LinearW4Args& a, hipStream_t s) {
  if (a.N < 16384) {
    // two tiles of weight rows share a pass of x, where a block would have more
    // than one anyway (6144 x 2048, 1 row: 8.2 -> 6.4 us); smaller groups spill
    if (G == 128 && a.N > 4096)
      launch_f32_tile<G == 128 ? 2 : 1, G>(a, s);
    else
      launch_f32_tile<1, G>(a, s);
  }
  else if (a.M > 16)
    launch_wide<2, G>(a, s);
  else
    launch_wide<1, G>(a, s);
}

hipError_t launch_linear_w4(const LinearW4Args& a, hipStream_t s) {
  if (a.M <= 0 || a.N <= 0) return hipSuccess;
  if (a.x_type == 0 || a.silu_in) {
    a.group == 32 ? launch_f32<32>(a, s) : a.group == 64 ? launch_f32<64>(a, s) : launch_f32<128>(a, s);
  } else if (a.x_type == 1) {
    a.group == 32 ? launch_x<false, 32>(a, s) : a.group == 64 ? launch_x<false, 64>(a, s) : launch_x<false, 128>(a, s);
  } else {
    a.group == 32 ? launch_x<true, 32>(a, s) : a.group == 64 ? launch_x<true, 64>(a, s) : launch_x<true, 128>(a, s);
  }
  return hipGetLastError();
}

}  // namespace sd
