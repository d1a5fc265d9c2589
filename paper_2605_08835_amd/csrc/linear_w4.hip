// Linear layer over a few rows with 4-bit weights in groups along K:
//   out[m, n] = f(bias[n] + add[m, n] + sum_g s[n, g] (sum_{k in g} x[m, k] q[n, k] - z[n, g] sum_{k in g} x[m, k])).
//
// Bound by the bytes of the codes, so they are read once, in their own
// layout, 16 bytes a lane, and the arithmetic on them is kept to a few
// instructions per 8 codes:
//  * The products run on bf16 MFMAs (16 rows of x by 16 weight rows, 32 k).
//    A code as a byte is the e4m3 number q * 2^-9 (subnormals and the first
//    binade are one even ladder), so 8 codes become bf16 with two masks, a
//    shift and four conversions, exactly.
//  * The zero point stays outside the products: sum x over the group, the
//    same for every weight row, comes from the staging pass or one more MFMA
//    with ones.
//  * A group's sums keep whole codes until its scale multiplies them in fp32:
//    the weights are never rounded.
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

// 8 codes -> bf16, in the order k = 0 2 4 6 1 3 5 7.
__device__ __forceinline__ u32x4 codes_bf16(uint32_t w) {
  u32x4 r = {0, 0, 0, 0};
#if defined(__HIP_DEVICE_COMPILE__)
  const uint32_t even = w & 0x0F0F0F0Fu, odd = (w >> 4) & 0x0F0F0F0Fu;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(even, 512.f, false));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(even, 512.f, true));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(odd, 512.f, false));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(odd, 512.f, true));
#endif
  return r;
}

// The high (low) halves of a (first) and b as one dword.
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }

// Codes of a tile of T x 16 weight rows, and the scale and zero point of a
// (row, group).  Offsets past the tile's last row read as zero; a row past N
// takes row N - 1's scales and is not stored.
template <int T, int G>
struct Weights {
  __amdgpu_buffer_rsrc_t rsrc;
  int off[T];
  long at[T];
  __device__ __forceinline__ Weights(const LinearW4Args& a, int n0, int col, int grp) {
    const int rowb = a.K >> 1;
    rsrc = make_rsrc(a.w + (long)n0 * rowb, (long)min(16 * T, a.N - n0) * rowb);
#pragma unroll
    for (int t = 0; t < T; ++t) {
      off[t] = (16 * t + col) * rowb + grp * 16;
      at[t] = (long)min(n0 + 16 * t + col, a.N - 1) * a.groups;
    }
  }
  __device__ __forceinline__ u32x4 codes(int t, int c) const {
    return __builtin_bit_cast(u32x4, buf_load16(rsrc, off[t] + c * (KC / 2)));
  }
  __device__ __forceinline__ void scales(const LinearW4Args& a, int t, int c, float (&s)[KC / G], float (&z)[KC / G]) const {
#pragma unroll
    for (int g = 0; g < KC / G; ++g) {
      const long i = at[t] + min(c * (KC / G) + g, a.groups - 1);
      s[g] = a.scale_f32 ? ((const float*)a.scale)[i] : (float)((const bf16*)a.scale)[i];
      z[g] = a.zero ? (float)(a.zero[i] & 15) : 8.0f;
    }
  }
};

// The sum of nw partial tiles of LDS ([wave][T][MT][4][64] accumulators) in
// order, and the epilogue, on rows of 16 T columns.
template <int T, int MT>
__device__ __forceinline__ void finish(const LinearW4Args& a, const float* red, int nw, int n0, int m0, int tid, int nt,
                                       bool row_scale) {
  constexpr int TILE = T * MT * 256;
  for (int e = tid; e < TILE; e += nt) {
    const int nl = e % (16 * T), ml = e / (16 * T);
    const int n = n0 + nl, m = m0 + ml;
    if (n >= a.N || m >= a.M) continue;
    const int at = (((nl >> 4) * MT + (ml >> 4)) * 4 + (ml & 3)) * 64 + ((ml & 15) >> 2) * 16 + (nl & 15);
    float v = red[at];
    for (int u = 1; u < nw; ++u) v += red[u * TILE + at];
    if (row_scale) v *= a.x_scale[m];
    if (a.bias) v += a.bias[n];
    if (a.add) v += a.add[(long)m * a.N + n];
    if (a.silu_out) v = silu_f(v);
    if (a.out_f32)
      ((float*)a.out)[m * a.out_ld + n] = v;
    else
      ((bf16*)a.out)[m * a.out_ld + n] = (bf16)v;
  }
}

}  // namespace

// bf16 (E8 = 0) and e4m3 (E8 = 1) x: every wave loads its own operands of x
// (through L1) for MT tiles of 16 rows and T of 16 weight rows.
template <bool E8, int MT, int T, int G>
__global__ __launch_bounds__(1024) void linear_w4_kernel(LinearW4Args a) {
  constexpr int GC = KC / G, JG = G / 32;  // groups per chunk; MFMA steps per group
  extern __shared__ float red[];           // [waves][T][MT][4][64]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, nw = blockDim.x >> 6;
  const int n0 = blockIdx.x * 16 * T, m0 = blockIdx.y * 16 * MT;
  const int col = lane & 15, grp = lane >> 4;
  const Weights<T, G> wt(a, n0, col, grp);
  const int chunks = (a.K + KC - 1) / KC;
  const uint8_t* xm[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) xm[i] = (const uint8_t*)a.x + (long)min(m0 + 16 * i + col, a.M - 1) * a.x_ld * (E8 ? 1 : 2);

  f32x4 acc[T][MT];
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 wn[T];
#pragma unroll
  for (int t = 0; t < T; ++t) wn[t] = wt.codes(t, wave);  // (nw <= chunks)
  for (int c = wave; c < chunks; c += nw) {
    u32x4 w[T], x[MT][4];
#pragma unroll
    for (int t = 0; t < T; ++t) w[t] = wn[t];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = c * KC + 32 * j + 8 * grp;  // (K is a multiple of 8: a lane's 8 k are all in or all out)
        u32x4 v = {0, 0, 0, 0};
        if (k < a.K) {
          if constexpr (E8) {
            const uint2 u = *(const uint2*)(xm[i] + k);
            v[0] = u.x; v[1] = u.y;
          } else {
            v = *(const u32x4*)(xm[i] + 2 * k);
          }
        }
        x[i][j] = v;
      }
    float s[T][GC], z[T][GC];
#pragma unroll
    for (int t = 0; t < T; ++t) wt.scales(a, t, c, s[t], z[t]);
    if (c + nw < chunks)
#pragma unroll
      for (int t = 0; t < T; ++t) wn[t] = wt.codes(t, c + nw);
#pragma unroll
    for (int t = 0; t < T; ++t) transpose_groups(w[t]);

    f32x4 part[T][MT];  // e4m3: the chunk's sums, until its scale of x multiplies them
#pragma unroll
    for (int g = 0; g < GC; ++g) {
      f32x4 d[T][MT], sx[MT];
#pragma unroll
      for (int j = g * JG; j < (g + 1) * JG; ++j) {
        u32x4 q[T];
#pragma unroll
        for (int t = 0; t < T; ++t) q[t] = codes_bf16(w[t][j]);
        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        const u32x4 ones = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          u32x4 b = {0, 0, 0, 0};  // the lane's 8 k in the order of codes_bf16
          if constexpr (E8) {
#if defined(__HIP_DEVICE_COMPILE__)
            const auto e0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)x[i][j][0], false), e1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)x[i][j][0], true);
            const auto e2 = __builtin_amdgcn_cvt_pk_f32_fp8((int)x[i][j][1], false), e3 = __builtin_amdgcn_cvt_pk_f32_fp8((int)x[i][j][1], true);
            b[0] = high_halves(__float_as_uint(e0[0]), __float_as_uint(e1[0]));
            b[1] = high_halves(__float_as_uint(e2[0]), __float_as_uint(e3[0]));
            b[2] = high_halves(__float_as_uint(e0[1]), __float_as_uint(e1[1]));
            b[3] = high_halves(__float_as_uint(e2[1]), __float_as_uint(e3[1]));
#endif
          } else {
            b[0] = low_halves(x[i][j][0], x[i][j][1]);
            b[1] = low_halves(x[i][j][2], x[i][j][3]);
            b[2] = high_halves(x[i][j][0], x[i][j][1]);
            b[3] = high_halves(x[i][j][2], x[i][j][3]);
          }
          const bool first = j == g * JG;
          sx[i] = mfma(b, ones, first ? zero : sx[i]);
#pragma unroll
          for (int t = 0; t < T; ++t) d[t][i] = mfma(b, q[t], first ? zero : d[t][i]);
        }
      }
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float v = fmaf(-z[t][g], sx[i][e], d[t][i][e]);
            if constexpr (E8)
              part[t][i][e] = g == 0 ? s[t][g] * v : fmaf(s[t][g], v, part[t][i][e]);
            else
              acc[t][i][e] = fmaf(s[t][g], v, acc[t][i][e]);
          }
    }
    if constexpr (E8) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int m = min(m0 + 16 * i + 4 * grp + e, a.M - 1);
          const float xs = a.x_blocks > 1 ? a.x_scale[(long)m * a.x_blocks + c] : 1.0f;
#pragma unroll
          for (int t = 0; t < T; ++t) acc[t][i][e] = fmaf(xs, part[t][i][e], acc[t][i][e]);
        }
    }
  }
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) red[((wave * T + t) * MT + i) * 256 + e * 64 + lane] = acc[t][i][e];
  __syncthreads();
  finish<T, MT>(a, red, nw, n0, m0, threadIdx.x, blockDim.x, E8 && a.x_blocks == 1);
}

// fp32 x, and any x under SiLU.  The activation and the cut into parts cost
// many times what a code does, so WN waves side by side (16 weight rows each)
// share one staging of x in LDS; wave rows wk split K.
template <int MT, int WN, int G>
__global__ __launch_bounds__(1024) void linear_w4_f32_kernel(LinearW4Args a) {
  constexpr int GC = KC / G, JG = G / 32, LD = KC + 8;  // LDS rows 272 bytes apart: no bank conflicts over 16 rows
  constexpr int ROWS = 16 * MT, NT = 64 * WN, PIECES = ROWS * (KC / 8), PPT = (PIECES + NT - 1) / NT;
  constexpr int XB = 3 * ROWS * LD;  // bf16 of one wave row's chunk
  extern __shared__ float lds[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, nwk = blockDim.x / NT;
  const int wn = wave % WN, wk = wave / WN, tid = threadIdx.x % NT;
  bf16* xs = (bf16*)lds + wk * XB;                               // [3][ROWS][LD]
  float* xsum = lds + nwk * (XB / 2) + wk * ROWS * GC;           // [GC][ROWS]
  const int n0 = blockIdx.x * 16 * WN, m0 = blockIdx.y * ROWS;
  const int col = lane & 15, grp = lane >> 4;
  const bool tile_on = n0 + 16 * wn < a.N;
  const Weights<1, G> wt(a, tile_on ? n0 + 16 * wn : n0, col, grp);
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
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float v = xr[p][e];
        if (a.silu_in) v = silu_f(v);
        sum += v;
        // (an infinity or NaN leaves a NaN in the second part)
        part[0][e] = __float_as_uint(v);
        v -= __uint_as_float(part[0][e] & 0xFFFF0000u);
        part[1][e] = __float_as_uint(v);
        v -= __uint_as_float(part[1][e] & 0xFFFF0000u);
        part[2][e] = __float_as_uint(v);
      }
#pragma unroll
      for (int u = 0; u < 3; ++u) {
        u32x4 b;  // the order of codes_bf16
        b[0] = high_halves(part[u][0], part[u][2]);
        b[1] = high_halves(part[u][4], part[u][6]);
        b[2] = high_halves(part[u][1], part[u][3]);
        b[3] = high_halves(part[u][5], part[u][7]);
        *(u32x4*)(xs + (u * ROWS + row) * LD + 8 * (idx % 16)) = b;
      }
#pragma unroll
      for (int o = 1; o < G / 8; o <<= 1) sum += __shfl_xor(sum, o, 64);
      if (idx % (G / 8) == 0) xsum[(idx % 16) / (G / 8) * ROWS + row] = sum;
    }
  };

  f32x4 acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  fetch(wk);  // (nwk <= chunks)
  u32x4 wnext = wt.codes(0, wk);
  const int rounds = (chunks + nwk - 1) / nwk;
  for (int r = 0; r < rounds; ++r) {
    const int c = r * nwk + wk;
    u32x4 w = wnext;
    if (r) __syncthreads();  // the last round's operands have been read
    if (c < chunks) stage();
    __syncthreads();
    float s[GC], z[GC];
    wt.scales(a, 0, min(c, chunks - 1), s, z);
    if (c + nwk < chunks) {
      fetch(c + nwk);
      wnext = wt.codes(0, c + nwk);
    }
    if (c >= chunks) continue;
    transpose_groups(w);
#pragma unroll
    for (int g = 0; g < GC; ++g) {
      u32x4 q[JG];
#pragma unroll
      for (int j = 0; j < JG; ++j) q[j] = codes_bf16(w[g * JG + j]);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 2; u >= 0; --u)
#pragma unroll
          for (int j = 0; j < JG; ++j)
            d = mfma(*(const u32x4*)(xs + (u * ROWS + 16 * i + col) * LD + 32 * (g * JG + j) + 8 * grp), q[j], d);
        const f32x4 sx = *(const f32x4*)(xsum + g * ROWS + 16 * i + 4 * grp);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][e] = fmaf(s[g], fmaf(-z[g], sx[e], d[e]), acc[i][e]);
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
  if (tile_on) finish<1, MT>(a, lds + wn * nwk * MT * 256, nwk, n0 + 16 * wn, m0, wk * 64 + lane, nwk * 64, false);
}

template <bool E8, int MT, int T>
static void launch_tile(const LinearW4Args& a, hipStream_t s) {
  const int chunks = (a.K + KC - 1) / KC, nw = chunks < 16 ? chunks : 16;
  const dim3 grid((unsigned)((a.N + 16 * T - 1) / (16 * T)), (unsigned)((a.M + 16 * MT - 1) / (16 * MT)));
  const size_t lds = (size_t)nw * T * MT * 1024;
  if (a.group == 32)
    linear_w4_kernel<E8, MT, T, 32><<<grid, 64 * nw, lds, s>>>(a);
  else if (a.group == 64)
    linear_w4_kernel<E8, MT, T, 64><<<grid, 64 * nw, lds, s>>>(a);
  else
    linear_w4_kernel<E8, MT, T, 128><<<grid, 64 * nw, lds, s>>>(a);
}

template <bool E8>
static void launch_x(const LinearW4Args& a, hipStream_t s) {
  if (a.M > 16)
    launch_tile<E8, 2, 1>(a, s);
  else if (a.N >= 8192)
    launch_tile<E8, 1, 2>(a, s);
  else
    launch_tile<E8, 1, 1>(a, s);
}

template <int MT, int WN>
static void launch_f32(const LinearW4Args& a, hipStream_t s) {
  constexpr int MOST = 16 / WN;  // wave rows
  const int chunks = (a.K + KC - 1) / KC, nwk = chunks < MOST ? chunks : MOST;
  const dim3 grid((unsigned)((a.N + 16 * WN - 1) / (16 * WN)), (unsigned)((a.M + 16 * MT - 1) / (16 * MT)));
  const size_t stage = (size_t)nwk * (3 * 16 * MT * (KC + 8) * 2 + 16 * MT * (KC / a.group) * 4), sum = (size_t)nwk * WN * MT * 1024;
  const size_t lds = stage > sum ? stage : sum;
  if (a.group == 32)
    linear_w4_f32_kernel<MT, WN, 32><<<grid, 64 * WN * nwk, lds, s>>>(a);
  else if (a.group == 64)
    linear_w4_f32_kernel<MT, WN, 64><<<grid, 64 * WN * nwk, lds, s>>>(a);
  else
    linear_w4_f32_kernel<MT, WN, 128><<<grid, 64 * WN * nwk, lds, s>>>(a);
}

hipError_t launch_linear_w4(const LinearW4Args& a, hipStream_t s) {
  if (a.M <= 0 || a.N <= 0) return hipSuccess;
  if (a.x_type == 0 || a.silu_in) {
    if (a.N < 4096)
      launch_f32<1, 2>(a, s);  // (8 wave rows' operands of 32 rows of x would pass the LDS)
    else if (a.N < 16384)
      a.M > 16 ? launch_f32<2, 4>(a, s) : launch_f32<1, 4>(a, s);
    else
      a.M > 16 ? launch_f32<2, 8>(a, s) : launch_f32<1, 8>(a, s);
  } else if (a.x_type == 1) {
    launch_x<false>(a, s);
  } else {
    launch_x<true>(a, s);
  }
  return hipGetLastError();
}

}  // namespace sd
