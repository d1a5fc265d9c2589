// Root-mean-square norm of rows, with the residual's addition and an e4m3
// output with scales: h = x + r, y = h / sqrt(mean h^2 + eps) * gamma.
//
// One pass: TPR lanes hold a row in fp32 registers, 16 bytes a load, R loads
// each, so that every input is read once and the sum, the norm and the scales'
// maxima come from the registers.  Bound by memory: 48 x 4096 rows of 320 bf16
// with a residual 93 us, 5.4 TB/s, 12301 of 1280 to e4m3 21 us, 5.3; one row 3 us,
// a launch and one round trip.
#include <type_traits>

#include "device_common.h"
#include "kernels.h"

namespace sd {

namespace {

// Pieces of 16 bytes at the alignment of their elements: the vector memory
// unit takes any address, and rows of odd widths start anywhere.
struct __attribute__((packed, aligned(2))) U16B { uint32_t w[4]; };
struct __attribute__((packed, aligned(1))) U8B { uint32_t w[2]; };
struct __attribute__((packed, aligned(1))) U4B { uint32_t w; };

template <typename T> struct Vec;
template <> struct Vec<float> { static constexpr int N = 4; };
template <> struct Vec<bf16> { static constexpr int N = 8; };

template <bool ANY>
__device__ __forceinline__ uint4 load_piece(const void* p) {
  if constexpr (ANY) {
    const U16B u = *(const U16B*)p;
    return make_uint4(u.w[0], u.w[1], u.w[2], u.w[3]);
  } else {
    return *(const uint4*)p;
  }
}
template <bool ANY>
__device__ __forceinline__ void store_piece(void* p, uint4 v) {
  if constexpr (ANY) {
    U16B u;
    u.w[0] = v.x; u.w[1] = v.y; u.w[2] = v.z; u.w[3] = v.w;
    *(U16B*)p = u;
  } else {
    *(uint4*)p = v;
  }
}
__device__ __forceinline__ void unpack(uint4 u, float (&v)[4]) {
  v[0] = __uint_as_float(u.x); v[1] = __uint_as_float(u.y); v[2] = __uint_as_float(u.z); v[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ void unpack(uint4 u, float (&v)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ uint4 pack(const float (&v)[4]) {
  return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
__device__ __forceinline__ uint4 pack(const float (&v)[8]) {
  bf16x8 b;
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = (bf16)v[i];
  return __builtin_bit_cast(uint4, b);
}

// Max of absolute values as their bits: a NaN's bits are above every
// number's, so a NaN stays.
template <int L>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
#pragma unroll
  for (int o = 1; o < L; o <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  return v;
}

}  // namespace

// TPR: lanes per row; R: pieces of 16 bytes per lane.  ANY: buffers or widths
// not in whole aligned pieces; the row's last piece then goes by elements.
template <typename T, int TPR, int R, bool ANY>
__global__ __launch_bounds__(256) void rmsnorm_kernel(RmsNormArgs a) {
  constexpr int N = Vec<T>::N, RPB = 256 / TPR, BL = 128 / N;  // BL: lanes of a 128-channel block
  const int lane = threadIdx.x % TPR;
  const long t = (long)blockIdx.x * RPB + threadIdx.x / TPR;
  const bool on = TPR == 256 || t < a.tokens;
  const long row = on ? t : 0;  // (lanes past the last row read row 0 and write nothing)
  const T* x = (const T*)a.x + row * a.x_ld;
  const T* res = (const T*)a.resid + row * a.resid_ld;
  const int C = a.C;

  float h[R][N];
  {
    uint4 xv[R], rv[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int c = (i * TPR + lane) * N;
      xv[i] = make_uint4(0, 0, 0, 0);
      if (c + N <= C) xv[i] = load_piece<ANY>(x + c);
    }
    if (a.resid)
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const int c = (i * TPR + lane) * N;
        rv[i] = make_uint4(0, 0, 0, 0);
        if (c + N <= C) rv[i] = load_piece<ANY>(res + c);
      }
#pragma unroll
    for (int i = 0; i < R; ++i) unpack(xv[i], h[i]);
    if (a.resid)
#pragma unroll
      for (int i = 0; i < R; ++i) {
        float rf[N];
        unpack(rv[i], rf);
#pragma unroll
        for (int e = 0; e < N; ++e) h[i][e] += rf[e];
      }
    if constexpr (ANY) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const int c = (i * TPR + lane) * N;
        if (c < C && c + N > C)
#pragma unroll
          for (int e = 0; e < N - 1; ++e)
            if (c + e < C) h[i][e] = to_f(x[c + e]) + (a.resid ? to_f(res[c + e]) : 0.f);
      }
    }
  }

  __shared__ float part[2][4];
  __shared__ uint32_t partm[4];
  // the row's sum of squares of f * h (the same in all its lanes)
  auto squares = [&](auto scaled, float f) __attribute__((always_inline)) {
    constexpr bool S = decltype(scaled)::value;
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float v = S ? h[i][e] * f : h[i][e];
        sq = fmaf(v, v, sq);
      }
#pragma unroll
    for (int o = 1; o < (TPR < 64 ? TPR : 64); o <<= 1) sq += __shfl_xor(sq, o, 64);
    if constexpr (TPR == 256) {
      if ((threadIdx.x & 63) == 0) part[S][threadIdx.x >> 6] = sq;
      __syncthreads();
      sq = (part[S][0] + part[S][1]) + (part[S][2] + part[S][3]);
    }
    return sq;
  };
  // A row whose squares pass fp32's range (values of 2^57 and more) is summed
  // again 2^80 times smaller, eps with it; its norm is undone in two steps.
  constexpr float DOWN = 0x1p-80f;
  float sq = squares(std::false_type{}, 1.f), eps = a.eps;
  const bool large = sq == INFINITY;  // (the same in all lanes of a row)
  if (large) {
    sq = squares(std::true_type{}, DOWN);
    eps = eps * DOWN * DOWN;
  }
  const float rstd = 1.0f / sqrtf(sq / (float)C + eps);

  if (a.sum && on) {
    T* sum = (T*)a.sum + row * a.sum_ld;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int c = (i * TPR + lane) * N;
      if (c + N <= C) {
        store_piece<ANY>(sum + c, pack(h[i]));
      } else if constexpr (ANY) {
#pragma unroll
        for (int e = 0; e < N - 1; ++e)
          if (c + e < C) sum[c + e] = from_f<T>(h[i][e]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int c = (i * TPR + lane) * N;
#pragma unroll
    for (int e = 0; e < N; ++e) h[i][e] *= rstd;
    if (large)
#pragma unroll
      for (int e = 0; e < N; ++e) h[i][e] *= DOWN;
    if (a.gamma) {
      if (c + N <= C) {
        float g[N];
#pragma unroll
        for (int e = 0; e < N; e += 4) {
          float g4[4];
          unpack(load_piece<ANY>(a.gamma + c + e), g4);
#pragma unroll
          for (int u = 0; u < 4; ++u) g[e + u] = g4[u];
        }
#pragma unroll
        for (int e = 0; e < N; ++e) h[i][e] *= g[e];
      } else if constexpr (ANY) {
#pragma unroll
        for (int e = 0; e < N - 1; ++e)
          if (c + e < C) h[i][e] *= a.gamma[c + e];
      }
    }
  }

  if (!a.y8) {
    if (!on) return;
    T* y = (T*)a.y + row * a.y_ld;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int c = (i * TPR + lane) * N;
      if (c + N <= C) {
        store_piece<ANY>(y + c, pack(h[i]));
      } else if constexpr (ANY) {
#pragma unroll
        for (int e = 0; e < N - 1; ++e)
          if (c + e < C) y[c + e] = from_f<T>(h[i][e]);
      }
    }
    return;
  }
  // e4m3: several blocks of 128 channels are each the BL = 128 / N lanes that
  // share a piece index (TPR >= 32, a multiple of BL); one scale's maximum is taken over the row.
  uint32_t top[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    top[i] = 0x0D800000u;  // 2^-100
#pragma unroll
    for (int e = 0; e < N; ++e) top[i] = max(top[i], __float_as_uint(h[i][e]) & 0x7FFFFFFFu);
  }
  const bool grouped = TPR >= 32 && a.blocks > 1;
  if (grouped) {
#pragma unroll
    for (int i = 0; i < R; ++i) top[i] = lanes_max<BL>(top[i]);
  } else {
#pragma unroll
    for (int i = 1; i < R; ++i) top[0] = max(top[0], top[i]);
    top[0] = lanes_max<(TPR < 64 ? TPR : 64)>(top[0]);
    if constexpr (TPR == 256) {
      if ((threadIdx.x & 63) == 0) partm[threadIdx.x >> 6] = top[0];
      __syncthreads();
      top[0] = max(max(partm[0], partm[1]), max(partm[2], partm[3]));
    }
#pragma unroll
    for (int i = 1; i < R; ++i) top[i] = top[0];
  }
  if (!on) return;
  uint8_t* y = (uint8_t*)a.y + row * a.y_ld;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int c = (i * TPR + lane) * N;
    if (c >= C) continue;
    const float s = __uint_as_float(top[i]) / 448.f;
    if (grouped ? lane % BL == 0 : i == 0 && lane == 0) a.scale[row * a.blocks + (grouped ? c / 128 : 0)] = s;
    // y / s: the product with 1 / s is off by up to 1.5 units in the last place, which
    // one step on what it leaves of y mends.  (s infinite: 0, and NaN for infinite y.)
    const float inv = 1.0f / s, by = s == INFINITY ? 0.f : s;
    float v[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float c0 = h[i][e] * inv;
      v[e] = fmaf(fmaf(-c0, by, h[i][e]), inv, c0);
    }
    uint32_t q[N / 4];
#pragma unroll
    for (int e = 0; e < N; e += 4) {
      int p = __builtin_amdgcn_cvt_pk_fp8_f32(v[e], v[e + 1], 0, false);
      q[e / 4] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[e + 2], v[e + 3], p, true);
    }
    if (c + N <= C) {
      if constexpr (ANY && N == 8) {
        U8B u;
        u.w[0] = q[0]; u.w[1] = q[1];
        *(U8B*)(y + c) = u;
      } else if constexpr (ANY) {
        U4B u;
        u.w = q[0];
        *(U4B*)(y + c) = u;
      } else if constexpr (N == 8) {
        *(uint2*)(y + c) = make_uint2(q[0], q[1]);
      } else {
        *(uint32_t*)(y + c) = q[0];
      }
    } else if constexpr (ANY) {
#pragma unroll
      for (int e = 0; e < N - 1; ++e)
        if (c + e < C) y[c + e] = (uint8_t)(q[e / 4] >> (8 * (e % 4)));
    }
  }
}

template <typename T, int TPR, int R>
static void launch_rows(const RmsNormArgs& a, bool any, hipStream_t s) {
  constexpr int RPB = 256 / TPR;
  const unsigned grid = (unsigned)((a.tokens + RPB - 1) / RPB);
  if (any)
    rmsnorm_kernel<T, TPR, R, true><<<grid, 256, 0, s>>>(a);
  else
    rmsnorm_kernel<T, TPR, R, false><<<grid, 256, 0, s>>>(a);
}

// The lanes per row follow the width alone (a row's bits are the same in
// every batch): the fewest that hold it in up to 8 pieces, and a count of
// pieces near the row's own; lanes without a piece still cost their row's time
// (142689 x 16 bf16 to e4m3 with a residual: 4.6 us on 2 lanes, 25.2 on 32;
// 80000 x 320 to e4m3 18.0 on 8, 23.1 on 32, but 50000 x 512 19.3 and 16.9).
template <typename T>
static void launch_width(const RmsNormArgs& a, bool any, hipStream_t s) {
  const int nv = (a.C + Vec<T>::N - 1) / Vec<T>::N;
  if (nv <= (!a.y8 ? 64 : a.blocks == 1 ? 40 : 0)) {
    if (nv <= 2) launch_rows<T, 2, 1>(a, any, s);
    else if (nv <= 4) launch_rows<T, 4, 1>(a, any, s);
    else if (nv <= 8) launch_rows<T, 8, 1>(a, any, s);
    else if (nv <= 16) launch_rows<T, 8, 2>(a, any, s);
    else if (nv <= 24) launch_rows<T, 8, 3>(a, any, s);
    else if (nv <= 40) launch_rows<T, 8, 5>(a, any, s);
    else launch_rows<T, 8, 8>(a, any, s);
  } else if (nv <= 256) {
    if (nv <= 32) launch_rows<T, 32, 1>(a, any, s);
    else if (nv <= 64) launch_rows<T, 32, 2>(a, any, s);
    else if (nv <= 96) launch_rows<T, 32, 3>(a, any, s);
    else if (nv <= 128) launch_rows<T, 32, 4>(a, any, s);
    else if (nv <= 160) launch_rows<T, 32, 5>(a, any, s);
    else if (nv <= 192) launch_rows<T, 32, 6>(a, any, s);
    else launch_rows<T, 32, 8>(a, any, s);
  } else if (nv <= 512) {
    if (nv <= 320) launch_rows<T, 64, 5>(a, any, s);
    else if (nv <= 384) launch_rows<T, 64, 6>(a, any, s);
    else launch_rows<T, 64, 8>(a, any, s);
  } else if (nv <= 768) launch_rows<T, 256, 3>(a, any, s);
  else if (nv <= 1024) launch_rows<T, 256, 4>(a, any, s);
  else if (nv <= 1536) launch_rows<T, 256, 6>(a, any, s);
  else if (nv <= 2048) launch_rows<T, 256, 8>(a, any, s);
  else if constexpr (Vec<T>::N == 4) launch_rows<T, 256, 16>(a, any, s);
}

hipError_t launch_rmsnorm(DType dt, const RmsNormArgs& a, hipStream_t s) {
  if (a.tokens <= 0) return hipSuccess;
  const long el = dt == BF16 ? 2 : 4, yel = a.y8 ? 1 : el;
  const uint64_t piece = (uint64_t)a.x | (uint64_t)a.resid | (uint64_t)a.sum | (uint64_t)a.gamma | (uint64_t)(a.x_ld * el) |
                         (uint64_t)((a.resid ? a.resid_ld : 0) * el) | (uint64_t)((a.sum ? a.sum_ld : 0) * el);
  const uint64_t yp = (uint64_t)a.y | (uint64_t)(a.y_ld * yel);
  const bool any = a.C % 8 != 0 || (piece & 15) || (yp & (a.y8 ? 7 : 15));
  // (a grid holds less than 2^32 threads)
  constexpr long MOST = 1 << 23;
  for (long t = 0; t < a.tokens; t += MOST) {
    RmsNormArgs b = a;
    b.tokens = a.tokens - t < MOST ? a.tokens - t : MOST;
    b.x = (const uint8_t*)a.x + t * a.x_ld * el;
    if (a.resid) b.resid = (const uint8_t*)a.resid + t * a.resid_ld * el;
    if (a.sum) b.sum = (uint8_t*)a.sum + t * a.sum_ld * el;
    b.y = (uint8_t*)a.y + t * a.y_ld * yel;
    if (a.scale) b.scale = a.scale + t * a.blocks;
    if (dt == BF16)
      launch_width<bf16>(b, any, s);
    else
      launch_width<float>(b, any, s);
  }
  return hipGetLastError();
}

}  // namespace sd
