// Linear layer whose rows may each have a low-rank adapter of their own:
//   out[m] = bias + W x[m] + scale[c] up[c] (down[c] x[m]),  c = index[m / group].
//
// Two launches: v = scale[c] down[c] x first, then the layer, which adds up[c] v.
//  * Many rows (bf16): v on MFMAs; then the GEMM of gemm.hip, whose accumulators
//    start with the adapters' part.  v is kept as two bf16 parts (2^-17 of it), so
//    that the second product is one of bf16 MFMAs too.
//  * Few rows (at most 64): bound by the bytes of W and of the adapters in use.
//    A block has 16 outputs of all rows, its waves share out K.  v is fp32; up to
//    64 values of it every block makes for itself, in one launch.
//  * Many rows, fp32: the adapters' part goes to `out` first and is the GEMM's residual.
// A row sees its own adapter only: what others hold, infinities and NaN included,
// does not reach it.
#include <string.h>

#include "device_common.h"
#include "kernels.h"

namespace sd {

namespace {

__device__ __forceinline__ int adapter_of(const LinearAdaptersArgs& a, int m) {
  const int c = a.index[a.group == 1 ? m : m / a.group];
  return c >= 0 && c < a.count ? c : -1;
}

__device__ __forceinline__ f32x16 mfma32(bf16x8 x, bf16x8 y, f32x16 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0);
#else
  return c;
#endif
}
// c + x y^T of 16 bytes a lane: row lane % 16, of 16 bytes' k values times 4 the
// lane / 16-th.  (fp32: the products take one element of every lane at a time.)
__device__ __forceinline__ f32x4 mfma16(bf16x8 x, bf16x8 y, f32x4 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0);
#else
  return c;
#endif
}
__device__ __forceinline__ f32x4 mfma16(f32x4 x, f32x4 y, f32x4 c) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], c, 0, 0, 0);
#endif
  return c;
}
template <typename T> struct Piece;  // 16 bytes
template <> struct Piece<bf16> { typedef bf16x8 type; };
template <> struct Piece<float> { typedef f32x4 type; };

}  // namespace

// ------------------------------------------------------------------ v, few rows
// v of row m and four of its adapter's rows from r0 on, by one wave: lanes share out
// K 8 at a time.  (rank is a multiple of 8.)
template <typename T>
__device__ __forceinline__ float4 down_four(const LinearAdaptersArgs& a, int m, int c, int r0, int lane) {
  constexpr int RW = 4;
  const T* x = (const T*)a.x + (long)m * a.K;
  const T* d = (const T*)a.down + ((long)c * a.rank + r0) * a.K;
  float s[RW];
#pragma unroll
  for (int r = 0; r < RW; ++r) s[r] = 0.f;
  for (int k = lane * 8; k < a.K; k += 512) {
    float xv[8], dv[RW][8];
    load8f(x + k, xv);
#pragma unroll
    for (int r = 0; r < RW; ++r) load8f(d + (long)r * a.K + k, dv[r]);
#pragma unroll
    for (int r = 0; r < RW; ++r)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[r] = fmaf(xv[e], dv[r][e], s[r]);
  }
#pragma unroll
  for (int r = 0; r < RW; ++r) s[r] = wave_sum(s[r]);
  const float f = a.scale ? a.scale[c] : 1.f;
  return make_float4(s[0] * f, s[1] * f, s[2] * f, s[3] * f);
}

// (M rank / 4 is below 2^31.  The grid is bounded, since its threads in x have to stay
// below 2^32: a wave takes several parts of many.)
constexpr unsigned DOWN_BLOCKS = 1u << 20;
template <typename T>
__global__ __launch_bounds__(256) void adapters_down_rows_kernel(LinearAdaptersArgs a) {
  const unsigned per = a.rank / 4, lane = threadIdx.x & 63, all = a.M * per;
  for (unsigned id = blockIdx.x * 4 + (threadIdx.x >> 6); id < all; id += gridDim.x * 4) {
    const int m = id / per, r0 = (id - m * per) * 4, c = adapter_of(a, m);
    if (c < 0) continue;  // (its v is not read)
    const float4 v = down_four<T>(a, m, c, r0, lane);
    if (lane == 0) *(float4*)(a.scratch + (long)m * a.rank + r0) = v;
  }
}

// ------------------------------------------------------------------ v, many rows
// A block has 32 MW rows and RT x 32 of the rank: V^T = down x^T, so that a lane has
// one row's values.  Tiles of 64 k of x and `down` go straight to LDS, two ahead of
// the one that is multiplied; MW waves have 32 rows each, the rest share out a tile's
// k and are summed at the end.  v's two parts go to scratch, [M, rank] each.
// Chunk c (16 bytes) of a tile's row r lies in slot c ^ (r / 2 % 8): fragment reads of
// 16 rows are spread over all banks.  Bound by x's bytes: 196608 x 320, rank 16 32 us, 3.9
// TB/s on inputs that change (20.5 on the same ones, partly from the cache behind the L2s);
// 16384 x 1280, rank 128 24 us (19), where every 64 rows read the adapter anew.  Fragments
// straight from memory, 32 bytes a row at a time, took 33 and 44 us on the same inputs.
template <int MW, int RT>
__global__ __launch_bounds__(256, 2) void adapters_down_kernel(LinearAdaptersArgs a) {
  constexpr int NW = 4, KW = NW / MW, BM = 32 * MW, BR = 32 * RT, NS = 3, XI = MW, DI = RT, LPT = XI + DI, STAGE = (BM + BR) * 64;
  constexpr int PART = (KW - 1) * MW * RT * 16 * 64;  // floats of the partial sums
  __shared__ __attribute__((aligned(1024))) bf16 smem[NS * STAGE > 2 * PART ? NS * STAGE : 2 * PART];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lr = lane & 31, lh = lane >> 5;
  const int wm = wave % MW, wk = wave / MW;
  const int m0 = blockIdx.x * BM, r0 = blockIdx.y * BR, rows = min(BM, a.M - m0);
  const int row_id = lane < rows ? adapter_of(a, m0 + lane) : -1;  // (lane: a row of the block)
  uint64_t left = __ballot(row_id >= 0);
  if (!left) return;
  const int own = __shfl(row_id, wm * 32 + lr, 64);
  const rsrc4 xr = resource((const bf16*)a.x + (long)m0 * a.K, (long)rows * a.K * 2);
  // loads i of a tile: rows 8 (wave + NW i) on, 8 lanes a row
  const int lrow = lane >> 3, slot = lane & 7;
  int xo[XI], dof[DI], kc[XI > DI ? XI : DI];
#pragma unroll
  for (int i = 0; i < (XI > DI ? XI : DI); ++i) {
    const int r = 8 * (wave + NW * i) + lrow, c = (slot ^ (r >> 1 & 7)) * 8;
    kc[i] = c;
    if (i < XI) xo[i] = r < rows ? (r * a.K + c) * 2 : OOB;
    if (i < DI) dof[i] = r0 + r < a.rank ? (r * a.K + c) * 2 : OOB;
  }
  const int tiles = (a.K + 63) / 64;
  for (unsigned turn = 0; left; ++turn) {  // (adapters in order of their first rows; blocks in z share them out)
    const int cur = __builtin_amdgcn_readlane(row_id, __builtin_ctzll(left));
    left &= ~__ballot(row_id == cur);
    if (turn % gridDim.z != blockIdx.z) continue;
    const rsrc4 dr = resource((const bf16*)a.down + ((long)cur * a.rank + r0) * a.K, (long)(a.rank - r0) * a.K * 2);
    auto issue = [&](int t, int stage) __attribute__((always_inline)) {  // (past the last tile: zeros)
      bf16* to = smem + stage * STAGE;
      const int k0 = 64 * t;
#pragma unroll
      for (int i = 0; i < XI; ++i) to_lds16(xr, to + 512 * (wave + NW * i), k0 + kc[i] < a.K && xo[i] >= 0 ? xo[i] + 2 * k0 : OOB);
#pragma unroll
      for (int i = 0; i < DI; ++i)
        to_lds16(dr, to + BM * 64 + 512 * (wave + NW * i), k0 + kc[i] < a.K && dof[i] >= 0 ? dof[i] + 2 * k0 : OOB);
    };
    f32x16 acc[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[t][i] = 0.f;
#pragma unroll
    for (int t = 0; t < NS - 1; ++t) issue(t, t);
    int st = 0;
    for (int t = 0; t < tiles; ++t) {
      wait_vmcnt<(NS - 2) * LPT>();
      stage_barrier();
      issue(t + NS - 1, st == 0 ? NS - 1 : st - 1);
      const bf16 *X = smem + st * STAGE + wm * 32 * 64, *D = smem + st * STAGE + BM * 64;
      bf16x8 xf[4 / KW], df[4 / KW][RT];
#pragma unroll
      for (int j = 0; j < 4 / KW; ++j) {
        const int c = ((2 * (wk + KW * j) + lh) ^ (lr >> 1 & 7)) * 8;
        xf[j] = *(const bf16x8*)(X + lr * 64 + c);
#pragma unroll
        for (int u = 0; u < RT; ++u) df[j][u] = *(const bf16x8*)(D + (32 * u + lr) * 64 + c);
      }
#pragma unroll
      for (int j = 0; j < 4 / KW; ++j)
#pragma unroll
        for (int u = 0; u < RT; ++u) acc[u] = mfma32(df[j][u], xf[j], acc[u]);
      wait_lgkm0();
      st = st == NS - 1 ? 0 : st + 1;
    }
    wait_vmcnt<0>();
    stage_barrier();
    float* part = (float*)smem;
    if (wk > 0)
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) part[(((wk - 1) * MW + wm) * RT * 16 + t * 16 + i) * 64 + lane] = acc[t][i];
    wait_lgkm0();
    stage_barrier();
    if (wk == 0) {
#pragma unroll 1
      for (int w = 0; w < KW - 1; ++w)
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[t][i] += part[((w * MW + wm) * RT * 16 + t * 16 + i) * 64 + lane];
      if (own == cur) {
        const float f = a.scale ? a.scale[cur] : 1.f;
        bf16 *hi = (bf16*)a.scratch + (long)(m0 + wm * 32 + lr) * a.rank, *lo = hi + (long)a.M * a.rank;
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int r = r0 + 32 * t + 8 * q + 4 * lh;
            if (r < a.rank) {
              bf16x4 h, l;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                // (bf16's largest value is the first part of what lies past it; an infinity is whole in it)
                const float v = acc[t][4 * q + e] * f;
                h[e] = (bf16)(odd_f(v) ? v : fminf(fmaxf(v, -0x1.FEp127f), 0x1.FEp127f));
                l[e] = (bf16)(odd_f(v) ? 0.f : v - (float)h[e]);
              }
              *(bf16x4*)(hi + r) = h;
              *(bf16x4*)(lo + r) = l;
            }
          }
      }
    }
    wait_lgkm0();
    stage_barrier();  // (the next adapter's tiles take the place of the partial sums)
  }
}

// ------------------------------------------------------------------ few rows
// A block has 16 outputs of all rows (MT x 16), its 8 waves share out K 128 bytes at
// a time and are summed in order.  OWN: it makes v itself (at most OWN_V values),
// beside the others' loads: 1 row, bf16 1280 x 1280, rank 16 in one launch of 6.0 us
// (10.5 a call) against two of 2.9 and 4.3 (14.4 a call).
constexpr int OWN_V = 64;
template <typename T, int MT, bool OWN>
__global__ __launch_bounds__(512) void adapters_rows_kernel(LinearAdaptersArgs a) {
  typedef typename Piece<T>::type P;
  constexpr int NW = 8, E = 16 / sizeof(T), STEP = 4 * E, U = 2;  // elements of a piece; k of a product; products a turn
  __shared__ float part[NW][MT][256];
  __shared__ __attribute__((aligned(16))) float own_v[OWN ? OWN_V : 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lr = lane & 15, lk = E * (lane >> 4);
  const int n0 = blockIdx.x * 16, el = (int)sizeof(T);
  const __amdgpu_buffer_rsrc_t wr = make_rsrc((const T*)a.w + (long)n0 * a.K, (long)min(16, a.N - n0) * a.K * el);
  const __amdgpu_buffer_rsrc_t xr = make_rsrc(a.x, (long)a.M * a.K * el);
  f32x4 acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int k0 = wave * U * STEP; k0 < a.K; k0 += NW * U * STEP) {
    P wv[U], xv[U][MT];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int k = k0 + STEP * j + lk;
      wv[j] = __builtin_bit_cast(P, buf_load16(wr, k < a.K ? (lr * a.K + k) * el : OOB));
#pragma unroll
      for (int t = 0; t < MT; ++t) xv[j][t] = __builtin_bit_cast(P, buf_load16(xr, k < a.K ? ((16 * t + lr) * a.K + k) * el : OOB));
    }
#pragma unroll
    for (int j = 0; j < U; ++j)
#pragma unroll
      for (int t = 0; t < MT; ++t) acc[t] = mfma16(wv[j], xv[j][t], acc[t]);  // (outputs 4 (lane / 16) + i of row lane % 16)
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) *(f32x4*)&part[wave][t][4 * lane] = acc[t];
  if constexpr (OWN) {
    const int per = a.rank / 4;
    for (int id = wave; id < a.M * per; id += NW) {
      const int m = id / per, r0 = (id - m * per) * 4, c = adapter_of(a, m);
      if (c < 0) continue;
      const float4 v = down_four<T>(a, m, c, r0, lane);
      if (lane == 0) *(float4*)(own_v + m * a.rank + r0) = v;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < MT * 256; i += 512) {
    // element i % 4 of lane i / 4: output 4 (lane / 16) + i % 4, row lane % 16
    const int t = i >> 8, at = i & 255, m = 16 * t + (at >> 2 & 15), n = n0 + 4 * (at >> 6) + (at & 3);
    if (m >= a.M || n >= a.N) continue;
    float s = a.bias ? a.bias[n] : 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) s += part[w][t][at];
    const int c = adapter_of(a, m);
    if (c >= 0) {
      const float* v = OWN ? own_v + m * a.rank : a.scratch + (long)m * a.rank;
      const T* u = (const T*)a.up + ((long)c * a.N + n) * a.rank;
      for (int r = 0; r < a.rank; r += 8) {
        float uv[8], vv[8];
        load8f(u + r, uv);
        load8f(v + r, vv);
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(uv[e], vv[e], s);
      }
    }
    ((T*)a.out)[(long)m * a.out_ld + n] = from_f<T>(s);
  }
}

// ------------------------------------------------------------------ many rows, fp32: the adapters' part
// A block has 8 rows, a thread per output column of all 8; rows of one adapter share
// the loads of its `up`.  OWN: the block makes their v first; else it comes from
// scratch, and blocks in y share out the columns.  Bound by latencies one after another
// (index, x and down, up): 6144 x 320 x 320, rank 8 17 us for 8 MB of `out`.
constexpr int F32_ROWS = 8;
template <bool OWN>
__global__ __launch_bounds__(256) void adapters_f32_kernel(LinearAdaptersArgs a) {
  constexpr int MR = F32_ROWS;
  extern __shared__ __attribute__((aligned(16))) float own_v[];  // [MR, rank]
  const int m0 = blockIdx.x * MR, rows = min(MR, a.M - m0), lane = threadIdx.x & 63, wave = threadIdx.x >> 6, per = a.rank / 4;
  const float* v = OWN ? own_v : a.scratch + (long)m0 * a.rank;
  if constexpr (OWN)
    for (int id = wave; id < rows * per; id += 4) {
      const int i = id / per, r0 = (id - i * per) * 4, c = adapter_of(a, m0 + i);
      if (c < 0) continue;
      const float4 f = down_four<float>(a, m0 + i, c, r0, lane);
      if (lane == 0) *(float4*)(own_v + i * a.rank + r0) = f;
    }
  int c[MR], all = 0;
#pragma unroll
  for (int i = 0; i < MR; ++i) {
    c[i] = i < rows ? adapter_of(a, m0 + i) : -1;
    all |= (c[i] >= 0) << i;
  }
  __syncthreads();
  for (int n = blockIdx.y * 256 + threadIdx.x; n < a.N; n += 256 * gridDim.y) {
    float s[MR];
#pragma unroll
    for (int i = 0; i < MR; ++i) s[i] = 0.f;
    for (int left = all; left;) {
      int cur = -1, mine = 0;
#pragma unroll
      for (int i = MR - 1; i >= 0; --i)
        if (left >> i & 1) cur = c[i];
#pragma unroll
      for (int i = 0; i < MR; ++i) mine |= (c[i] == cur) << i;
      left &= ~mine;
      const float* u = (const float*)a.up + ((long)cur * a.N + n) * a.rank;
      for (int r = 0; r < a.rank; r += 4) {
        const float4 uv = *(const float4*)(u + r);
#pragma unroll
        for (int i = 0; i < MR; ++i)
          if (mine >> i & 1) {
            const float4 vv = *(const float4*)(v + i * a.rank + r);
            s[i] = fmaf(uv.x, vv.x, fmaf(uv.y, vv.y, fmaf(uv.z, vv.z, fmaf(uv.w, vv.w, s[i]))));
          }
      }
    }
#pragma unroll
    for (int i = 0; i < MR; ++i)
      if (i < rows) ((float*)a.out)[(long)(m0 + i) * a.out_ld + n] = s[i];
  }
}

// ------------------------------------------------------------------ launch
constexpr int FEW = 64;  // rows the few-row kernel is built for
// fp32 blocks make their own v where they fill the card and the ranks are low, else a
// launch of its own does (whole calls, us, own and two launches: 65 x 1280 x 1280, rank
// 128 180 and 58; 1024 x 320 x 320, rank 8 22.7 and 20.8; 2048 rows 29.9 and 29.4, 6144
// 39.9 and 42.1; 2048 x 1280 x 640, rank 64 160 and 141).
static bool f32_own(int M, int rank) { return M >= 256 * F32_ROWS && rank <= 16; }

long linear_adapters_scratch_floats(DType dt, int M, int rank) {
  if (M <= FEW) return (long)M * rank <= OWN_V ? 0 : (long)M * rank;
  return dt != BF16 && f32_own(M, rank) ? 0 : (long)M * rank;
}

// 64 rows a block for many rows, else 32 (whole calls, us, 32 and 64: 8192 x 640, rank
// 16 18.9 and 19.0; 12288 x 1280, rank 64 59.6 and 57.8; 32768 x 320, rank 128 58.9 and
// 40.4; 4096 x 1280, rank 32 30.8 and 31.5).  An index per row may bring several
// adapters to a block: 4 blocks share them out then (one, and four: 1872 x 768, rank 16,
// in runs of 40 rows 15.9 and 13.1, in one run 12.6 and 12.5; 512 x 320, rank 32, every row
// another 28.3 and 16.6; 12288 x 320, rank 16, in runs of 40 20.0 and 17.1, every row
// another 36.8 and 25.5, in one run 14.9 and 14.8; 32768 x 640, rank 32, in runs of 40
// 59 and 55, in one run 43.9 and 43.7), up to 32768 rows (196608 x 320, rank 16, in runs of
// 40 126 and 138, of 4096 112 and 116).
template <int RT>
static void launch_down(const LinearAdaptersArgs& a, hipStream_t s) {
  const unsigned y = (unsigned)((a.rank + 32 * RT - 1) / (32 * RT));
  if (a.M <= 8192)
    adapters_down_kernel<1, RT><<<dim3((unsigned)((a.M + 31) / 32), y, a.group < 32 ? 4 : 1), 256, 0, s>>>(a);
  else
    adapters_down_kernel<2, RT><<<dim3((unsigned)((a.M + 63) / 64), y, a.group < 32 && a.M <= 32768 ? 4 : 1), 256, 0, s>>>(a);
}

// (What reads v is not launched where v was not.)
template <typename T>
static hipError_t launch_down_rows(const LinearAdaptersArgs& a, hipStream_t s) {
  const long blocks = ((long)a.M * (a.rank / 4) + 3) / 4;
  adapters_down_rows_kernel<T><<<dim3(blocks < DOWN_BLOCKS ? (unsigned)blocks : DOWN_BLOCKS), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}

template <typename T, int MT>
static hipError_t launch_few(const LinearAdaptersArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.N + 15) / 16));
  if ((long)a.M * a.rank <= OWN_V)
    adapters_rows_kernel<T, MT, true><<<grid, 512, 0, s>>>(a);
  else {
    const hipError_t e = launch_down_rows<T>(a, s);
    if (e != hipSuccess) return e;
    adapters_rows_kernel<T, MT, false><<<grid, 512, 0, s>>>(a);
  }
  return hipGetLastError();
}
template <typename T>
static hipError_t launch_rows(const LinearAdaptersArgs& a, hipStream_t s) {
  if (a.M <= 16) return launch_few<T, 1>(a, s);
  if (a.M <= 32) return launch_few<T, 2>(a, s);
  return launch_few<T, 4>(a, s);
}

static hipError_t launch_bf16(const LinearAdaptersArgs& a, hipStream_t s) {
  if (a.rank <= 32) launch_down<1>(a, s);
  else if (a.rank <= 64) launch_down<2>(a, s);
  else launch_down<4>(a, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // (rows in parts whose offsets fit 32 bits)
  const long widest = a.K > a.rank ? a.K : a.rank;
  const long step = ((1L << 30) - 1) / widest / 256 * 256;
  for (long m0 = 0; m0 < a.M; m0 += step) {
    AdapterArgs g;
    memset(&g, 0, sizeof(g));
    g.M = (int)(a.M - m0 < step ? a.M - m0 : step);
    g.N = a.N;
    g.K = a.K;
    ASeg& seg = g.seg[0];
    seg.src0 = (const bf16_t*)a.x + m0 * a.K;
    seg.c0 = seg.cin = seg.K = a.K;
    seg.ks = seg.stride = 1;
    seg.Hi = seg.Ho = 1;
    seg.Wi = seg.Wo = g.M;
    g.B = a.w;
    g.ldb = a.K;
    g.epi.bias = a.bias;
    g.epi.out = (bf16_t*)a.out + m0 * a.out_ld;
    g.epi.ldo = (int)a.out_ld;
    g.hi = (const bf16_t*)a.scratch;
    g.lo = g.hi + (long)a.M * a.rank;
    g.up = (const bf16_t*)a.up;
    g.index = a.index;
    g.group = a.group;
    g.count = a.count;
    g.rank = a.rank;
    g.row0 = (int)m0;
    const hipError_t e = launch_gemm_adapters(g, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

static hipError_t launch_f32(const LinearAdaptersArgs& a, hipStream_t s) {
  const unsigned blocks = (unsigned)((a.M + F32_ROWS - 1) / F32_ROWS);
  if (f32_own(a.M, a.rank)) {
    adapters_f32_kernel<true><<<dim3(blocks), 256, (unsigned)(F32_ROWS * a.rank * 4), s>>>(a);
  } else {
    const hipError_t e = launch_down_rows<float>(a, s);
    if (e != hipSuccess) return e;
    adapters_f32_kernel<false><<<dim3(blocks, (unsigned)((a.N + 255) / 256)), 256, 0, s>>>(a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  GemmArgs g;
  memset(&g, 0, sizeof(g));
  g.M = a.M;
  g.N = a.N;
  g.K = a.K;
  ASeg& seg = g.seg[0];
  seg.src0 = a.x;
  seg.c0 = seg.cin = seg.K = a.K;
  seg.ks = seg.stride = 1;
  seg.Hi = seg.Ho = 1;
  seg.Wi = seg.Wo = a.M;
  g.B = a.w;
  g.ldb = a.K;
  g.epi.bias = a.bias;
  g.epi.hw = 1;
  g.epi.resid = a.out;
  g.epi.ldr = (int)a.out_ld;
  g.epi.out = a.out;
  g.epi.ldo = (int)a.out_ld;
  g.epi.out_f32 = 1;
  g.ksplit = 1;
  return launch_gemm(F32, g, s);
}

hipError_t launch_linear_adapters(DType dt, const LinearAdaptersArgs& a, hipStream_t s) {
  if (a.M <= 0 || a.N <= 0) return hipSuccess;
  // (33 to 64 rows of more than 2048 bf16 channels are better off in tiles: 64 x 4096
  // x 4096 18 us against 23; 64 x 1280 x 1280 13.5 against 13.2)
  if (a.M <= 32 || (a.M <= FEW && (dt != BF16 || a.K <= 2048))) return dt == BF16 ? launch_rows<bf16>(a, s) : launch_rows<float>(a, s);
  return dt == BF16 ? launch_bf16(a, s) : launch_f32(a, s);
}

}  // namespace sd
