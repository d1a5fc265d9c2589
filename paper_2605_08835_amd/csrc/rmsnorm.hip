// Root-mean-square norm of rows, with the residual's addition and an e4m3
// output with scales.
#include "device_common.h"
#include "kernels.h"

namespace sd {

// One block per row.
template <typename T>
__global__ __launch_bounds__(256) void rmsnorm_kernel(RmsNormArgs a) {
  __shared__ float red[256];
  const long t = blockIdx.x;
  const T* x = (const T*)a.x + t * a.x_ld;
  const T* r = a.resid ? (const T*)a.resid + t * a.resid_ld : nullptr;
  __shared__ float h[RMSNORM_MAX_C];
  float sq = 0.f;
  for (int c = threadIdx.x; c < a.C; c += 256) {
    h[c] = to_f(x[c]) + (r ? to_f(r[c]) : 0.f);
    sq += h[c] * h[c];
  }
  red[threadIdx.x] = sq;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if (threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
    __syncthreads();
  }
  const float rstd = 1.0f / sqrtf(red[0] / a.C + a.eps);
  for (int c = threadIdx.x; c < a.C; c += 256) {
    if (a.sum) ((T*)a.sum)[t * a.sum_ld + c] = from_f<T>(h[c]);
    h[c] = h[c] * rstd * (a.gamma ? a.gamma[c] : 1.f);
    if (!a.y8) ((T*)a.y)[t * a.y_ld + c] = from_f<T>(h[c]);
  }
  if (!a.y8) return;
  __syncthreads();
  for (int b = threadIdx.x; b < a.blocks; b += 256) {
    unsigned top = 0x0D800000u;  // 2^-100
    const int end = min(a.C, (b + 1) * a.group);
    for (int c = b * a.group; c < end; ++c) top = max(top, __float_as_uint(h[c]) & 0x7FFFFFFFu);
    const float s = __uint_as_float(top) / 448.f;
    a.scale[t * a.blocks + b] = s;
    for (int c = b * a.group; c < end; ++c) {
      const int p = __builtin_amdgcn_cvt_pk_fp8_f32(h[c] / s, 0.f, 0, false);
      ((uint8_t*)a.y)[t * a.y_ld + c] = (uint8_t)p;
    }
  }
}

hipError_t launch_rmsnorm(DType dt, const RmsNormArgs& a, hipStream_t s) {
  if (a.tokens <= 0) return hipSuccess;
  if (dt == BF16)
    rmsnorm_kernel<bf16><<<(unsigned)a.tokens, 256, 0, s>>>(a);
  else
    rmsnorm_kernel<float><<<(unsigned)a.tokens, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace sd
