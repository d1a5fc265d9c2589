// Linear layer over a few rows with 4-bit weights in groups along K.
#include "device_common.h"
#include "kernels.h"

namespace sd {

__device__ inline float e4m3_f(uint8_t v) { return __builtin_amdgcn_cvt_f32_fp8((int)v, 0); }

// One wave per output element.
__global__ __launch_bounds__(256) void linear_w4_kernel(LinearW4Args a) {
  const int lane = threadIdx.x & 63;
  const long e = blockIdx.x * 4L + (threadIdx.x >> 6);
  if (e >= (long)a.M * a.N) return;
  const int m = (int)(e / a.N), n = (int)(e % a.N);
  float acc = 0.f;
  for (int k = lane; k < a.K; k += 64) {
    float x;
    if (a.x_type == 0) x = ((const float*)a.x)[m * a.x_ld + k];
    else if (a.x_type == 1) x = (float)((const bf16*)a.x)[m * a.x_ld + k];
    else x = e4m3_f(((const uint8_t*)a.x)[m * a.x_ld + k]) * a.x_scale[(long)m * a.x_blocks + (a.x_blocks > 1 ? k / 128 : 0)];
    if (a.silu_in) x = x / (1.f + expf(-x));
    const int byte = a.w[(long)n * (a.K / 2) + k / 2];
    const int q = k & 1 ? byte >> 4 : byte & 15;
    const long g = (long)n * a.groups + k / a.group;
    const float s = a.scale_f32 ? ((const float*)a.scale)[g] : (float)((const bf16*)a.scale)[g];
    acc += x * s * (float)(q - (a.zero ? (int)a.zero[g] : 8));
  }
  acc = wave_sum(acc);
  if (lane) return;
  if (a.bias) acc += a.bias[n];
  if (a.add) acc += a.add[(long)m * a.N + n];
  if (a.silu_out) acc = acc / (1.f + expf(-acc));
  if (a.out_f32) ((float*)a.out)[m * a.out_ld + n] = acc;
  else ((bf16*)a.out)[m * a.out_ld + n] = (bf16)acc;
}

hipError_t launch_linear_w4(const LinearW4Args& a, hipStream_t s) {
  const long waves = (long)a.M * a.N;
  if (waves <= 0) return hipSuccess;
  if (waves > 0x7FFFFFFFL) return hipErrorInvalidValue;
  linear_w4_kernel<<<(unsigned)((waves + 3) / 4), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace sd
