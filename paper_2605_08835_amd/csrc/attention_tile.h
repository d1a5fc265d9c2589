// What the attention kernels over texts share: their softmax's constants and the
// pieces of a 32-row MFMA tile whose scores are held transposed (a lane has one row).
#pragma once
#include "device_common.h"

namespace sd {
namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float TAU = 8.0f;  // the running maximum moves when a tile's passes it by this much (log2 units)

// What a row's exponents are taken against: its running maximum, or 0 as long as
// every key so far scored -inf (then every p is 0; -inf minus -inf is NaN).
__device__ __forceinline__ float exp_ref(float m) { return m == -INFINITY ? 0.f : m; }

__device__ __forceinline__ float2 half_swap(float v) {  // (v of lanes l and l ^ 32)
#if defined(__HIP_DEVICE_COMPILE__)
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
#else
  return make_float2(v, v);
#endif
}

// Four keys (LDS rows) of one channel for each lane of a group of 16: lane i
// names the 8 bytes of row i / 4, channels 4 (i % 4) on, and gets channel i of rows 0 to 3.
__device__ __forceinline__ bf16x4 read_transposed(const bf16* p) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p));
#else
  return *(const bf16x4*)p;
#endif
}

// l + the eight rounded probabilities, two to an instruction (taking them apart
// again cost three each, a third of a 64-key tile's vector instructions).
__device__ __forceinline__ float sum_probs(bf16x8 p, float l) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 one = {(bf16)1.0f, (bf16)1.0f};
  l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p, p, 0, 1), one, l, false);
  l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p, p, 2, 3), one, l, false);
  l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p, p, 4, 5), one, l, false);
  l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p, p, 6, 7), one, l, false);
#endif
  return l;
}

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
#else
  return c;
#endif
}

__device__ __forceinline__ f32x16 mfma_f32(float a, float b, f32x16 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
#else
  return c;
#endif
}

}  // namespace
}  // namespace sd
