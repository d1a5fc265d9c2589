// Attention of each row's queries over a text of its own length.
#include "device_common.h"
#include "kernels.h"

namespace sd {

// The rows of K / V that row `img` reads: first row, count and the mask bytes from the first row on.
struct Text {
  long k0, v0;   // element offset of key 0 (without the head)
  long m0;       // mask byte of key 0
  int len;       // 0: nothing to read
};
__device__ inline Text text_of(const CrossArgs& a, int img) {
  Text t = {0, 0, 0, 0};
  const int c = a.kv_index ? a.kv_index[img] : img;
  if (c < 0 || c >= a.n_ctx) return t;
  int len = a.kv_len ? a.kv_len[c] : a.max_len;
  len = min(max(len, 0), a.max_len);
  if (a.kv_start) {
    long start = a.kv_start[c];
    if (start < 0 || start >= a.kv_tokens) return t;
    len = (int)min((long)len, a.kv_tokens - start);
    t.k0 = start * a.k_ld;
    t.v0 = start * a.v_ld;
    t.m0 = start;
  } else {
    t.k0 = c * a.k_ctx;
    t.v0 = c * a.v_ctx;
    t.m0 = (long)c * a.max_len;
  }
  t.len = len;
  return t;
}

// One wave per (row, query, head): lanes over the head's channels.
template <typename T>
__global__ __launch_bounds__(256) void cross_simple_kernel(CrossArgs a) {
  const int lane = threadIdx.x & 63;
  const long e = blockIdx.x * 4L + (threadIdx.x >> 6);
  if (e >= (long)a.n * a.n_q * a.heads) return;
  const int h = (int)(e % a.heads), t = (int)(e / a.heads % a.n_q), img = (int)(e / a.heads / a.n_q);
  const Text tx = text_of(a, img);
  const T* q = (const T*)a.q + img * a.q_img + t * a.q_ld + h * a.q_head;
  const T* k = (const T*)a.k + tx.k0 + (h / a.rep) * a.k_head;
  const T* v = (const T*)a.v + tx.v0 + (h / a.rep) * a.v_head;
  float qv[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
  for (int i = 0; i < 4; ++i) qv[i] = lane + 64 * i < a.d ? to_f(q[lane + 64 * i]) * a.scale : 0.f;
  for (int j = 0; j < tx.len; ++j) {
    if (a.mask && !a.mask[tx.m0 + j]) continue;
    float s = 0.f;
    for (int i = 0; i < 4; ++i)
      if (lane + 64 * i < a.d) s += qv[i] * to_f(k[j * a.k_ld + lane + 64 * i]);
    s = wave_sum(s);
    const float mn = fmaxf(m, s), al = expf(m - mn), p = expf(s - mn);
    l = l * al + p;
    for (int i = 0; i < 4; ++i)
      if (lane + 64 * i < a.d) o[i] = o[i] * al + p * to_f(v[j * a.v_ld + lane + 64 * i]);
    m = mn;
  }
  T* out = (T*)a.o + img * a.o_img + t * a.o_ld + h * a.o_head;
  for (int i = 0; i < 4; ++i)
    if (lane + 64 * i < a.d) out[lane + 64 * i] = from_f<T>(l > 0.f ? o[i] / l : 0.f);
}

long cross_attention_scratch_floats(DType dt, int n, int heads, int kv_heads, int d, int n_q, int max_len) { return 0; }

hipError_t launch_cross_attention(DType dt, const CrossArgs& a, hipStream_t s) {
  const long waves = (long)a.n * a.n_q * a.heads;
  if (waves <= 0) return hipSuccess;
  if (waves > 0x7FFFFFFFL) return hipErrorInvalidValue;
  const unsigned blocks = (unsigned)((waves + 3) / 4);
  if (dt == BF16)
    cross_simple_kernel<bf16><<<blocks, 256, 0, s>>>(a);
  else
    cross_simple_kernel<float><<<blocks, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace sd
