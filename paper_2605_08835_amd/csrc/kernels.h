// Internal interface between the host runtime and the HIP kernels.
// Activations are NHWC ("rows" = packed CFG rows = images), stored in the
// handle's dtype (fp32 or bf16); statistics, biases and accumulators are fp32.
#pragma once
#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace sd {

enum DType { F32 = 0, BF16 = 1 };
// bf16 storage as seen from host code (the kernels read it as __bf16).
typedef uint16_t bf16_t;

// One K-segment of an implicit-GEMM A operand.  Row m of A is output pixel
// (img, oy, ox) of an Ho x Wo image; column k is (tap, c) with
// tap = k / cin (ky = tap / ks, kx = tap % ks) and input channel c.  The
// element is the input pixel under that tap, after the optional nearest-2x
// upsample, the optional per-(img, channel) affine (GroupNorm) and SiLU, and
// zero outside the image (conv zero padding).  Channels c < c0 come from
// src0, the rest from src1 (the skip concat [h | skip] of the up path).
struct ASeg {
  const void* src0;
  const void* src1;
  const float* scale;  // [imgs, cin] or null
  const float* shift;  // [imgs, cin]
  int c0, c1, cin;     // cin = c0 + c1; c0, c1 multiples of 8
  int ks;              // 1 or 3; 2: one phase of a nearest-2x upsample + 3x3 conv (below)
  int stride;          // 1 or 2
  int up;              // 1: nearest-2x upsample before the conv
  int Hi, Wi, Ho, Wo;  // input (before upsampling) and output sizes
  int K;               // ks * ks * cin
  int silu;
  int py, px;          // ks == 2: output phase (2 y + py, 2 x + px); tap (ty, tx) reads the
                       //   input at (y + py - 1 + ty, x + px - 1 + tx), zero outside
};

// Epilogue: out[m, n] = acc + bias[n] + tbias[row_req... ] + resid[m, n].
struct Epi {
  const float* bias;      // [N] or null
  const float* tbias;     // time bias: tbias[img * tb_ld + tb_off + n], or null
  int tb_ld, tb_off, hw;  // img = m / hw
  const void* resid;      // [M, ldr] in the activation dtype, or null (may equal out)
  int ldr;
  void* out;              // [M, ldo]
  int ldo;
  int out_f32;            // 1: fp32 output regardless of the activation dtype
  int geglu;              // bf16 only: columns packed as 32-blocks [a(16) | gate(16)];
                          // out[m, 16t + u] = (a + b) * GELU(gate + b), ldo = N / 2
  void* vt_out;           // bf16 only: columns n >= vt_col0 are written transposed (no bias),
  int vt_col0, vt_hw;     //   vt_out[(m / vt_hw) * vt_img + (n - vt_col0) * vt_ld + m % vt_hw]
  int vt_ld;
  long vt_img;
  int qcols;              // columns n < qcols are multiplied by qscale before rounding
  float qscale;           //   (attention queries stored in base-2 logit units)
  int phase, ph_h, ph_w;  // phase = 1 + 2 py + px: GEMM row m = (image i, y, x) of an ph_h x ph_w
                          //   grid is output row i (4 ph_h ph_w) + (2 y + py) (2 ph_w) + 2 x + px;
                          //   0: row m is output row m
  const float* rowscale;  // bf16 only: acc -> rowscale[m] * acc before the bias, or null (the
                          //   LayerNorm rstd of input row m when the LN is folded into the weights)
};

struct GemmArgs {
  int M, N, K;       // K = seg[0].K + seg[1].K (seg[1].K = 0 if unused)
  ASeg seg[2];
  const void* B;     // packed weights [N, ldb], K contiguous, activation dtype
  int ldb;
  Epi epi;
  int ksplit;        // >= 1; > 1: K split into ksplit ranges, fp32 partials in
  float* partial;    //   partial[ksplit][M][N], summed in order by a second kernel
};

// bf16 requires N % 4 == 0, 8-byte aligned outputs and ldo, ldr % 4 == 0.
hipError_t launch_gemm(DType dt, const GemmArgs& a, hipStream_t s);

// A GEMM of one contiguous 1x1 source whose rows also get their adapter's part:
//   out[m, n] = bias[n] + sum_k A[m, k] B[n, k] + sum_r (hi + lo)[m, r] up[id(m), n, r]
// with id(m) = index[m / group] (none if outside 0 .. count - 1).
struct AdapterArgs : GemmArgs {
  const bf16_t *hi, *lo;  // [M, rank]
  const bf16_t* up;       // [count, N, rank]
  const int* index;
  int group, count, rank; // rank a multiple of 8
  int row0;               // row 0 of the GEMM is row row0 of hi, lo and the index
  unsigned group_mul, group_shift;  // m / group = umulhi(m, mul) >> shift (group > 1)
};
// bf16; K and N multiples of 8; M K and N K below 2^30; out and ldo at multiples of 16 bytes.
hipError_t launch_gemm_adapters(const AdapterArgs& a, hipStream_t s);
// Split-K factor launch_gemm supports for this bf16 GEMM (1 = no split).
int gemm_ksplit(const GemmArgs& a);

// Attention: O = softmax(Q K^T * scale) V per (img, head).
struct AttnArgs {
  const void* q; long q_ld, q_img;   // Q[img][token][c]: token stride, image stride (elements)
  const void* k; long k_ld, k_img;   // K likewise
  const void* v; long v_ld, v_img;   // V: vt = 0 like K; vt = 1 transposed, V[img][c][token] at
  int vt;                            //    v + img*v_img + c*v_ld + token (bf16 only)
  const int* kv_index;               // kv image of each q image, or null (= same)
  void* o; long o_ld, o_img;
  int imgs, heads, d, Nq, Nk;
  float scale;
  int q_log2;                        // 1: Q already holds q * scale * log2(e) (bf16 only)
};
hipError_t launch_attention(DType dt, const AttnArgs& a, hipStream_t s);
// bf16 head widths the attention kernel is built for: d a multiple of 8
// whose rounding up to 16 is 16..96, 128, 160, 192 or 256.
bool attention_width_ok(int d);

// GroupNorm statistics over up to two channel-concatenated NHWC sources;
// writes per-(img, channel) scale = gamma*rstd and shift = beta - mean*scale.
hipError_t launch_groupnorm_stats(DType dt, const void* src0, int c0, const void* src1, int c1,
                                  int imgs, int hw, int groups, float eps, const float* gamma,
                                  const float* beta, float* partial, float* scale, float* shift,
                                  hipStream_t s);
size_t groupnorm_partial_floats(int imgs, int hw, int cin);
size_t groupnorm_noalloc_floats(int imgs, int hw, int cin);
// The library's own partial-sum array on the current device (a static
// __device__ array of groupnorm_scratch_floats_max() floats; its address is
// looked up once per device) for the entry point that allocates nothing.
size_t groupnorm_scratch_floats_max();
hipError_t groupnorm_scratch(float** out);
// out = act(x * scale + shift) over the concat [src0 | src1] (act = SiLU or identity).
// Statistics and apply in one launch for small images (see
// groupnorm_fused_ok for the shapes it takes).
bool groupnorm_fused_ok(DType dt, int c0, int c1, int hw, int groups);
hipError_t launch_groupnorm_fused(DType dt, const void* src0, int c0, const void* src1, int c1, int imgs, int hw,
                                  int groups, float eps, const float* gamma, const float* beta, int silu, void* out,
                                  hipStream_t s);
hipError_t launch_groupnorm_apply(DType dt, const void* src0, int c0, const void* src1, int c1, int imgs,
                                  int hw, const float* scale, const float* shift, int silu, void* out,
                                  hipStream_t s);

hipError_t launch_layernorm(DType dt, const void* x, void* y, long tokens, int C, const float* gamma,
                            const float* beta, float eps, hipStream_t s);
// Per-token LayerNorm scale: rstd[t] = 1 / sqrt(var_t + eps) (biased variance).
hipError_t launch_layernorm_rstd(DType dt, const void* x, float* rstd, long tokens, int C, float eps,
                                 hipStream_t s);

// y[t, j] = x[t, j] * gelu(x[t, half + j]), j < half; x is [tokens, 2*half].
hipError_t launch_geglu(DType dt, const void* x, void* y, long tokens, int half, hipStream_t s);

// Per-row scalars of a step (device arrays in the workspace).
struct RowMaps {
  const int* row_req;     // [rows]
  const int* row_branch;  // [rows]
  const int* row_ctx;     // [rows]
  const float* row_t;     // [rows]
  const int* req_row_u;   // [n_req]
  const float* req_coef;  // [n_req, 3] = (A, B, w)
};

hipError_t launch_pack_latents(DType dt, const float* lat, void* x0, int rows, int lc, int hw,
                               int cpad, const int* row_req, hipStream_t s);
// e[row, :] = [cos(t f_i) | sin(t f_i)] (+ [pooled | sinusoids of time ids] for add_in)
hipError_t launch_time_inputs(const float* row_t, int rows, int temb_in, float* e,
                              const float* pooled_cond, const float* pooled_uncond,
                              const int* row_req, const int* row_branch, int pooled_dim,
                              const float* time_ids_dev, int n_ids, int id_dim, float* a,
                              hipStream_t s);
// out[m, n] = act_out(sum_k act_in(in[m, k]) W[n, k] + bias[n] + add[m, n]) for a few rows; K % 4 == 0.
hipError_t launch_linear_smallm(DType wdt, const float* in, int M, int K, const void* W,
                                const float* bias, const float* add, float* out, int N,
                                int silu_in, int silu_out, hipStream_t s);
// Rows dst0 .. dst0 + n - 1 of a row-major tensor (row_bytes each, a
// multiple of 16) become copies of rows src_rows[0 .. n - 1].
hipError_t launch_copy_rows(void* base, long row_bytes, int dst0, int n, const int* src_rows, hipStream_t s);
// Output conv (3x3, C -> 4) of each request's rows + CFG combine + DDIM in
// one kernel (bf16): x holds the normalised (GroupNorm + SiLU) rows
// [rows, H, W, C]; w the conv weight packed [4][9 C] (tap-major, channel-
// minor), bias [4].  Request r reads row r and, if req_row_u[r] >= 0, that
// unconditional row; lat_* are [n_req, 4, H, W] fp32.  order (or null)
// lists the requests in launch order.
struct OutArgs {
  const bf16_t* x;
  const bf16_t* w;
  const float* bias;
  const float* lat_in;
  float* lat_out;
  float* eps_out;  // or null
  const int* req_row_u;
  const float* req_coef;  // [n_req, 3] = (A, B, w)
  const int* order;
  int n_req, H, W, C;
  int tiles, P;  // blocks per request, pixels per block: set by the launcher
};
bool out_cfg_ddim_ok(DType dt, int latent_c, int H, int W, int C);
hipError_t launch_out_cfg_ddim(const OutArgs& a, hipStream_t s);
hipError_t launch_cfg_ddim(const float* eps_rows, const float* lat_in, float* lat_out,
                           float* eps_out, int n_req, int lc, int hw, const int* req_row_u,
                           const float* req_coef, hipStream_t s);

// Root-mean-square norm of rows of x (+ resid), see synerdiff_op_rmsnorm.
struct RmsNormArgs {
  const void* x; long x_ld;
  const void* resid; long resid_ld;  // or null
  void* sum; long sum_ld;            // or null
  const float* gamma;                // [C] or null
  float eps;
  long tokens;
  int C;
  int y8;                            // 1: y is e4m3, with scale[t * blocks + b]
  void* y; long y_ld;
  float* scale;
  int blocks;                        // scale blocks per row: 1, or one per 128 channels
};
hipError_t launch_rmsnorm(DType dt, const RmsNormArgs& a, hipStream_t s);
constexpr int RMSNORM_MAX_C = 16384;

// Linear layer over a few rows with 4-bit weights, see synerdiff_op_linear_rows_w4.
struct LinearW4Args {
  const void* x; long x_ld;      // fp32, bf16 or e4m3 rows (x_type 0, 1, 2)
  int x_type;
  const float* x_scale;          // e4m3: [M, x_blocks]
  int x_blocks;                  // 1: one scale a row, else one per 128 k
  int M, K, N;
  const uint8_t* w;              // [N, K / 2]
  int group, groups;             // 32, 64 or 128; ceil(K / group)
  const void* scale; int scale_f32;
  const uint8_t* zero;           // or null (8)
  const float* bias;             // [N] or null
  const float* add;              // [M, N] or null
  int silu_in, silu_out;
  void* out; long out_ld; int out_f32;
};
hipError_t launch_linear_w4(const LinearW4Args& a, hipStream_t s);

// Linear layer with a low-rank adapter per row, see synerdiff_op_linear_adapters.
struct LinearAdaptersArgs {
  const void* x;       // [M, K]
  const void* w;       // [N, K]
  const void *down, *up;  // [count, rank, K], [count, N, rank]
  const float* scale;  // [count] or null
  const int* index;    // one entry per `group` rows
  const float* bias;   // [N] or null
  void* out; long out_ld;
  int M, K, N, rank, count, group;
  float* scratch;
};
hipError_t launch_linear_adapters(DType dt, const LinearAdaptersArgs& a, hipStream_t s);
long linear_adapters_scratch_floats(DType dt, int M, int rank);

// Attention over contexts of their own lengths, see synerdiff_op_cross_attention.
struct CrossArgs {
  const void* q; long q_ld, q_head, q_img;
  const void* k; long k_ld, k_head, k_ctx;
  const void* v; long v_ld, v_head, v_ctx;
  long kv_tokens;
  int n_ctx, max_len;
  const int* kv_start;  // null: padded contexts
  const int* kv_len;    // or null
  const int* kv_index;  // or null
  const uint8_t* mask;  // or null
  void* o; long o_ld, o_head, o_img;
  int n, heads, kv_heads, rep, d, n_q;
  unsigned rep_mul, rep_shift;  // r / rep = umulhi(r, rep_mul) >> rep_shift, r < 2^31 (rep > 1): set by the launcher
  float scale;
  float* scratch;
};
hipError_t launch_cross_attention(DType dt, CrossArgs a, hipStream_t s);
long cross_attention_scratch_floats(DType dt, int n, int heads, int kv_heads, int d, int n_q, int max_len);

// Attention inside texts of their own lengths, see synerdiff_op_text_attention.
struct TextArgs {
  const void* q; long q_ld, q_head, q_img;
  const void* k; long k_ld, k_head, k_img;
  const void* v; long v_ld, v_head, v_img;
  void* o; long o_ld, o_head, o_img;
  long tokens;          // packed rows
  int n, max_len;
  const int* start;     // [n + 1]; null: padded texts
  const int* length;    // padded: [n] or null
  const int* prefix;    // or null
  const uint8_t* mask;  // or null
  const float* bias;    // [heads, 2 reach + 1] or null
  int reach;
  const float* slope;   // [heads] or null
  float cap, scale;     // cap 0: none
  int causal, zero;     // zero: rows of o in no text become 0
  int heads, kv_heads, rep, d;
  int chunk, chunks;    // set by the launcher
};
hipError_t launch_text_attention(DType dt, TextArgs a, hipStream_t s);
bool text_attention_fits(int n, int heads, int kv_heads, int max_len);

}  // namespace sd
