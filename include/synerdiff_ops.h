/*
 * synerdiff_ops.h - kernel-level entry points of the UNet step.
 *
 * Each call runs one of the step's kernels on caller-owned device buffers so
 * that a kernel can be checked on its own against the layer it implements.
 * Conventions as in synerdiff.h: device pointers, the caller's stream,
 * validation before enqueue, SD_ERR_HIP on a launch failure.  `dtype` is
 * SD_F32 or SD_BF16 and types every activation and weight argument; norm
 * statistics, biases and affine parameters are always fp32.
 * Activations are channels-last: [n, H, W, C].
 */
#ifndef SYNERDIFF_OPS_H
#define SYNERDIFF_OPS_H

#include "synerdiff.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Convolution as an implicit GEMM (3x3 or 1x1 layers of the UNet):
 *   out[i, y, x, o] = bias[o] + resid[i, y, x, o]
 *       + sum_{ky, kx, c} A(i, s*y + ky - p, s*x + kx - p, c) * w[o, (ky*ks + kx)*cin + c]
 * with p = (ks - 1) / 2, cin = c0 + c1, A the channel concat [x0 | x1]
 * (x1 may be NULL with c1 = 0), optionally nearest-2x upsampled first
 * (up = 1), optionally transformed per (image, channel) as
 * v * scale + shift (GroupNorm affine; scale/shift [n, cin] fp32 or NULL)
 * and then SiLU (silu = 1), and zero outside the image (zero padding after
 * the transform).  Output size: H/stride (stride 2 needs even H, W) or 2H
 * when upsampling.  w is the packed weight [cout, ks*ks*cin] (tap-major,
 * channel-minor).  bias may be NULL; resid ([n, Ho, Wo, cout], activation
 * dtype) may be NULL or equal to out.  out_f32 = 1 writes fp32 output.
 * d_scratch (fp32, scratch_floats long, may be NULL) lets the call split K
 * the way the step does for long-K 3x3 layers on small images (ks = 1 never
 * splits);
 * synerdiff_op_conv_scratch_floats returns the floats that needs (0 = no
 * split for this shape).
 * Constraints: ks in {1, 3}; stride in {1, 2}; c0, c1 multiples of 8;
 * bf16: cout a multiple of 4. */
sd_status synerdiff_op_conv(int32_t dtype, const void* d_x0, int32_t c0, const void* d_x1, int32_t c1,
                            int32_t n, int32_t H, int32_t W, int32_t ks, int32_t stride, int32_t up,
                            const float* d_scale, const float* d_shift, int32_t silu, const void* d_w,
                            int32_t cout, const float* d_bias, const void* d_resid, void* d_out,
                            int32_t out_f32, float* d_scratch, int64_t scratch_floats, void* hip_stream);
int64_t synerdiff_op_conv_scratch_floats(int32_t dtype, int32_t c0, int32_t c1, int32_t n, int32_t H, int32_t W,
                                         int32_t ks, int32_t stride, int32_t up, int32_t cout);

/* The 3x3 convolution (zero padding 1) of a nearest-2x upsampled input, as
 * the bf16 step runs the UNet's upsampling layers: four 2x2 convolutions on
 * the input grid, one per output phase.  Output pixel (2y + py, 2x + px)
 * = bias + sum over taps (ty, tx) in {0,1}^2 and channels c of
 * x[y + py - 1 + ty, x + px - 1 + tx, c] (zero outside) * w[2 py + px, o, 2 ty + tx, c],
 * where phase weight (ty, tx) is the sum of the 3x3 taps (ky, kx) with
 * floor((py + ky - 1) / 2) = py - 1 + ty and floor((px + kx - 1) / 2) =
 * px - 1 + tx.  x [n, H, W, cin] and out [n, 2H, 2W, cout] bf16, w bf16
 * [4][cout][4 cin], bias fp32 [cout] or NULL.  dtype must be SD_BF16;
 * cin a multiple of 32, cout of 160 (else SD_ERR_INVALID_ARG). */
sd_status synerdiff_op_upconv(int32_t dtype, const void* d_x, int32_t n, int32_t H, int32_t W, int32_t cin,
                              const void* d_w, int32_t cout, const float* d_bias, void* d_out, void* hip_stream);

/* Multi-head attention O = softmax(Q K^T * scale) V per image and head
 * (head h uses channels [h*d, (h+1)*d)).  Q: image i, token t, channel c at
 * q + i*q_img + t*q_ld + c; K likewise with k_img, k_ld and image
 * kv_index[i] (d_kv_index NULL = image i); V likewise with v_img, v_ld
 * (fp32), or, with v_transposed = 1 (required for bf16), at
 * v + j*v_img + c*v_ld + t (channel-major, the layout the step's
 * projections write); O like Q with o_img, o_ld.  Strides in elements.
 * q_log2 = 1: Q already holds q * scale * log2(e), as the step's bf16
 * projections write it (scale is then unused).  Constraints: d a multiple
 * of 8; bf16: d rounded up to 16 is 16..96, 128, 160, 192 or 256; fp32:
 * d <= 256 (V row-major).  bf16 reads Q and K in 16-byte and writes O in
 * 8-byte pieces: start their rows at multiples of those (O rows at multiples
 * of 16 bytes leave in 16-byte pieces). */
sd_status synerdiff_op_attention(int32_t dtype, const void* d_q, int64_t q_ld, int64_t q_img,
                                 const void* d_k, int64_t k_ld, int64_t k_img, const void* d_v,
                                 int64_t v_ld, int64_t v_img, int32_t v_transposed,
                                 const int32_t* d_kv_index, void* d_o, int64_t o_ld, int64_t o_img,
                                 int32_t n, int32_t heads, int32_t d, int32_t n_q, int32_t n_k,
                                 float scale, int32_t q_log2, void* hip_stream);

/* GroupNorm statistics of the concat [x0 | x1] ([n, hw, c0 + c1]) with
 * `groups` groups of consecutive channels, biased variance, eps: writes the
 * per-(image, channel) affine scale = gamma * rstd, shift = beta - mean *
 * scale (fp32 [n, cin]) that synerdiff_op_conv applies.  d_partial is
 * scratch of synerdiff_op_groupnorm_scratch_floats(n, hw, cin) floats. */
size_t synerdiff_op_groupnorm_scratch_floats(int32_t n, int32_t hw, int32_t cin);
sd_status synerdiff_op_groupnorm_stats(int32_t dtype, const void* d_x0, int32_t c0, const void* d_x1,
                                       int32_t c1, int32_t n, int32_t hw, int32_t groups, float eps,
                                       const float* d_gamma, const float* d_beta, float* d_partial,
                                       float* d_scale, float* d_shift, void* hip_stream);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc):
 * synerdiff_op_groupnorm_stats without d_partial.  The partial sums go to a
 * device array the library owns, SYNERDIFF_GN_NOALLOC_SCRATCH_FLOATS floats
 * (16 MiB) per device, held until the process ends; the call itself
 * allocates nothing.  A call whose partial sums exceed that size, counting
 * at most 64 pixel ranges per image (2 (c0 + c1) floats each), returns
 * SD_ERR_CAPACITY before enqueueing anything; one whose partials only exceed
 * it at the finer ranges of larger images runs in several passes, one after
 * the other on the stream.  Every call on a device shares its array: calls
 * that overlap in time on one device (different streams or host threads)
 * race.  Each call writes every partial it reads,
 * so no clearing is needed between calls.  Arguments and outputs as for
 * synerdiff_op_groupnorm_stats. */
#define SYNERDIFF_GN_NOALLOC_SCRATCH_FLOATS (1u << 22)
sd_status synerdiff_op_groupnorm_stats_noalloc(int32_t dtype, const void* d_x0, int32_t c0, const void* d_x1,
                                               int32_t c1, int32_t n, int32_t hw, int32_t groups, float eps,
                                               const float* d_gamma, const float* d_beta, float* d_scale,
                                               float* d_shift, void* hip_stream);

/* GroupNorm of the concat [x0 | x1] ([n, hw, c0 + c1], `groups` groups of
 * consecutive channels, biased variance, eps) followed by SiLU when silu =
 * 1, written to out [n, hw, c0 + c1]: the normalisation in front of every
 * ResBlock conv of the latent-diffusion UNet the paper serves (Sec. IV-A),
 * as the step runs it on its small images, statistics and apply in one
 * kernel (one block per (group, image)).  bf16 only; the channels per group
 * a multiple of 4, c0 and c1 multiples of 4, and hw * (channels per group)
 * / 4 <= 5120 (SD_ERR_UNSUPPORTED otherwise).  gamma, beta fp32 [c0 + c1].
 * n = 0 does nothing. */
sd_status synerdiff_op_groupnorm_fused(int32_t dtype, const void* d_x0, int32_t c0, const void* d_x1, int32_t c1,
                                       int32_t n, int32_t hw, int32_t groups, float eps, const float* d_gamma,
                                       const float* d_beta, int32_t silu, void* d_out, void* hip_stream);

/* LayerNorm over the last axis of x [tokens, C] (biased variance):
 * y = (x - mean) * rstd * gamma + beta.  C a multiple of 8, <= 2048. */
sd_status synerdiff_op_layernorm(int32_t dtype, const void* d_x, void* d_y, int64_t tokens, int32_t C,
                                 const float* d_gamma, const float* d_beta, float eps, void* hip_stream);

/* The LayerNorm scale alone, rstd[t] = 1 / sqrt(var_t + eps) with the
 * biased variance of token t of x [tokens, C] (C a multiple of 8, <= 2048):
 * the per-token factor of the SD transformer blocks' LayerNorms when their
 * mean, gain and shift are folded into the projection weights (the
 * latent-diffusion UNet the paper serves, Sec. IV-A).  rstd is fp32
 * [tokens], device memory owned by the caller; nothing else is written.
 * tokens = 0 does nothing. */
sd_status synerdiff_op_layernorm_rstd(int32_t dtype, const void* d_x, float* d_rstd, int64_t tokens, int32_t C,
                                      float eps, void* hip_stream);

/* Linear layer over a few fp32 rows, the per-request timestep-embedding
 * MLP and time projections of the latent-diffusion UNet the paper serves
 * (Sec. IV-A):
 *   out[m, n] = act_out(bias[n] + add[m, n] + sum_k act_in(in[m, k]) * w[n, k])
 * with act_* = SiLU where silu_* = 1, else the identity.  in [M, K] and out
 * [M, N] fp32 (out must not overlap in; add may equal out), w [N, K] in
 * `dtype`, bias [N] fp32; bias and add may be NULL.  K a multiple of 4;
 * buffers 16-byte aligned.  M = 0 or N = 0 does nothing. */
sd_status synerdiff_op_linear_rows(int32_t dtype, const float* d_in, int32_t M, int32_t K, const void* d_w,
                                   const float* d_bias, const float* d_add, float* d_out, int32_t N,
                                   int32_t silu_in, int32_t silu_out, void* hip_stream);

/* GEGLU: y[t, j] = x[t, j] * GELU(x[t, half + j]) with exact GELU; x is
 * [tokens, 2*half], y [tokens, half]; half a multiple of 8. */
sd_status synerdiff_op_geglu(int32_t dtype, const void* d_x, void* d_y, int64_t tokens, int32_t half,
                             void* hip_stream);

/* The step's last stage as one kernel: the UNet's output convolution, the
 * classifier-free guidance combine and the DDIM update (CFG as in Ho &
 * Salimans 2022; Skip-CFG bypasses the unconditional branch, Sec. II-B and
 * Sec. III-B; DDIM eta = 0, Song et al. 2021).  For request r < n_req and
 * each pixel p, channel o < 4:
 *   eps_c = b[o] + sum_{ky, kx, c} x[r, y + ky - 1, x + kx - 1, c] w[o, (3 ky + kx) C + c]
 *   (zero outside the image); eps_u likewise from row req_row_u[r] when it
 *   is >= 0; eps = eps_u + w_r (eps_c - eps_u) if so, else eps_c;
 *   lat_out[r, o, p] = A_r lat_in[r, o, p] + B_r eps;  eps_out (if not NULL) = eps.
 * x: device bf16 [rows, H, W, C] (rows covering every index used), the
 * normalised (GroupNorm + SiLU) input of the output conv.  w: device bf16
 * [4][9 C] (the layout synerdiff_op_conv takes), bias fp32 [4].
 * d_req_row_u: device int32 [n_req]; d_req_coef: device fp32 [n_req, 3] =
 * (A_r, B_r, w_r).  lat_in, lat_out, eps_out: device fp32 [n_req, 4, H, W]
 * (NCHW); lat_out may equal lat_in, eps_out must not overlap either.
 * dtype must be SD_BF16; C a multiple of 32 and <= 320, W <= 128
 * (SD_ERR_UNSUPPORTED otherwise).  n_req = 0 does nothing. */
sd_status synerdiff_op_conv_out_cfg_ddim(int32_t dtype, const void* d_x, int32_t H, int32_t W, int32_t C,
                                         const void* d_w, const float* d_bias, int32_t n_req,
                                         const int32_t* d_req_row_u, const float* d_req_coef,
                                         const float* d_lat_in, float* d_lat_out, float* d_eps_out,
                                         void* hip_stream);

/* ---- Operators on texts of their own lengths and on few-bit weights ----
 * Further element type of these operators: OCP e4m3 (4 exponent bits, 3
 * fraction bits, largest value 448, no infinities). */
#define SD_E4M3 2

/* Root-mean-square norm over the last axis, with the residual's addition and
 * an 8-bit output when asked for (the norms around a text encoder's or a
 * transformer's sublayers):
 *   h[t, c] = x[t, c] + resid[t, c]        (x alone when resid is NULL)
 *   y[t, c] = h[t, c] / sqrt(mean_c(h[t, c]^2) + eps) * gamma[c]
 * x, resid, sum in `dtype`; row t of each starts at t * its ld (elements, >=
 * C).  h is kept in fp32 for the norm, at any finite size (with eps below
 * 2^-100 a row wants a value of 2^-60 or more: smaller squares vanish); d_sum (may be NULL; NULL without
 * resid) receives it rounded to dtype.  gamma fp32 [C] or NULL (all ones).
 * y_type = dtype: y is rounded to dtype.  y_type = SD_E4M3: per row, or per
 * block of 128 channels of a row (the last block may be narrower),
 *   s = max(max|y|, 2^-100) / 448,   y8 = e4m3(y / s),   y ~ y8 * s,
 * d_scale fp32 [tokens, blocks] with scale_group = 128, or [tokens] with
 * scale_group = 0; a NaN in a row makes all its y and scales NaN.
 * sum may equal x or resid, and y (of y_type dtype) may equal x or resid,
 * with the same ld; otherwise outputs overlap nothing.  Any alignment and ld;
 * buffers whose rows all start at multiples of 16 bytes (y8: 8) and C a
 * multiple of 8 move in 16-byte pieces.  1 <= C <= 16384 (SD_ERR_UNSUPPORTED
 * past it), eps >= 0.  tokens = 0 does nothing. */
sd_status synerdiff_op_rmsnorm(int32_t dtype, const void* d_x, int64_t x_ld, const void* d_resid, int64_t resid_ld,
                               void* d_sum, int64_t sum_ld, const float* d_gamma, float eps, int64_t tokens,
                               int32_t C, int32_t y_type, void* d_y, int64_t y_ld, float* d_scale,
                               int32_t scale_group, void* hip_stream);

/* synerdiff_op_linear_rows with weights of 4 bits in groups along K:
 *   out[m, n] = act_out(bias[n] + add[m, n] + sum_k act_in(x[m, k]) * w[n, k])
 *   w[n, k] = scale[n, k / group] * (q[n, k] - zero[n, k / group])
 * q: 4-bit codes 0..15, two a byte along K (the even k in the low half), [N,
 * K / 2] bytes, rows at multiples of 4 bytes.  group 32, 64 or 128 (the last
 * group of a row may be narrower); scale [N, ceil(K / group)] in scale_type
 * (SD_F32 or SD_BF16); zero bytes 0..15 of the same shape, or NULL (8).
 * x [M, K] in x_type SD_F32, SD_BF16 or SD_E4M3, row m at m * x_ld
 * (elements); e4m3 rows stand for x8 * x_scale, fp32 [M] with x_group = 0 or
 * [M, ceil(K / 128)] with x_group = 128, as synerdiff_op_rmsnorm writes them
 * (x_scale NULL and x_group 0 for the other types).  act_* = SiLU where
 * silu_* = 1, else the identity (silu_in not with e4m3: SD_ERR_UNSUPPORTED).
 * out [M, N] in out_type SD_F32 or SD_BF16, row m at m * out_ld; bias fp32 [N], add
 * fp32 [M, N], may be NULL; add may equal an fp32 out of out_ld = N; out
 * overlaps nothing else.  Products x * (q - zero) are exact for every x_type
 * (bits of an fp32 x below 2^-133 apart) and summed in fp32; a group's sum may
 * pass fp32's range as long as scale times it does not.  |scale| below 2^116.
 * A row of x with an infinity or NaN gives no finite value.
 * K a multiple of 8; K, N and x_ld <= 2^24, M <= 2^19 (SD_ERR_UNSUPPORTED past
 * them); x and its rows 16-byte aligned (e4m3: 8).  The rows of a result do not
 * depend on M.  M = 0 or N = 0 does nothing. */
sd_status synerdiff_op_linear_rows_w4(int32_t x_type, const void* d_x, int64_t x_ld, const float* d_x_scale,
                                      int32_t x_group, int32_t M, int32_t K, const uint8_t* d_w, int32_t group,
                                      int32_t scale_type, const void* d_scale, const uint8_t* d_zero,
                                      const float* d_bias, const float* d_add, int32_t silu_in, int32_t silu_out,
                                      int32_t out_type, void* d_out, int64_t out_ld, int32_t N, void* hip_stream);

/* Attention of each row's queries over a text of its own length:
 *   o[i, t, h] = sum_j p_j v[j, g] / sum_j p_j,  p_j = exp(scale * q[i, t, h] . k[j, g])
 * over the keys j of row i's context that take part, g = h / (heads /
 * kv_heads).  Row i reads context c = kv_index[i] (NULL: c = i, n_ctx >= n);
 * key j < kv_len[c] (NULL: max_len for all) takes part if its mask byte is not
 * 0 (NULL: all do).  Keys that take no part are not read: they may hold
 * anything.  A row without a key, or whose kv_index lies outside [0, n_ctx),
 * gives zeros.  Keys that score -inf take no weight, and a row whose keys all
 * do gives zeros.  Scores, sums and results are fp32 until the result is
 * rounded to dtype.  bf16 probabilities are rounded to bf16 (by up to 2^-8 of
 * each) where a K/V head has more than 128 rows, heads / kv_heads * n_q; up to
 * 128 keep 2^-17.
 * Layouts: element (i, t, h, e) of q is at q + i * q_img + t * q_ld + h *
 * q_head + e, o likewise.  Contexts one after another (d_kv_start not NULL):
 * key j of context c is row kv_start[c] + j of k: k + row * k_ld + g *
 * k_head + e, and mask byte `row` of [kv_tokens]; a context that starts
 * outside [0, kv_tokens) is empty, one that ends past it is cut there.  Padded
 * contexts (d_kv_start NULL): k + c * k_ctx + j * k_ld + g * k_head + e, and
 * mask byte c * max_len + j.  v likewise.  A
 * kv_len past max_len counts as max_len, a negative one as 0.  Strides in
 * elements, not negative (0 for a shared head; that of an axis of one element
 * is not looked at).
 * Constraints: d a multiple of 8, <= 256; heads a multiple of kv_heads, <=
 * 2^16; max_len <= 2^30; q_ld, k_ld, v_ld, o_ld <= 2^23; a grid of less than
 * 2^32 threads (a block of 512 per 32 rows of a K/V head and split); q, k, v, o
 * and all their strides at multiples of 16 bytes.  o overlaps nothing.  Few
 * queries over long texts are split along the keys: d_scratch (fp32, 16-byte
 * aligned) has to hold synerdiff_op_cross_attention_scratch_floats(...) floats
 * then (0: none needed, -1: the grid is too large; SD_ERR_WORKSPACE if smaller),
 * and belongs to this call until it has run.  The bits of a row depend on its own inputs, n_q, heads,
 * kv_heads and d, not on the other rows or max_len.  n = 0 or n_q = 0 does nothing. */
int64_t synerdiff_op_cross_attention_scratch_floats(int32_t dtype, int32_t n, int32_t heads, int32_t kv_heads,
                                                    int32_t d, int32_t n_q, int32_t max_len);
sd_status synerdiff_op_cross_attention(int32_t dtype, const void* d_q, int64_t q_ld, int64_t q_head, int64_t q_img,
                                       const void* d_k, int64_t k_ld, int64_t k_head, int64_t k_ctx, const void* d_v,
                                       int64_t v_ld, int64_t v_head, int64_t v_ctx, int64_t kv_tokens, int32_t n_ctx,
                                       int32_t max_len, const int32_t* d_kv_start, const int32_t* d_kv_len,
                                       const int32_t* d_kv_index, const uint8_t* d_mask, void* d_o, int64_t o_ld,
                                       int64_t o_head, int64_t o_img, int32_t n, int32_t heads, int32_t kv_heads,
                                       int32_t d, int32_t n_q, float scale, float* d_scratch, int64_t scratch_floats,
                                       void* hip_stream);

/* Attention inside texts of their own lengths (a text encoder's layers):
 *   o[i, h] = sum_j p_j v[j, g] / sum_j p_j,   g = h / (heads / kv_heads)
 *   p_j = exp(f(scale * q[i, h] . k[j, g]) + bias[h, clip(j - i, -reach, reach) + reach] - slope[h] |j - i|)
 * i and j count from the text's first token; f(s) = cap * tanh(s / cap), or s
 * with cap = 0; bias fp32 [heads, 2 reach + 1] and slope fp32 [heads] may be
 * NULL (bias NULL: reach 0).  Key j takes part if it lies in the query's own
 * text, its mask byte is not 0 (mask NULL: all) and, with causal = 1, j <= i or
 * j < prefix[c] (int32 [n], NULL: 0; counts past the text's end end there,
 * negative ones are 0).  Queries of masked tokens are computed like others.
 * Keys that take no part for any query of their text are not read, and what k
 * and v hold behind a query's causal border does not reach it, infinities and
 * NaN included; nor does what bias holds at the distance of a key that takes no part.
 * Keys that score -inf (a bias of -inf, say) take no weight, as long as their v is
 * finite; a query without a key of any weight gives zeros.  (An infinite v under a
 * weight that fp32 does not hold may give NaN.  A scale of 0 is one for finite q and k.)
 * A finite bias, lowest value of fp32 included, stays finite: a query whose keys all
 * have it weighs them alike.  Scores, sums and results are fp32 until the result is
 * rounded to dtype; sums over keys, of weights up to 2^8, come before the division, so
 * values of v up to 2^90 are safe.  bf16 probabilities are rounded to bf16 (by up to 2^-8
 * of each) and summed as rounded, and capped bf16 scores are right to 2^-21 of the cap.
 * Layouts (strides in elements, 0 or more; that of an axis of one element is
 * not looked at).  Packed texts (d_start not NULL, int32 [n + 1], not
 * decreasing): text c is rows start[c] .. start[c + 1] - 1 of [tokens], cut at
 * both ends of it; element (row, h, e) of q at q + row * q_ld + h * q_head +
 * e, k, v, o likewise, mask [tokens].  Padded texts (d_start NULL): text c is the first
 * length[c] (int32 [n], NULL: max_len) of max_len rows at c * q_text and so on,
 * mask [n, max_len]; tokens is not looked at.  No text is longer than max_len (what lies past
 * it is left out).  Rows of o in no text keep what they hold; with zero_rest =
 * 1 they become 0 (padded: all rows past the lengths; packed: those before
 * start[0], from start[n] on, and past a text's first max_len).
 * Constraints: d a multiple of 8, <= 256; heads a multiple of kv_heads, <=
 * 2^16; n kv_heads <= 2^19 - 8; max_len <= 2^30; q_ld, k_ld, v_ld, o_ld <= 2^23;
 * scale 0 or 2^-60 to 2^60 in size, cap 0 or 2^-20 to 2^12; reach <= 2^24; a grid
 * of less than 2^32 threads (256 per 128 queries of a head, in chunks of 8); q,
 * k, v, o and their strides at multiples of 16 bytes.  o overlaps nothing.  No
 * workspace.  n = 0 does nothing.  The bits of a query depend on its own text alone. */
sd_status synerdiff_op_text_attention(int32_t dtype, const void* d_q, int64_t q_ld, int64_t q_head, int64_t q_text,
                                      const void* d_k, int64_t k_ld, int64_t k_head, int64_t k_text, const void* d_v,
                                      int64_t v_ld, int64_t v_head, int64_t v_text, void* d_o, int64_t o_ld,
                                      int64_t o_head, int64_t o_text, int64_t tokens, int32_t n, int32_t max_len,
                                      const int32_t* d_start, const int32_t* d_length, const uint8_t* d_mask,
                                      int32_t causal, const int32_t* d_prefix, float cap, const float* d_bias,
                                      int32_t reach, const float* d_slope, int32_t heads, int32_t kv_heads, int32_t d,
                                      float scale, int32_t zero_rest, void* hip_stream);

/* Linear layer that all rows share, plus a low-rank adapter for each (requests
 * of one batch with styles of their own):
 *   out[m, n] = bias[n] + sum_k x[m, k] w[n, k] + scale[c] sum_r v[m, r] up[c, n, r]
 *   v[m, r] = sum_k x[m, k] down[c, r, k],   c = index[m / group]
 * x [M, K], w [N, K], down [count, rank, K], up [count, N, rank] and out (row m
 * at m * out_ld) in dtype; scale fp32 [count] (NULL: 1) and bias fp32 [N] (NULL:
 * 0); index int32 [M / group rounded up].  A row whose index lies outside [0,
 * count) has no adapter (count may be 0, down and up NULL then).  A row depends
 * on no other row and on no other adapter than its own, whatever they hold.
 * Narrower adapters are padded with zeros.  Sums are fp32; v is fp32 for fp32
 * and for up to 32 rows (64 up to K = 2048), else held to 2^-17 of it (two bf16
 * parts; below 2^-110 less).  Infinities give what the formula gives.  Any order of indices is right; runs of 32 rows or
 * more of one adapter are fast.
 * Constraints: K, N, rank multiples of 8; K, N <= 2^20, rank <= 1024; w, up[c] and
 * down[c] below 2^31 bytes; M <= 2^26, M N < 2^35, M rank < 2^33; all
 * buffers and rows of out at multiples of 16 bytes (scale, index: 4).  out
 * overlaps nothing.  d_scratch (fp32, 16-byte aligned) holds
 * synerdiff_op_linear_adapters_scratch_floats(...) floats (0: none needed;
 * SD_ERR_WORKSPACE if fewer), and belongs to this call until it has run.  M = 0 or N = 0 does nothing. */
int64_t synerdiff_op_linear_adapters_scratch_floats(int32_t dtype, int32_t M, int32_t rank);
sd_status synerdiff_op_linear_adapters(int32_t dtype, const void* d_x, int32_t M, int32_t K, const void* d_w, int32_t N,
                                       const void* d_down, const void* d_up, int32_t rank, int32_t count,
                                       const float* d_scale, const int32_t* d_index, int32_t group,
                                       const float* d_bias, void* d_out, int64_t out_ld, float* d_scratch,
                                       int64_t scratch_floats, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SYNERDIFF_OPS_H */
