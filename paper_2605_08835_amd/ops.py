"""Python wrappers of the kernel-level entry points (include/synerdiff_ops.h).
Tensors are torch device tensors; activations channels-last."""
import torch

from .binding import SD_BF16, SD_E4M3, SD_F32, _check, _ptr, lib


def _dt(t):
    if t.dtype == torch.bfloat16:
        return SD_BF16
    if t.dtype == torch.float32:
        return SD_F32
    raise TypeError(t.dtype)


def _s():
    return torch.cuda.current_stream().cuda_stream


def conv(x0, w_packed, cout, ks=3, stride=1, up=0, x1=None, scale=None, shift=None, silu=0, bias=None,
         resid=None, out=None, out_f32=False, split=True):
    n, H, W, c0 = x0.shape
    c1 = 0 if x1 is None else x1.shape[3]
    Ho, Wo = (2 * H, 2 * W) if up else (H // stride, W // stride)
    if out is None:
        out = torch.empty(n, Ho, Wo, cout, device=x0.device, dtype=torch.float32 if out_f32 else x0.dtype)
    nsc = lib().synerdiff_op_conv_scratch_floats(_dt(x0), c0, c1, n, H, W, ks, stride, up, cout) if split else 0
    scratch = torch.empty(nsc, device=x0.device) if nsc > 0 else None
    _check(lib().synerdiff_op_conv(_dt(x0), _ptr(x0), c0, _ptr(x1), c1, n, H, W, ks, stride, up, _ptr(scale),
                                   _ptr(shift), silu, _ptr(w_packed), cout, _ptr(bias), _ptr(resid), _ptr(out),
                                   int(out_f32), _ptr(scratch), nsc, _s()))
    return out


def attention(q, k, v, o, n, heads, d, n_q, n_k, q_ld, q_img, k_ld, k_img, v_ld, v_img, o_ld, o_img, scale,
              kv_index=None, v_transposed=False, q_log2=False):
    _check(lib().synerdiff_op_attention(_dt(q), _ptr(q), q_ld, q_img, _ptr(k), k_ld, k_img, _ptr(v), v_ld, v_img,
                                        int(v_transposed), _ptr(kv_index), _ptr(o), o_ld, o_img, n, heads, d, n_q,
                                        n_k, float(scale), int(q_log2), _s()))
    return o


def groupnorm_stats(x0, groups, eps, gamma, beta, x1=None):
    n, H, W, c0 = x0.shape
    c1 = 0 if x1 is None else x1.shape[3]
    cin = c0 + c1
    part = torch.empty(lib().synerdiff_op_groupnorm_scratch_floats(n, H * W, cin), device=x0.device)
    scale = torch.empty(n, cin, device=x0.device)
    shift = torch.empty(n, cin, device=x0.device)
    _check(lib().synerdiff_op_groupnorm_stats(_dt(x0), _ptr(x0), c0, _ptr(x1), c1, n, H * W, groups, float(eps),
                                              _ptr(gamma), _ptr(beta), _ptr(part), _ptr(scale), _ptr(shift), _s()))
    return scale, shift


def layernorm(x, gamma, beta, eps=1e-5):
    y = torch.empty_like(x)
    C = x.shape[-1]
    _check(lib().synerdiff_op_layernorm(_dt(x), _ptr(x), _ptr(y), x.numel() // C, C, _ptr(gamma), _ptr(beta),
                                        float(eps), _s()))
    return y


def layernorm_rstd(x, eps=1e-5):
    """fp32 [tokens] = 1 / sqrt(var + eps) of each row of x [tokens, C]."""
    C = x.shape[-1]
    rstd = torch.empty(x.numel() // C, device=x.device)
    _check(lib().synerdiff_op_layernorm_rstd(_dt(x), _ptr(x), _ptr(rstd), x.numel() // C, C, float(eps), _s()))
    return rstd


def upconv(x, w_phases, cout, bias=None):
    """Nearest-2x upsample + 3x3 conv of bf16 x [n, H, W, cin] as four phase
    convolutions; w_phases bf16 [4, cout, 4 * cin]."""
    n, H, W, cin = x.shape
    out = torch.empty(n, 2 * H, 2 * W, cout, device=x.device, dtype=x.dtype)
    _check(lib().synerdiff_op_upconv(_dt(x), _ptr(x), n, H, W, cin, _ptr(w_phases), cout, _ptr(bias), _ptr(out),
                                     _s()))
    return out


def linear_rows(x, w, bias=None, add=None, silu_in=0, silu_out=0):
    """x fp32 [M, K], w [N, K] (fp32 or bf16) -> fp32 [M, N]."""
    M, K = x.shape
    N = w.shape[0]
    y = torch.empty(M, N, device=x.device, dtype=torch.float32)
    _check(lib().synerdiff_op_linear_rows(_dt(w), _ptr(x), M, K, _ptr(w), _ptr(bias), _ptr(add), _ptr(y), N,
                                          int(silu_in), int(silu_out), _s()))
    return y


def geglu(x):
    half = x.shape[-1] // 2
    y = torch.empty(x.shape[:-1] + (half,), device=x.device, dtype=x.dtype)
    _check(lib().synerdiff_op_geglu(_dt(x), _ptr(x), _ptr(y), x.numel() // x.shape[-1], half, _s()))
    return y


def conv_out_cfg_ddim(x, w_packed, bias, req_row_u, req_coef, lat_in, lat_out=None, eps_out=None):
    """Output conv (3x3, C -> 4) + CFG combine + DDIM; x [rows, H, W, C] bf16,
    req_row_u int32 [n_req] and req_coef fp32 [n_req, 3] on the device."""
    n, H, W, C = x.shape
    n_req = int(req_row_u.shape[0])
    if lat_out is None:
        lat_out = torch.empty_like(lat_in)
    _check(lib().synerdiff_op_conv_out_cfg_ddim(_dt(x), _ptr(x), H, W, C, _ptr(w_packed), _ptr(bias), n_req,
                                                _ptr(req_row_u), _ptr(req_coef), _ptr(lat_in), _ptr(lat_out),
                                                _ptr(eps_out), _s()))
    return lat_out


def groupnorm_fused(x0, groups, eps, gamma, beta, x1=None, silu=True):
    """GroupNorm (+ SiLU) of [x0 | x1] in one kernel (bf16, small images)."""
    n, H, W, c0 = x0.shape
    c1 = 0 if x1 is None else x1.shape[3]
    out = torch.empty(n, H, W, c0 + c1, device=x0.device, dtype=x0.dtype)
    _check(lib().synerdiff_op_groupnorm_fused(_dt(x0), _ptr(x0), c0, _ptr(x1), c1, n, H * W, groups, float(eps),
                                              _ptr(gamma), _ptr(beta), int(silu), _ptr(out), _s()))
    return out


def groupnorm_stats_noalloc(x0, groups, eps, gamma, beta, x1=None, scale=None, shift=None):
    """GroupNorm statistics through the entry point that allocates nothing
    (the partial sums live in the library's own device array)."""
    n, H, W, c0 = x0.shape
    c1 = 0 if x1 is None else x1.shape[3]
    cin = c0 + c1
    scale = torch.empty(n, cin, device=x0.device) if scale is None else scale
    shift = torch.empty(n, cin, device=x0.device) if shift is None else shift
    _check(lib().synerdiff_op_groupnorm_stats_noalloc(_dt(x0), _ptr(x0), c0, _ptr(x1), c1, n, H * W, groups,
                                                      float(eps), _ptr(gamma), _ptr(beta), _ptr(scale),
                                                      _ptr(shift), _s()))
    return scale, shift


# Operators on texts of their own lengths and on few-bit weights.  Their
# tensors may live on any one device: the call runs there, on that device's
# current stream.
_TYPE = {torch.float32: SD_F32, torch.bfloat16: SD_BF16, torch.float8_e4m3fn: SD_E4M3}


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _enqueue(fn, like, args, others):
    """fn(*args, stream) on the device of `like`, which the tensors `others` (or
    None) share.  (The raw-stream and device queries cost 0.2 us together, the
    public ones 3, of a call of about 8.)"""
    dev = like.get_device()
    for t in others:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"tensors on {like.device} and {t.device}")
    if dev < 0:
        raise ValueError(f"tensors on {like.device}: the kernels run on the GPU")
    stream = torch._C._cuda_getCurrentRawStream(dev)
    if dev == torch._C._cuda_getDevice():
        _check(fn(*args, stream))
    else:
        with torch.cuda.device(dev):
            _check(fn(*args, stream))


def _row_stride(t, what):
    """Distance between the rows (last axis) of t, whose rows lie evenly."""
    if t.dim() == 2:
        rows, c = t.shape
        s0, s1 = t.stride()
        _need(s1 == 1 or c == 1, f"{what}: the last axis must be contiguous")
        return s0 if rows > 1 else c
    _need(t.dim() >= 1 and t.is_contiguous(), f"{what}: more than two axes must be contiguous")
    return t.shape[-1]


def rmsnorm(x, gamma=None, eps=1e-6, resid=None, sum_out=None, out=None, fp8=False, scale_group=0):
    """Root-mean-square norm of the rows of x + resid (fp32 or bf16 [..., C]):
    y = h / sqrt(mean(h^2) + eps) * gamma, gamma fp32 [C] or None.
    Returns y, or (y, h) with a residual (h rounded to x's type, into sum_out
    when given).  fp8: y is float8_e4m3fn and fp32 scales [..., C / 128 rounded
    up] (scale_group = 128) or [..., 1] (scale_group = 0) follow it, y ~ y8 *
    scale.  sum_out may be x or resid, out (not fp8) likewise, but not both the same."""
    if x.dtype is not torch.bfloat16 and x.dtype is not torch.float32:
        raise TypeError(x.dtype)
    C = x.shape[-1]
    rows = x.numel() // C if C else 0
    x_ld = _row_stride(x, "x")
    y_type = torch.float8_e4m3fn if fp8 else x.dtype
    if resid is not None:
        _need(resid.shape == x.shape and resid.dtype is x.dtype, "resid has another shape or type than x")
        if sum_out is None:
            sum_out = torch.empty_like(x)
        else:
            _need(sum_out.shape == x.shape and sum_out.dtype is x.dtype, "sum_out has another shape or type than x")
    else:
        _need(sum_out is None, "sum_out without resid")
    if gamma is not None:
        _need(gamma.dtype is torch.float32 and gamma.shape == (C,) and gamma.is_contiguous(), "gamma must be fp32 [C]")
    _need(scale_group in (0, 128) and (fp8 or not scale_group), "scale_group is 0 or 128, and 128 only with fp8")
    if out is None:
        out = torch.empty_like(x, dtype=y_type) if fp8 else torch.empty_like(x)
    else:
        _need(out.shape == x.shape and out.dtype is y_type, "out has another shape or type than the result")
    scale = None
    if fp8:
        blocks = -(-C // 128) if scale_group else 1
        scale = x.new_empty(x.shape[:-1] + (blocks,), dtype=torch.float32)
    _enqueue(lib().synerdiff_op_rmsnorm, x,
             (_TYPE[x.dtype], x.data_ptr(), x_ld, _ptr(resid), 0 if resid is None else _row_stride(resid, "resid"),
              _ptr(sum_out), 0 if sum_out is None else _row_stride(sum_out, "sum_out"), _ptr(gamma), float(eps), rows, C,
              _TYPE[y_type], out.data_ptr(), _row_stride(out, "out"), _ptr(scale), scale_group),
             (resid, sum_out, gamma, out))
    got = (out, scale) if fp8 else (out,)
    if resid is not None:
        got += (sum_out,)
    return got if len(got) > 1 else out


def linear_rows_w4(x, w, scale, group, zero=None, x_scale=None, bias=None, add=None, silu_in=0, silu_out=0,
                   out_dtype=torch.float32, out=None):
    """x [M, K] (fp32, bf16, or float8_e4m3fn with x_scale fp32 [M, 1] or [M,
    K / 128 rounded up]) times 4-bit weights: w uint8 [N, K / 2], two codes a
    byte (the even k in the low half), scale fp32 or bf16 [N, K / group rounded
    up], zero uint8 of that shape or None (8), weight = scale * (code - zero).
    bias fp32 [N] and add fp32 [M, N] are added, silu_in / silu_out as in
    linear_rows; returns [M, N] in out_dtype (fp32 or bf16)."""
    t = _TYPE.get(x.dtype)
    if t is None:
        raise TypeError(x.dtype)
    if scale.dtype is not torch.float32 and scale.dtype is not torch.bfloat16:
        raise TypeError(scale.dtype)
    if out_dtype is not torch.float32 and out_dtype is not torch.bfloat16:
        raise TypeError(out_dtype)
    _need(x.dim() == 2 and w.dim() == 2 and w.dtype is torch.uint8, "x must be [M, K], w uint8 [N, K / 2]")
    M, K = x.shape
    N = w.shape[0]
    _need(group in (32, 64, 128), "group must be 32, 64 or 128")
    _need(K > 0 and K % 8 == 0 and w.shape[1] * 2 == K and w.is_contiguous(), "w must be [N, K / 2], contiguous, K a multiple of 8")
    shape = (N, -(-K // group))
    _need(scale.shape == shape and scale.is_contiguous(), "scale must be [N, K / group rounded up], contiguous")
    if zero is not None:
        _need(zero.dtype is torch.uint8 and zero.shape == shape and zero.is_contiguous(), "zero must be uint8 of scale's shape")
    x_group = 0
    if t == SD_E4M3:
        _need(x_scale is not None and x_scale.dtype is torch.float32 and x_scale.is_contiguous() and x_scale.dim() == 2 and
              x_scale.shape[0] == M and x_scale.shape[1] in (1, -(-K // 128)),
              "e4m3 rows need x_scale fp32 [M, 1] or [M, K / 128 rounded up]")
        x_group = 128 if x_scale.shape[1] > 1 else 0
    else:
        _need(x_scale is None, "x_scale belongs to e4m3 rows")
    if bias is not None:
        _need(bias.dtype is torch.float32 and bias.shape == (N,) and bias.is_contiguous(), "bias must be fp32 [N]")
    if add is not None:
        _need(add.dtype is torch.float32 and add.shape == (M, N) and add.is_contiguous(), "add must be fp32 [M, N]")
    if out is None:
        out = x.new_empty((M, N), dtype=out_dtype)
    else:
        _need(out.shape == (M, N) and out.dtype is out_dtype, "out has another shape or type than the result")
    _enqueue(lib().synerdiff_op_linear_rows_w4, x,
             (t, x.data_ptr(), _row_stride(x, "x"), _ptr(x_scale), x_group, M, K, w.data_ptr(), group,
              _TYPE[scale.dtype], scale.data_ptr(), _ptr(zero), _ptr(bias), _ptr(add), 1 if silu_in else 0,
              1 if silu_out else 0, _TYPE[out_dtype], out.data_ptr(), _row_stride(out, "out"), N),
             (w, scale, zero, x_scale, bias, add, out))
    return out


def cross_attention(q, k, v, max_len, kv_start=None, kv_len=None, kv_index=None, mask=None, scale=None, out=None):
    """Attention of q [n, n_q, heads, d] over a text of its own length for
    every row.  Packed texts: k, v [tokens, kv_heads, d], text c at rows
    kv_start[c] .. + kv_len[c] (int32 [n_ctx]), mask (bool or uint8) [tokens].
    Padded texts (kv_start None): k, v [n_ctx, max_len, kv_heads, d], kv_len
    int32 [n_ctx] or None (all max_len), mask [n_ctx, max_len].  kv_index int32
    [n]: the text of each row (None: row i reads text i).  No text is longer
    than max_len.  heads may be a multiple of kv_heads (shared in order); q, k,
    v and out may be strided as long as d is contiguous.  scale defaults to
    1 / sqrt(d).  A row without keys gives zeros.  Returns [n, n_q, heads, d]
    in q's type."""
    if q.dtype is not torch.bfloat16 and q.dtype is not torch.float32:
        raise TypeError(q.dtype)
    _need(q.dim() == 4 and k.dim() == (4 if kv_start is None else 3), "q [n, n_q, heads, d]; k, v [tokens, kv_heads, d] "
          "with kv_start, [n_ctx, max_len, kv_heads, d] without")
    n, n_q, heads, d = q.shape
    _need(k.dtype is q.dtype and v.dtype is q.dtype and k.shape == v.shape and k.shape[-1] == d,
          "k and v must have q's type and width, and one shape")
    kv_heads = k.shape[-2]
    qs, ks, vs = q.stride(), k.stride(), v.stride()
    _need(d == 1 or qs[3] == ks[-1] == vs[-1] == 1, "d must be contiguous")
    if kv_start is None:
        n_ctx, tokens = k.shape[0], 0
        _need(k.shape[1] == max_len, "padded k, v must be [n_ctx, max_len, kv_heads, d]")
        k_ctx, v_ctx = ks[0], vs[0]
    else:
        n_ctx, tokens, k_ctx, v_ctx = kv_start.shape[0], k.shape[0], 0, 0
        _need(kv_len is not None, "packed texts need kv_len")
    for a, length, name in ((kv_start, n_ctx, "kv_start"), (kv_len, n_ctx, "kv_len"), (kv_index, n, "kv_index")):
        if a is not None:
            _need(a.dtype is torch.int32 and a.shape == (length,) and a.is_contiguous(), f"{name} must be int32 [{length}]")
    if mask is not None:
        _need(mask.dtype in (torch.bool, torch.uint8) and mask.shape == k.shape[:-2] and mask.is_contiguous(),
              "mask must be bool or uint8, one value per token")
    if out is None:
        out = q.new_empty((n, n_q, heads, d))
        os = (n_q * heads * d, heads * d, d)
    else:
        _need(out.shape == q.shape and out.dtype is q.dtype and out.stride(3) == 1, "out must have q's shape and type, d contiguous")
        os = out.stride()
    L, t = lib(), _TYPE[q.dtype]
    floats = L.synerdiff_op_cross_attention_scratch_floats(t, n, heads, kv_heads, d, n_q, max_len)
    scratch = q.new_empty(floats, dtype=torch.float32) if floats > 0 else None
    _enqueue(L.synerdiff_op_cross_attention, q,
             (t, q.data_ptr(), qs[1], qs[2], qs[0], k.data_ptr(), ks[-3], ks[-2], k_ctx, v.data_ptr(), vs[-3], vs[-2],
              v_ctx, tokens, n_ctx, max_len, _ptr(kv_start), _ptr(kv_len), _ptr(kv_index), _ptr(mask), out.data_ptr(),
              os[1], os[2], os[0], n, heads, kv_heads, d, n_q, d ** -0.5 if scale is None else float(scale),
              _ptr(scratch), floats),
             (k, v, kv_start, kv_len, kv_index, mask, out))
    return out
