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
# current stream.  (A call takes about 8 us on the host, 4 of them the launch;
# the checks are written for that: no message is built unless it is raised.)
# Forward only: nothing here records a gradient.
_TYPE = {torch.float32: SD_F32, torch.bfloat16: SD_BF16, torch.float8_e4m3fn: SD_E4M3}


def _at(t):
    return None if t is None else t.data_ptr()


def _bad(what):
    raise ValueError(what)


def _int32(largest):
    if largest >= 1 << 31:  # (ctypes would pass the low 32 bits)
        _bad("a size of 2^31 or more")


def _enqueue(fn, like, others, args):
    """fn(*args, stream) on the device of `like`, which the tensors `others` (or
    None) share.  (The raw-stream and device queries cost 0.2 us together, the
    public ones 3.)"""
    dev = like.get_device()
    for t in others:
        if t is not None and t.get_device() != dev:
            _bad(f"tensors on {like.device} and {t.device}")
    if dev < 0:
        _bad(f"tensors on {like.device}: the kernels run on the GPU")
    stream = torch._C._cuda_getCurrentRawStream(dev)
    if dev == torch._C._cuda_getDevice():
        status = fn(*args, stream)
    else:
        with torch.cuda.device(dev):
            status = fn(*args, stream)
    if status:
        _check(status)


def _row_stride(t, what):
    """Distance between the rows (last axis) of t, whose rows lie evenly."""
    if t.is_contiguous():
        return t.shape[-1]
    if t.dim() != 2 or (t.stride(1) != 1 and t.shape[1] != 1):
        _bad(f"{what}: the last axis must be contiguous, and more than two axes all of them")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def rmsnorm(x, gamma=None, eps=1e-6, resid=None, sum_out=None, out=None, fp8=False, scale_group=0):
    """Root-mean-square norm of the rows of x + resid (fp32 or bf16 [..., C]):
    y = h / sqrt(mean(h^2) + eps) * gamma, gamma fp32 [C] or None.
    Returns y, or (y, h) with a residual (h rounded to x's type, into sum_out
    when given).  fp8: y is float8_e4m3fn and fp32 scales [..., C / 128 rounded
    up] (scale_group = 128) or [..., 1] (scale_group = 0) follow it, y ~ y8 *
    scale.  sum_out may be x or resid, and so may out (not with fp8), but not
    both the same one."""
    dt = x.dtype
    if dt is not torch.bfloat16 and dt is not torch.float32:
        raise TypeError(dt)
    shape = x.shape
    C = shape[-1] if shape else _bad("x must have rows")
    _int32(C)
    x_ld = _row_stride(x, "x")
    r_ld = s_ld = 0
    if resid is not None:
        if resid.shape != shape or resid.dtype is not dt:
            _bad("resid has another shape or type than x")
        r_ld = _row_stride(resid, "resid")
        if sum_out is None:
            sum_out = torch.empty_like(x)
        elif sum_out.shape != shape or sum_out.dtype is not dt:
            _bad("sum_out has another shape or type than x")
        s_ld = _row_stride(sum_out, "sum_out")
    elif sum_out is not None:
        _bad("sum_out without resid")
    if gamma is not None and (gamma.dtype is not torch.float32 or gamma.shape != (C,) or not gamma.is_contiguous()):
        _bad("gamma must be fp32 [C]")
    if scale_group and (scale_group != 128 or not fp8):
        _bad("scale_group is 0 or 128, and 128 only with fp8")
    y_type = torch.float8_e4m3fn if fp8 else dt
    if out is None:
        out = torch.empty_like(x, dtype=y_type) if fp8 else torch.empty_like(x)
    elif out.shape != shape or out.dtype is not y_type:
        _bad("out has another shape or type than the result")
    scale = None
    if fp8:
        scale = x.new_empty(shape[:-1] + ((C + 127) // 128 if scale_group else 1,), dtype=torch.float32)
    _enqueue(lib().synerdiff_op_rmsnorm, x, (resid, sum_out, gamma, out),
             (_TYPE[dt], x.data_ptr(), x_ld, _at(resid), r_ld, _at(sum_out), s_ld, _at(gamma), eps,
              x.numel() // C if C else 0, C, _TYPE[y_type], out.data_ptr(), _row_stride(out, "out"), _at(scale), scale_group))
    if resid is None:
        return (out, scale) if fp8 else out
    return (out, scale, sum_out) if fp8 else (out, sum_out)


def linear_rows_w4(x, w, scale, group, zero=None, x_scale=None, bias=None, add=None, silu_in=0, silu_out=0,
                   out_dtype=torch.float32, out=None):
    """x [M, K] (fp32, bf16, or float8_e4m3fn with x_scale fp32 [M, 1] or [M,
    K / 128 rounded up]) times 4-bit weights: w uint8 [N, K / 2], two codes a
    byte (the even k in the low half), scale fp32 or bf16 [N, K / group rounded
    up], zero uint8 of that shape or None (8), weight = scale * (code - zero).
    bias fp32 [N] and add fp32 [M, N] are added, silu_in / silu_out as in
    linear_rows; returns [M, N] in out_dtype (fp32 or bf16)."""
    t, st, ot = _TYPE.get(x.dtype), _TYPE.get(scale.dtype), _TYPE.get(out_dtype)
    if t is None or st not in (SD_F32, SD_BF16) or ot not in (SD_F32, SD_BF16):
        raise TypeError((x.dtype, scale.dtype, out_dtype))
    if x.dim() != 2 or w.dim() != 2 or w.dtype is not torch.uint8:
        _bad("x must be [M, K], w uint8 [N, K / 2]")
    M, K = x.shape
    N, half = w.shape
    _int32(max(M, K, N))
    if group != 128 and group != 64 and group != 32:
        _bad("group must be 32, 64 or 128")
    if K == 0 or K % 8 or half * 2 != K or not w.is_contiguous():
        _bad("w must be [N, K / 2], contiguous, K a multiple of 8")
    shape = (N, (K + group - 1) // group)
    if scale.shape != shape or not scale.is_contiguous():
        _bad("scale must be [N, K / group rounded up], contiguous")
    if zero is not None and (zero.dtype is not torch.uint8 or zero.shape != shape or not zero.is_contiguous()):
        _bad("zero must be uint8 of scale's shape")
    x_group = 0
    if t == SD_E4M3:
        blocks = (K + 127) // 128
        if x_scale is None or x_scale.dtype is not torch.float32 or not x_scale.is_contiguous() or (
                x_scale.shape != (M, 1) and x_scale.shape != (M, blocks)):
            _bad("e4m3 rows need x_scale fp32 [M, 1] or [M, K / 128 rounded up]")
        x_group = 128 if x_scale.shape[1] > 1 else 0
    elif x_scale is not None:
        _bad("x_scale belongs to e4m3 rows")
    if bias is not None and (bias.dtype is not torch.float32 or bias.shape != (N,) or not bias.is_contiguous()):
        _bad("bias must be fp32 [N]")
    if add is not None and (add.dtype is not torch.float32 or add.shape != (M, N) or not add.is_contiguous()):
        _bad("add must be fp32 [M, N]")
    if out is None:
        out, out_ld = x.new_empty((M, N), dtype=out_dtype), N
    else:
        if out.shape != (M, N) or out.dtype is not out_dtype:
            _bad("out has another shape or type than the result")
        out_ld = _row_stride(out, "out")
    _enqueue(lib().synerdiff_op_linear_rows_w4, x, (w, scale, zero, x_scale, bias, add, out),
             (t, x.data_ptr(), _row_stride(x, "x"), _at(x_scale), x_group, M, K, w.data_ptr(), group, st, scale.data_ptr(),
              _at(zero), _at(bias), _at(add), 1 if silu_in else 0, 1 if silu_out else 0, ot, out.data_ptr(), out_ld, N))
    return out


def _index(a, length, name):
    if a.dtype is not torch.int32 or a.shape != (length,) or not a.is_contiguous():
        _bad(f"{name} must be int32 [{length}]")
    return a.data_ptr()


def cross_attention(q, k, v, max_len, kv_start=None, kv_len=None, kv_index=None, mask=None, scale=None, out=None):
    """Attention of q [n, n_q, heads, d] over a text of its own length for
    every row.  Packed texts: k, v [tokens, kv_heads, d], text c at rows
    kv_start[c] .. + kv_len[c] (int32 [n_ctx]), mask (bool or uint8) [tokens].
    Padded texts (kv_start None): k, v [n_ctx, max_len, kv_heads, d], kv_len
    int32 [n_ctx] or None (all max_len), mask [n_ctx, max_len].  kv_index int32
    [n]: the text of each row (None: row i reads text i).  No text is longer
    than max_len.  heads may be a multiple of kv_heads (shared in order); q, k,
    v and out may be strided as long as d is contiguous.  scale defaults to
    1 / sqrt(d).  Keys that score -inf take no weight; a row without keys of
    any weight gives zeros.  Returns [n, n_q, heads, d] in q's type."""
    dt = q.dtype
    if dt is not torch.bfloat16 and dt is not torch.float32:
        raise TypeError(dt)
    packed = kv_start is not None
    ks = k.stride()
    if q.dim() != 4 or len(ks) != (3 if packed else 4):
        _bad("q [n, n_q, heads, d]; k, v [tokens, kv_heads, d] with kv_start, [n_ctx, max_len, kv_heads, d] without")
    n, n_q, heads, d = q.shape
    kshape = k.shape
    if k.dtype is not dt or v.dtype is not dt or kshape != v.shape or kshape[-1] != d:
        _bad("k and v must have q's type and width, and one shape")
    kv_heads = kshape[-2]
    qs, vs = q.stride(), v.stride()
    if d > 1 and (qs[3] != 1 or ks[-1] != 1 or vs[-1] != 1):
        _bad("d must be contiguous")
    if packed:
        n_ctx, tokens, k_ctx, v_ctx = kv_start.shape[0], kshape[0], 0, 0
        if kv_len is None:
            _bad("packed texts need kv_len")
    else:
        n_ctx, tokens, k_ctx, v_ctx = kshape[0], 0, ks[0], vs[0]
        if kshape[1] != max_len:
            _bad("padded k, v must be [n_ctx, max_len, kv_heads, d]")
    _int32(max(n, n_q, heads, kv_heads, d, n_ctx, abs(max_len)))
    start_p = _index(kv_start, n_ctx, "kv_start") if packed else None
    len_p = _index(kv_len, n_ctx, "kv_len") if kv_len is not None else None
    index_p = _index(kv_index, n, "kv_index") if kv_index is not None else None
    if mask is not None and ((mask.dtype is not torch.bool and mask.dtype is not torch.uint8) or mask.shape != kshape[:-2]
                             or not mask.is_contiguous()):
        _bad("mask must be bool or uint8, one value per token")
    if out is None:
        out, os = q.new_empty((n, n_q, heads, d)), (n_q * heads * d, heads * d, d)
    else:
        os = out.stride()
        if out.shape != q.shape or out.dtype is not dt or (d > 1 and os[3] != 1):
            _bad("out must have q's shape and type, d contiguous")
    L, t = lib(), _TYPE[dt]
    floats, scratch = 0, None
    if max_len > 512:  # (no shorter text is split)
        floats = L.synerdiff_op_cross_attention_scratch_floats(t, n, heads, kv_heads, d, n_q, max_len)
        if floats > 0:
            scratch = q.new_empty(floats, dtype=torch.float32)
    _enqueue(L.synerdiff_op_cross_attention, q, (k, v, kv_start, kv_len, kv_index, mask, out),
             (t, q.data_ptr(), qs[1], qs[2], qs[0], k.data_ptr(), ks[-3], ks[-2], k_ctx, v.data_ptr(), vs[-3], vs[-2],
              v_ctx, tokens, n_ctx, max_len, start_p, len_p, index_p, _at(mask), out.data_ptr(), os[1], os[2], os[0], n,
              heads, kv_heads, d, n_q, d ** -0.5 if scale is None else scale, _at(scratch), floats))
    return out


def text_attention(q, k, v, max_len, start=None, length=None, mask=None, causal=False, prefix=None, cap=None, bias=None,
                   slope=None, scale=None, out=None):
    """Attention inside texts of their own lengths.  Packed texts: q [tokens,
    heads, d], k, v [tokens, kv_heads, d], text c at rows start[c] .. start[c +
    1] - 1 (int32 [n + 1], not decreasing), mask (bool or uint8) [tokens].
    Padded texts (start None): q [n, max_len, heads, d] and so on, length int32
    [n] or None (all max_len), mask [n, max_len].  No text is longer than
    max_len.  causal: a query sees the keys up to its own, and the first
    prefix[c] (int32 [n]) of its text.  cap: a score s becomes cap tanh(s /
    cap).  bias fp32 [heads, 2 reach + 1] is added by key less query, constant
    past its ends; slope fp32 [heads] times their distance is taken off.  heads may be a
    multiple of kv_heads (shared in order); q, k, v and out may be strided as
    long as d is contiguous.  scale defaults to 1 / sqrt(d).  A query that sees
    no key gives zeros.  Returns q's shape and type; rows in no text are zeros
    in a new result and stay as they are in `out`."""
    dt = q.dtype
    if dt is not torch.bfloat16 and dt is not torch.float32:
        raise TypeError(dt)
    packed = start is not None
    qshape, kshape = q.shape, k.shape
    if len(qshape) != (3 if packed else 4) or len(kshape) != len(qshape):
        _bad("q, k, v [tokens, heads, d] with start, [n, max_len, heads, d] without")
    heads, d = qshape[-2:]
    kv_heads = kshape[-2]
    if k.dtype is not dt or v.dtype is not dt or kshape != v.shape or kshape[0] != qshape[0] or kshape[-1] != d or (
            not packed and kshape[1] != qshape[1]):
        _bad("k and v must have q's type, tokens and width, and one shape")
    qs, ks, vs = q.stride(), k.stride(), v.stride()
    if d > 1 and (qs[-1] != 1 or ks[-1] != 1 or vs[-1] != 1):
        _bad("d must be contiguous")
    if packed:
        if start.dim() != 1 or start.shape[0] < 1:
            _bad("start must be int32 [n + 1]")
        n, tokens, q_text, k_text, v_text = start.shape[0] - 1, qshape[0], 0, 0, 0
        if length is not None:
            _bad("packed texts end where the next one starts: no length")
    else:
        n, tokens, q_text, k_text, v_text = qshape[0], 0, qs[0], ks[0], vs[0]
        if qshape[1] != max_len:
            _bad("padded q, k, v must be [n, max_len, heads, d]")
    _int32(n | tokens | heads | kv_heads | d | abs(max_len))
    start_p = _index(start, n + 1, "start") if packed else None
    length_p = _index(length, n, "length") if length is not None else None
    prefix_p = _index(prefix, n, "prefix") if prefix is not None else None
    if mask is not None and ((mask.dtype is not torch.bool and mask.dtype is not torch.uint8) or mask.shape != qshape[:-2]
                             or not mask.is_contiguous()):
        _bad("mask must be bool or uint8, one value per token")
    reach = 0
    if bias is not None:
        if bias.dtype is not torch.float32 or bias.dim() != 2 or bias.shape[0] != heads or bias.shape[1] % 2 == 0 or (
                not bias.is_contiguous()):
            _bad("bias must be fp32 [heads, 2 reach + 1], contiguous")
        reach = bias.shape[1] // 2
        _int32(reach)
    if slope is not None and (slope.dtype is not torch.float32 or slope.shape != (heads,) or not slope.is_contiguous()):
        _bad("slope must be fp32 [heads]")
    if cap is not None and not cap > 0:
        _bad("cap must be above 0")
    fresh = out is None
    if fresh:
        out = q.new_empty(qshape)
        if n == 0:
            out.zero_()
    elif out.shape != qshape or out.dtype is not dt:
        _bad("out must have q's shape and type")
    os = out.stride()
    if d > 1 and os[-1] != 1:
        _bad("out must have a contiguous d")
    _enqueue(lib().synerdiff_op_text_attention, q, (k, v, start, length, mask, prefix, bias, slope, out),
             (_TYPE[dt], q.data_ptr(), qs[-3], qs[-2], q_text, k.data_ptr(), ks[-3], ks[-2], k_text, v.data_ptr(), vs[-3],
              vs[-2], v_text, out.data_ptr(), os[-3], os[-2], 0 if packed else os[0], tokens, n, max_len, start_p, length_p,
              _at(mask), 1 if causal else 0, prefix_p, cap or 0.0, _at(bias), reach, _at(slope), heads, kv_heads, d,
              d ** -0.5 if scale is None else scale, 1 if fresh else 0))
    return out


def linear_adapters(x, w, down, up, index, scale=None, bias=None, out=None):
    """x [..., K] (fp32 or bf16, contiguous) times w [N, K], plus a low-rank
    adapter of each row's own: + scale[c] up[c] (down[c] x), with down [count,
    rank, K] and up [count, N, rank] in x's type.  index int32, c of every row
    (shape x.shape[:-1]) or of every x[i] (shape x.shape[:1]); outside [0,
    count): none.  scale fp32 [count] (default 1), bias fp32 [N].  K, N and
    rank are multiples of 8 (narrower adapters padded with zeros).  Returns
    [..., N] in x's type, out when given (a matrix out may have rows further apart)."""
    dt = x.dtype
    if dt is not torch.bfloat16 and dt is not torch.float32:
        raise TypeError(dt)
    shape = x.shape
    if len(shape) < 2 or w.dim() != 2 or down.dim() != 3 or up.dim() != 3:
        _bad("x [..., K], w [N, K], down [count, rank, K], up [count, N, rank]")
    K, N = shape[-1], w.shape[0]
    count, rank = down.shape[:2]
    if w.dtype is not dt or down.dtype is not dt or up.dtype is not dt:
        _bad("w, down and up must have x's type")
    if w.shape[1] != K or down.shape[2] != K or up.shape != (count, N, rank):
        _bad("w, down and up must be [N, K], [count, rank, K] and [count, N, rank]")
    if not (x.is_contiguous() and w.is_contiguous() and down.is_contiguous() and up.is_contiguous()):
        _bad("x, w, down and up must be contiguous")
    if K == 0:
        _bad("K must be above 0")
    M = x.numel() // K
    _int32(M | K | N | count | rank)
    if index.dtype is not torch.int32 or not index.is_contiguous():
        _bad("index must be int32, contiguous")
    ishape = index.shape
    if len(ishape) == 1 and ishape[0] == shape[0]:
        group = max(M // shape[0], 1) if shape[0] else 1
    elif ishape == shape[:-1]:
        group = 1
    else:
        _bad("index must have one entry per row of x, or per x[i]")
    if scale is not None and (scale.dtype is not torch.float32 or scale.shape != (count,) or not scale.is_contiguous()):
        _bad("scale must be fp32 [count]")
    if bias is not None and (bias.dtype is not torch.float32 or bias.shape != (N,) or not bias.is_contiguous()):
        _bad("bias must be fp32 [N]")
    if out is None:
        out, out_ld = x.new_empty((M, N) if len(shape) == 2 else shape[:-1] + (N,)), N
    else:
        if out.shape != shape[:-1] + (N,) or out.dtype is not dt:
            _bad("out has another shape or type than the result")
        out_ld = _row_stride(out, "out")
    L, t = lib(), _TYPE[dt]
    floats, scratch = 0, None
    if M * rank > 64:  # (fewer need none)
        floats = L.synerdiff_op_linear_adapters_scratch_floats(t, M, rank)
        if floats > 0:
            scratch = x.new_empty(floats, dtype=torch.float32)
    _enqueue(L.synerdiff_op_linear_adapters, x, (w, down, up, index, scale, bias, out),
             (t, x.data_ptr(), M, K, w.data_ptr(), N, down.data_ptr() if count else None, up.data_ptr() if count else None, rank,
              count, _at(scale), index.data_ptr(), group, _at(bias), out.data_ptr(), out_ld, _at(scratch), floats))
    return out
