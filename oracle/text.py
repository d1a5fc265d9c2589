"""Text-side operations, float64: the root-mean-square norm with an 8-bit
output, linear layers with 4-bit weights, and attention over texts of their
own lengths.  Plain textbook definitions, one row at a time."""
import numpy as np

F = np.float64


def e4m3(v):
    """Nearest OCP e4m3 value (ties to even): 3 fraction bits, exponents from
    -6 (subnormals below, in steps of 2^-9) to 8, largest value 448."""
    v = np.asarray(v, F)
    e = np.maximum(np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -20))), -6)
    step = 2.0 ** (e - 3)
    return np.clip(np.rint(v / step) * step, -448, 448)


def rmsnorm(x, gamma=None, eps=1e-6, resid=None):
    """(y, h): h = x + resid, y = h / sqrt(mean(h^2) + eps) * gamma per row."""
    h = np.asarray(x, F) + (0 if resid is None else np.asarray(resid, F))
    y = h / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    return y * (1 if gamma is None else np.asarray(gamma, F)), h


def block_scales(y, group):
    """Scales max(max|y|, 2^-100) / 448 of each row's blocks of `group` channels (0: the row)."""
    C = y.shape[-1]
    g = group or C
    return np.stack([np.maximum(np.abs(y[:, a:a + g]).max(1), 2.0 ** -100) / 448 for a in range(0, C, g)], 1)


def w4_weights(codes, scale, zero, group):
    """[N, K] weights scale * (q - zero) from bytes of two codes (even k low)."""
    N, K = codes.shape[0], 2 * codes.shape[1]
    q = np.empty((N, K), F)
    q[:, 0::2], q[:, 1::2] = codes & 15, codes >> 4
    of = np.arange(K) // group
    z = 8.0 if zero is None else np.asarray(zero, F)[:, of]
    return (q - z) * np.asarray(scale, F)[:, of]


def cross_attention(q, k, v, texts, scale):
    """q [n, n_q, heads, d]; k, v [tokens, kv_heads, d]; texts[i]: the token
    rows that row i attends to.  An empty text gives zeros.  Returns (o, w)
    with w the same sum over |v|, which bounds the rounding of o."""
    q, k, v = (np.asarray(t, F) for t in (q, k, v))
    n, n_q, heads, d = q.shape
    rep = heads // k.shape[1]
    o, w = np.zeros(q.shape, F), np.zeros(q.shape, F)
    for i in range(n):
        rows = np.asarray(texts[i], np.int64)
        if not len(rows):
            continue
        for h in range(heads):
            s = q[i, :, h] @ k[rows, h // rep].T * scale
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            o[i, :, h] = p @ v[rows, h // rep]
            w[i, :, h] = p @ np.abs(v[rows, h // rep])
    return o, w


def text_attention(q, k, v, texts, scale, mask=None, causal=False, prefix=None, cap=None, bias=None, slope=None):
    """Attention inside texts: q [tokens, heads, d], k, v [tokens, kv_heads,
    d], texts[c] = (first row, length), one query at a time.  Rows in no text
    give 0, as do queries without a key that scores above -inf.  Returns (o,
    w), w the same sum over |v|."""
    q, k, v = (np.asarray(t, F) for t in (q, k, v))
    heads, rep = q.shape[1], q.shape[1] // k.shape[1]
    o, w = np.zeros(q.shape, F), np.zeros(q.shape, F)
    for c, (first, size) in enumerate(texts):
        for i in range(size):
            js = [j for j in range(size) if (mask is None or mask[first + j])
                  and (not causal or j <= i or (prefix is not None and j < prefix[c]))]
            if not js:
                continue
            js = np.asarray(js)
            far = js - i
            for h in range(heads):
                s = k[first + js, h // rep] @ q[first + i, h] * scale
                if cap:
                    s = cap * np.tanh(s / cap)
                if bias is not None:
                    reach = bias.shape[1] // 2
                    s = s + np.asarray(bias, F)[h, np.clip(far, -reach, reach) + reach]
                if slope is not None:
                    s = s - float(slope[h]) * np.abs(far)
                on = s > -np.inf
                if not on.any():
                    continue
                p = np.exp(s[on] - s[on].max())
                p /= p.sum()
                o[first + i, h] = p @ v[first + js[on], h // rep]
                w[first + i, h] = p @ np.abs(v[first + js[on], h // rep])
    return o, w


def linear_adapters(x, w, down, up, index, scale=None, bias=None):
    """Rows x [M, K]: w x + bias + scale[c] up[c] (down[c] x), c = index[m]
    where it lies in 0 .. count - 1.  Returns (y, s, t): s the sum of the terms'
    sizes of the shared product, t that of the adapter's, of |down x| times |up|."""
    x, w, down, up = (np.asarray(t, F) for t in (x, w, down, up))
    b = 0 if bias is None else np.asarray(bias, F)
    y = x @ w.T + b
    s = np.abs(x) @ np.abs(w).T + np.abs(b)
    t = np.zeros_like(y)
    for m, c in enumerate(index):
        if 0 <= c < len(down):
            f = 1.0 if scale is None else float(scale[c])
            y[m] += f * (up[c] @ (down[c] @ x[m]))
            t[m] = abs(f) * (np.abs(up[c]) @ (np.abs(down[c]) @ np.abs(x[m])))
    return y, s, t
