"""Operator definitions in fp64 numpy (test oracle; not used by the product path).

Each function is the plain mathematical definition of one operator type of the
model DAG (paper Sec. 3.1: a vertex is a DNN operator such as Conv or MaxPool).
The paper does not define the operators' arithmetic (it uses vendor libraries,
Sec. 5.1), so the standard definitions are used; readings where a config is silent
are stated per function.  Inputs and outputs are fp64 arrays; rounding to the
storage type happens in the executor, between operators.
"""
import numpy as np
from scipy.special import erf


def conv2d(x, w, b, stride, pad, relu):
    """Cross-correlation with zero padding, dilation 1, groups 1, floor output size.
    x [Cin,H,W], w [Cout,Cin,kh,kw], b [Cout];
    y[co,oh,ow] = b[co] + sum_{ci,i,j} x[ci, oh*sh+i-ph, ow*sw+j-pw] * w[co,ci,i,j]."""
    cin, h, wd = x.shape
    cout, cin2, kh, kw = w.shape
    assert cin == cin2
    sh, sw = stride
    ph, pw = pad
    ho = (h + 2 * ph - kh) // sh + 1
    wo = (wd + 2 * pw - kw) // sw + 1
    xp = np.zeros((cin, h + 2 * ph, wd + 2 * pw), dtype=np.float64)
    xp[:, ph:ph + h, pw:pw + wd] = x
    y = np.zeros((cout, ho, wo), dtype=np.float64)
    for i in range(kh):
        for j in range(kw):
            patch = xp[:, i:i + sh * (ho - 1) + 1:sh, j:j + sw * (wo - 1) + 1:sw]
            y += np.tensordot(w[:, :, i, j], patch, axes=([1], [0]))
    y += b[:, None, None]
    return np.maximum(y, 0.0) if relu else y


def gemm(x, w, b, extras=(), relu=False):
    """Y = X.W + b (+ sum of extra [M,N] inputs); X [M,K], W [K,N], b [N]."""
    y = x @ w + b[None, :]
    for e in extras:
        y = y + e
    return np.maximum(y, 0.0) if relu else y


def bgemm_qk(q, k, heads, alpha):
    """Per-head scaled scores S_h = alpha * Q_h . K_h^T; q,k [S, heads*d] -> [heads,S,S].
    No mask, no dropout."""
    s, hd = q.shape
    d = hd // heads
    out = np.empty((heads, s, s), dtype=np.float64)
    for h in range(heads):
        out[h] = alpha * (q[:, h * d:(h + 1) * d] @ k[:, h * d:(h + 1) * d].T)
    return out


def bgemm_pv(p, v, heads, alpha=1.0):
    """Per-head context C_h = alpha * P_h . V_h, heads written back side by side:
    p [heads,S,S], v [S, heads*d] -> [S, heads*d]."""
    s, hd = v.shape
    d = hd // heads
    out = np.empty((s, hd), dtype=np.float64)
    for h in range(heads):
        out[:, h * d:(h + 1) * d] = alpha * (p[h] @ v[:, h * d:(h + 1) * d])
    return out


def _windows(x, k, stride, pad, fill):
    c, h, w = x.shape
    kh, kw = k
    sh, sw = stride
    ph, pw = pad
    ho = (h + 2 * ph - kh) // sh + 1
    wo = (w + 2 * pw - kw) // sw + 1
    xp = np.full((c, h + 2 * ph, w + 2 * pw), fill, dtype=np.float64)
    xp[:, ph:ph + h, pw:pw + w] = x
    for i in range(kh):
        for j in range(kw):
            yield xp[:, i:i + sh * (ho - 1) + 1:sh, j:j + sw * (wo - 1) + 1:sw]


def maxpool(x, k, stride, pad):
    """Window maximum, padding acts as -inf, floor output size."""
    y = None
    for win in _windows(x, k, stride, pad, -np.inf):
        y = win.copy() if y is None else np.maximum(y, win)
    return y


def avgpool(x, k, stride, pad):
    """Window mean with zero padding, divisor always kh*kw (padding counted)."""
    y = None
    for win in _windows(x, k, stride, pad, 0.0):
        y = win.copy() if y is None else y + win
    return y / float(k[0] * k[1])


def gavgpool(x):
    """Mean over H x W; [C,H,W] -> [C,1,1]."""
    return x.mean(axis=(1, 2), keepdims=True)


def concat(xs, axis):
    """Join along the channel axis ([C,H,W], axis 0) or the columns ([R,C], axis 1)."""
    return np.concatenate(xs, axis=axis)


def _sum(xs):
    y = xs[0]
    for e in xs[1:]:
        y = y + e
    return y


def layernorm(xs, eps):
    """Row-wise (x-mean)/sqrt(var+eps) with biased variance, gamma=1, beta=0,
    applied to the sum of the inputs."""
    x = _sum(xs)
    mu = x.mean(axis=-1, keepdims=True)
    var = ((x - mu) ** 2).mean(axis=-1, keepdims=True)
    return (x - mu) / np.sqrt(var + eps)


def softmax(xs):
    """Row-wise softmax over the last axis (max-subtracted) of the sum of the inputs."""
    x = _sum(xs)
    e = np.exp(x - x.max(axis=-1, keepdims=True))
    return e / e.sum(axis=-1, keepdims=True)


def gelu(xs):
    """Exact (erf) GELU 0.5*x*(1+erf(x/sqrt(2))) of the sum of the inputs."""
    x = _sum(xs)
    return 0.5 * x * (1.0 + erf(x / np.sqrt(2.0)))


def relu(xs):
    return np.maximum(_sum(xs), 0.0)


def add(xs):
    return _sum(xs)


def rotary(x, heads, width, rotated, interleaved, positions, base, factor, original, low, high, alpha=1.0):
    """Every head's first `rotated` columns in pairs, as complex numbers, times alpha * exp(i p f_j): pair j is
    (2j, 2j+1) or (j, j + rotated/2), f_j = base^(-2j/rotated) radians per position.  Stretched for
    long contexts: f_j / factor; with original > 0 only for pairs that turn less than `low` times within
    `original` positions, unchanged from `high` turns on, mixed linearly in the number of turns between."""
    m = x.shape[0]
    j = np.arange(rotated // 2)
    f = np.power(float(base), -2.0 * j / rotated)
    if original > 0:
        turns = original * f / (2.0 * np.pi)
        keep = np.clip((turns - low) / (high - low), 0.0, 1.0)
        f = keep * f + (1.0 - keep) * f / factor
    else:
        f = f / factor
    z = alpha * np.exp(1j * np.asarray(positions, dtype=np.float64)[:, None] * f[None, :])[:, None, :]
    y = x.reshape(m, heads, width).copy()
    a, b = (slice(0, rotated, 2), slice(1, rotated, 2)) if interleaved else (slice(0, rotated // 2), slice(rotated // 2, rotated))
    c = (y[..., a] + 1j * y[..., b]) * z
    y[..., a], y[..., b] = c.real, c.imag
    return y.reshape(m, heads * width)


def residual_norm(x, residual, gate, w, b, rms, after, before, alpha, beta, eps):
    """(result, sum or None).  z = x or its norm; s = alpha * residual + beta * gate * z, a gate row serving
    rows / gates rows in turn; the result is the norm of s (the sum beside it) or s.  w, b: a row per norm."""
    def norm(t, i):
        if not rms:
            t = t - t.mean(axis=-1, keepdims=True)
        t = t / np.sqrt((t * t).mean(axis=-1, keepdims=True) + eps)
        return t * (1.0 if w is None else w[i]) + (0.0 if b is None else b[i])
    z = norm(x, 0) if after else x
    if gate is not None:
        z = z * np.repeat(gate, x.shape[0] // gate.shape[0], axis=0)
    s = beta * z + (0.0 if residual is None else alpha * residual)
    return (norm(s, int(after)), s) if before else (s, None)


def gated(x, w, b, activation):
    """activation(X.Wg + bg) * (X.Wu + bu); w [K, 2N], gate columns first."""
    g, u = np.split(x @ w + b[None, :], 2, axis=1)
    act = {"silu": lambda t: t / (1.0 + np.exp(-t)), "gelu": lambda t: 0.5 * t * (1.0 + erf(t / np.sqrt(2.0))),
           "gelu_tanh": lambda t: 0.5 * t * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (t + 0.044715 * t ** 3))),
           "relu": lambda t: np.maximum(t, 0.0), "sigmoid": lambda t: 1.0 / (1.0 + np.exp(-t))}[activation]
    return act(g) * u


def attention(q, k, v, batch, heads, kv_heads, width, v_width, alpha, lengths=None, causal=None, first=0):
    """Softmax of alpha Q.K^T over the visible keys, times V, head by head; a run of heads / kv_heads query heads
    shares a key head.  A query row sees the first `lengths[b]` keys, of these, causal "start", the first
    i + first + 1 and, causal "end", the first i + lengths[b] - m + 1; one that sees none gives zeros."""
    m, n = q.shape[0] // batch, k.shape[0] // batch
    y = np.zeros((batch * m, heads * v_width))
    for b in range(batch):
        length = n if lengths is None else int(min(max(lengths[b], 0), n))
        for h in range(heads):
            g = h // (heads // kv_heads)
            kb = k[b * n:b * n + length, g * width:(g + 1) * width]
            vb = v[b * n:b * n + length, g * v_width:(g + 1) * v_width]
            for i in range(m):
                seen = length if causal is None else min(length, i + 1 + (first if causal == "start" else length - m))
                if seen <= 0:
                    continue
                s = alpha * (kb[:seen] @ q[b * m + i, h * width:(h + 1) * width])
                e = np.exp(s - s.max())
                y[b * m + i, h * v_width:(h + 1) * v_width] = (e @ vb[:seen]) / e.sum()
    return y
