"""Plain 64-bit forms of a decoder's operators with bounds on what one evaluation in the kernels' precisions
may be off, and operators bound to tensors on a device.

Bounds count roundings: `half` is half a step of the result's type (fp16 2^-11, fp32 2^-24, relative to the
value; below the normal range half a subnormal step), an fp32 operation 2^-24 of its result, and a sum of products on the matrix cores one rounding per
step of its accumulator (32 products in fp16, 4 in fp32) and per product inside a step."""
import numpy as np
import torch

from paper_2312_10351_amd import binding as B
from paper_2312_10351_amd.runtime import Session
from workloads import Builder, Workload

U = 2.0 ** -24
HALF = {"f16": 2.0 ** -11, "f32": 2.0 ** -24}
TINY = {"f16": 2.0 ** -25, "f32": 2.0 ** -149}
TORCH = {"f16": torch.float16, "f32": torch.float32}


# rows, columns of residual norms that take every form
NORM = [(1, 1), (1, 768), (5, 1024), (3, 1027), (77, 33), (4, 4096), (2, 8200), (3, 16384), (2, 16385), (1, 20011), (2, 2051), (3, 6000),
        (4300, 40), (1100, 2056), (2100, 7)]
# rows, K, columns of gated blocks that take every form the planner has
GATED = [(1, 8, 1), (1, 64, 33), (2, 768, 2048), (3, 1027, 100), (4, 4096, 512), (5, 256, 96), (16, 512, 130), (17, 40, 31), (33, 320, 640),
         (64, 64, 64), (77, 768, 2048), (128, 1024, 768), (130, 200, 72), (257, 512, 520), (300, 33, 257), (512, 2048, 1024),
         (300, 1024, 2100), (520, 512, 4100), (1000, 640, 4000), (2040, 1032, 4090), (256, 264, 4092)]

# batch, m, n, heads, kv_heads, width, v_width, lengths, causal, first
ATTEND = [
    (1, 1, 1, 1, 1, 8, 8, None, None, 0),
    (1, 1, 1500, 12, 12, 64, 64, None, None, 0),
    (1, 1, 5000, 8, 2, 128, 128, None, None, 0),
    (1, 3, 4099, 6, 1, 64, 128, None, "end", 0),
    (4, 77, 130, 4, 4, 64, 64, [130, 1, 0, 77], None, 0),
    (3, 20, 50, 6, 2, 32, 48, [-5, 99, 13], "end", 0),
    (1, 128, 128, 2, 1, 128, 128, None, "start", 0),
    (2, 65, 65, 3, 3, 40, 40, None, "start", 0),
    (1, 30, 90, 2, 2, 64, 64, None, "start", 60),
    (1, 30, 90, 2, 2, 64, 64, None, "start", -10),
    (1, 5, 33, 2, 1, 20, 24, None, None, 0),
    (2, 9, 70, 2, 2, 37, 19, [70, 31], "end", 0),
    (1, 50, 300, 1, 1, 256, 256, None, None, 0),
    (1, 2, 3000, 4, 4, 200, 72, None, "start", 2998),
    (1, 16, 31, 7, 1, 96, 96, None, None, 0),
    (1, 200, 515, 8, 4, 128, 128, [515], "end", 0),
    (2, 300, 300, 4, 2, 64, 64, [300, 201], "start", 0),
    (1, 513, 257, 2, 2, 128, 64, None, "end", 0),
    (1, 1, 20000, 1, 1, 64, 64, None, None, 0),
    (1, 12, 150, 1, 1, 130, 30, None, None, 0),
    (1, 700, 2100, 4, 1, 64, 64, [2077], "end", 0),
    (1, 1000, 1000, 8, 8, 128, 128, None, "start", 0),
    (2, 700, 130, 8, 8, 128, 96, [101, 130], None, 0),
    (1, 1000, 130, 8, 8, 48, 64, None, "end", 0),
    (2, 333, 1111, 12, 12, 64, 40, [1111, 5], None, 0),
    (3, 1500, 400, 24, 8, 96, 128, [400, 0, 77], None, 0),
    (2, 40, 300, 4, 2, 101, 77, [300, 222], "end", 0),
    (1, 300, 12000, 7, 1, 128, 128, None, "start", 11650),
    (1, 1000, 1000, 24, 8, 64, 64, None, "start", 0),
    (2, 600, 5000, 6, 1, 64, 56, [5000, 3], None, 0),
    (1, 70, 700, 4, 4, 128, 104, [680], "end", 0),
    (1, 200, 6000, 2, 1, 64, 64, None, "end", 0),
    (1, 1, 1500, 12, 4, 128, 128, [1499], None, 0),
]


def normal(gen, shape, dtype, std=1.0, mean=0.0):
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * std + mean).to(TORCH[dtype])


def within(got, want, bound, dtype, what=""):
    got, want, bound = (t.double().cpu() for t in (got, want, bound))
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.isfinite(got).all(), what
    over = (got - want).abs() - (HALF[dtype] * want.abs() + TINY[dtype] + bound)
    i = int(over.argmax())
    assert over.max() <= 0, (f"{what}: {int((over > 0).sum())} of {over.numel()} off; worst at {np.unravel_index(i, got.shape)}: "
                             f"{got.reshape(-1)[i]} for {want.reshape(-1)[i]}, {float(over.max())} over the bound")


def bind(build, tensors, weights=None, dtype="f16", device="cuda:0"):
    """A session of the operators that build(builder, external ids) adds, over tensors on the device."""
    b = Builder("operators", dtype)
    on = [t.to(device) for t in tensors]
    build(b, [b.ext(t.shape) for t in on])
    w = {v: {k: None if t is None else t.to(device) for k, t in d.items()} for v, d in (weights or {}).items()}
    return Session(Workload(b.name, dtype, b.ops, on, w), device=device)


def rotary(x, heads, width, rotated, interleaved, positions, base=10000.0, factor=1.0, original=0.0, low=1.0, high=4.0, alpha=1.0):
    """(value, bound).  The frequency table is in 2^-64 turns, so a position p adds p * 2^-65 turns; the kernels'
    sine and cosine are off by 2^-19 in fp16 (the hardware's) and by three roundings in fp32."""
    m = x.shape[0]
    dtype = "f16" if x.dtype == torch.float16 else "f32"
    i = torch.arange(rotated // 2, dtype=torch.float64)
    f = float(base) ** (-2.0 * i / rotated)
    if original > 0:
        keep = ((original * f / (2 * np.pi) - low) / (high - low)).clamp(0, 1)
        f = f * keep + f / factor * (1 - keep)
    else:
        f = f / factor
    p = torch.as_tensor(positions, dtype=torch.float64)
    angle = p[:, None] * f
    y = x.double().view(m, heads, width).clone()
    a, b = (slice(0, rotated, 2), slice(1, rotated, 2)) if interleaved else (slice(0, rotated // 2), slice(rotated // 2, rotated))
    u, v = y[..., a].clone(), y[..., b].clone()
    c, s = alpha * angle.cos()[:, None], alpha * angle.sin()[:, None]
    y[..., a], y[..., b] = u * c - v * s, v * c + u * s
    # an angle in float64 is off by 2^-53 of itself, in the table by p * 2^-65 turns
    off = (2.0 ** -19 if dtype == "f16" else 6 * U) + p.abs().max() * (2.0 ** -52 + 2 * np.pi * 2.0 ** -65)
    bound = torch.zeros_like(y)
    bound[..., a] = bound[..., b] = abs(alpha) * off * (u.abs() + v.abs())
    return y.view(m, -1), bound.view(m, -1)


def _norm(x, off, w, b, rms, eps):
    """Norm of rows x that are off by at most `off`, and a bound on the result.  A statistic adds up to 64 values
    one after another in a lane, then eleven partial sums: 75 roundings, taken as 2^-17."""
    n = x.shape[1]
    mean = x.mean(1, keepdim=True) if not rms else torch.zeros_like(x[:, :1])
    d = x - mean
    k = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + eps)
    size = x.abs().max(1, keepdim=True).values
    doff = off.max(1, keepdim=True).values * (1 if rms else 2) + 2.0 ** -17 * size * (0 if rms else 1) + U * size
    y = d * k
    # |y| rows have mean square at most one; k is off relatively by that of the root mean square
    yoff = doff * k + y.abs() * (2.0 ** -17 + doff * k + (doff * k) ** 2)
    w, b = (None if t is None else t.double() for t in (w, b))
    yoff = yoff * (1.0 if w is None else w.abs()) + 4 * U * (y.abs() * (1.0 if w is None else w.abs()) + (0.0 if b is None else b.abs()))
    return y * (1.0 if w is None else w) + (0.0 if b is None else b), yoff


def residual_norm(x, r=None, g=None, w=None, b=None, rms=True, after=False, before=True, alpha=1.0, beta=1.0, eps=1e-5):
    """((result, bound), (sum, bound) or None)."""
    z, off = x.double(), torch.zeros(x.shape, dtype=torch.float64)
    row = lambda t, i: None if t is None else t[i]
    if after:
        z, off = _norm(z, off, row(w, 0), row(b, 0), rms, eps)
    if g is not None:
        g = g.double().repeat_interleave(x.shape[0] // g.shape[0], 0)
        z, off = z * g, off * g.abs()
    terms = (beta * z).abs() + (0.0 if r is None else (alpha * r.double()).abs())
    s, off = beta * z + (0.0 if r is None else alpha * r.double()), abs(beta) * off + 4 * U * terms
    if not before:
        return (s, off), None
    return _norm(s, off, row(w, -1), row(b, -1), rms, eps), (s, off)


def _gate(name, x):
    if name == "silu":
        return x * torch.sigmoid(x)
    if name == "gelu":
        return 0.5 * x * torch.special.erfc(-x / np.sqrt(2.0))
    if name == "gelu_tanh":
        return x * torch.sigmoid(2 * np.sqrt(2 / np.pi) * (x + 0.044715 * x ** 3))
    return x.clamp(min=0) if name == "relu" else torch.sigmoid(x)


def gated(x, w, b, act, dtype):
    """(value, bound).  No activation is steeper than 1.13; in fp16 the error function is off by 1.5e-7 and the
    hardware's exponential and reciprocal by 2^-20."""
    x, w = x.double(), w.double()
    n, k = w.shape[0] // 2, x.shape[1]
    y, size = x @ w.t(), x.abs() @ w.abs().t()
    if b is not None:
        y, size = y + b.double(), size + b.double().abs()
    gamma = ((k / 32 + 36) if dtype == "f16" else (k / 4 + 8)) * U
    a, u = _gate(act, y[:, :n]), y[:, n:]
    aoff = 1.13 * gamma * size[:, :n] + (1 + y[:, :n].abs()) * 2.0 ** (-20 if dtype == "f16" else -22)
    uoff = gamma * size[:, n:]
    return a * u, aoff * u.abs() + a.abs() * uoff + aoff * uoff + 2 * U * (a * u).abs()


def attention(q, k, v, dtype, batch=1, heads=1, kv_heads=None, width=64, v_width=None, alpha=None, lengths=None, causal=None, first=0):
    """(value, bound) on the tensors' device.  A score is off by its products' roundings and by three of its
    own size, a probability relatively by twice that of the largest score plus the exponential's 2^-22; in
    fp16 it is rounded once; the sums over the keys take at most n / 64 + 64 roundings a lane."""
    kv_heads, v_width = kv_heads or heads, v_width or width
    alpha = width ** -0.5 if alpha is None else alpha
    m, n = q.shape[0] // batch, k.shape[0] // batch
    q, k, v = (t.double() for t in (q, k, v))
    y = torch.zeros(batch * m, heads * v_width, dtype=torch.float64, device=q.device)
    off = torch.zeros_like(y)
    gamma = ((width / 32 + 36) if dtype == "f16" else (width / 4 + 8)) * U
    for b in range(batch):
        length = n if lengths is None else int(min(max(int(lengths[b]), 0), n))
        if length == 0:
            continue
        i, j = torch.arange(m, device=q.device)[:, None], torch.arange(length, device=q.device)[None]
        seen = (j <= i + {None: n + m, "start": first, "end": length - m}[causal]).expand(m, length)
        for h in range(heads):
            g = h // (heads // kv_heads)
            qb, kb = q[b * m:(b + 1) * m, h * width:(h + 1) * width], k[b * n:b * n + length, g * width:(g + 1) * width]
            vb = v[b * n:b * n + length, g * v_width:(g + 1) * v_width]
            s = (alpha * (qb @ kb.t())).masked_fill(~seen, -np.inf)
            soff = (abs(alpha) * gamma * (qb.abs() @ kb.abs().t()) + 3 * U * s.abs()).masked_fill(~seen, 0.0).amax(1, keepdim=True)
            p = torch.softmax(s, 1).nan_to_num(0.0)
            rel = 4 * soff + 2.0 ** -21 + (n / 64 + 64) * U + (2.0 ** -11 if dtype == "f16" else 0.0)
            y[b * m:(b + 1) * m, h * v_width:(h + 1) * v_width] = p @ vb
            off[b * m:(b + 1) * m, h * v_width:(h + 1) * v_width] = rel * (p @ vb.abs())
            if dtype == "f16":       # probabilities below fp16's normal range are off by half its smallest step
                off[b * m:(b + 1) * m, h * v_width:(h + 1) * v_width] += 2.0 ** -25 * (seen.double() @ vb.abs()) / torch.exp(s - s.amax(1, keepdim=True)).nan_to_num(0.0).sum(1, keepdim=True).clamp(min=1.0)
    return y, off


MORE = {name for name, _ in B.OpMore._fields_}


def describe(op_type, dtype, n_inputs, **fields):
    """(OpDesc, OpMore) of one operator with fake addresses where none are given."""
    d, e = B.OpDesc(), B.OpMore()
    d.op_type, d.op_class, d.dtype, d.n_inputs = op_type, B.CLASS_DEFAULT, B.F16 if dtype == "f16" else B.F32, n_inputs
    for i in range(n_inputs):
        d.inputs[i] = -(i + 1)
    d.out = 0x100000
    for name, value in fields.items():
        if name == "strides":
            for i in range(4):
                for j in range(3):
                    e.strides[i][j] = value[i][j]
        elif name in MORE:
            setattr(e, name, value)
        else:
            setattr(d if name in ("weight", "bias", "out") else d.params, name, value)
    return d, e


def build(*ops, ext=8):
    """Kernels the library takes for operators from `describe`."""
    dag = B.opara_build_dag_more([d for d, _ in ops], [e for _, e in ops], [0x1000000 * (i + 1) for i in range(ext)])
    kernels = [B.opara_kernel_info(x.kernel_id)[0] for x in B.opara_get_demands(dag)]
    B.load().opara_dag_destroy(dag)
    return kernels
