"""The operators of a decoder block, as cases that can be timed and compared.

Four operators: rotary positions, attention (of states of another length, or causal over
the own ones), the norms around a residual sum, and the gated half of a feed-forward block.
A case is one call of one of them.  `prepare` makes what a program that serves a model holds
before the call (activations, weights, the DAG bound to them), `run` is one pass through the
operator on the caller's stream.

With `own` false the operators are computed in their plain form from elementary torch
operations, in 32 bits (angles in 64), rounded once.
"""
import math

import torch

own = False

_TYPES = {"f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # The query of one token far into a long text (BERT-sized heads, half layout): launch latency.
        {"name": "rotary_token", "op": "rotary", "dtype": "f16", "m": 1, "heads": 12, "width": 64, "rotated": 64, "pairs": "half",
         "first": 1048000, "base": 10000.0, "factor": 1.0, "original": 0.0, "low": 0.0, "high": 0.0},
        # Keys or queries of a whole prompt, interleaved pairs in a part of the head, stretched for long contexts.
        {"name": "rotary_prompt", "op": "rotary", "dtype": "f16", "m": 4096, "heads": 32, "width": 128, "rotated": 96, "pairs": "interleaved",
         "first": 60000, "base": 500000.0, "factor": 8.0, "original": 8192.0, "low": 1.0, "high": 4.0},
        # Between two blocks of one token: the residual sum and the next block's norm.
        {"name": "norm_token", "op": "norm", "dtype": "f16", "m": 1, "n": 768, "kind": "rms", "after": False, "gates": 0, "alpha": 1.0, "beta": 1.0},
        # The same for a prompt, with a norm after the block too, one gate per channel and a scaled residual.
        {"name": "norm_prompt", "op": "norm", "dtype": "f16", "m": 4096, "n": 4096, "kind": "rms", "after": True, "gates": 1, "alpha": 0.7071, "beta": 1.0},
        # Odd rows in fp32, mean and variance, a gate for every element.
        {"name": "norm_ragged", "op": "norm", "dtype": "f32", "m": 1000, "n": 1027, "kind": "layer", "after": True, "gates": 1000, "alpha": 1.0, "beta": 0.5},
        # One token through the gated half of a large feed-forward block: both weights are read once.
        {"name": "gated_token", "op": "gated", "dtype": "f16", "m": 1, "k": 4096, "n": 12288, "act": "silu"},
        # A sentence of 77 tokens through a BERT-sized block in fp32.
        {"name": "gated_sentence", "op": "gated", "dtype": "f32", "m": 77, "k": 768, "n": 2048, "act": "gelu"},
        # A long prompt through the large block: matrix cores.
        {"name": "gated_prompt", "op": "gated", "dtype": "f16", "m": 4096, "k": 4096, "n": 12288, "act": "silu"},
        # One decoder token looks at the 1500 states of an encoder.
        {"name": "cross_token", "op": "attention", "dtype": "f16", "batch": 1, "m": 1, "n": 1500, "heads": 12, "kv_heads": 12,
         "width": 64, "v_width": 64, "mask": "none"},
        # A padded batch of sentences looks at states of other lengths, one of them empty, in fp32.
        {"name": "cross_batch", "op": "attention", "dtype": "f32", "batch": 4, "m": 77, "n": 512, "heads": 12, "kv_heads": 12,
         "width": 64, "v_width": 64, "mask": "lengths"},
        # One token of a long conversation with shared key and value heads: the states are read once.
        {"name": "long_token", "op": "attention", "dtype": "f16", "batch": 1, "m": 1, "n": 65536, "heads": 32, "kv_heads": 8,
         "width": 128, "v_width": 128, "mask": "none"},
        # Causal attention of a long prompt: matrix cores.
        {"name": "long_prompt", "op": "attention", "dtype": "f16", "batch": 1, "m": 8192, "n": 8192, "heads": 32, "kv_heads": 8,
         "width": 128, "v_width": 128, "mask": "causal"},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(("rotary", "norm", "gated", "gated", "attention", "attention", "attention"))
    dtype = rng.choice(("f16", "f16", "f32"))
    case = {"op": op, "dtype": dtype}
    if op == "rotary":
        width = rng.choice((64, 80, 96, 128, 2 * rng.randint(8, 128)))
        rotated = rng.choice((width, width, 2 * rng.randint(1, width // 2)))
        case.update(m=_spread(rng, 1, 4096), heads=rng.randint(1, 32), width=width, rotated=rotated, pairs=rng.choice(("half", "interleaved")),
                    first=_spread(rng, 1, 1 << 20) - 1, base=rng.choice((10000.0, 500000.0)), factor=rng.choice((1.0, 4.0, 8.0)), original=0.0,
                    low=0.0, high=0.0)
        if rng.random() < 0.5:
            case.update(original=8192.0, low=1.0, high=4.0)
    elif op == "norm":
        n = rng.choice((8 * _spread(rng, 8, 1024), _spread(rng, 50, 4096)))
        m = _spread(rng, 1, max(1, min(4096, (4096 * 4096 if dtype == "f16" else 2048 * 4096) // n)))
        case.update(m=m, n=n, kind=rng.choice(("rms", "layer")), after=rng.random() < 0.5, gates=rng.choice((0, 1, m)),
                    alpha=rng.choice((1.0, 0.7071)), beta=rng.choice((1.0, 0.5)))
    elif op == "gated":
        k = rng.choice((64 * _spread(rng, 2, 64), _spread(rng, 100, 2048)))
        n = rng.choice((64 * _spread(rng, 4, 192), _spread(rng, 100, 4096)))
        most = 4096 * 4096 * 12288 if dtype == "f16" else 1 << 34
        if k % 8:                                   # rows that no vector reads: smaller models
            most = 1 << 33
        case.update(m=_spread(rng, 1, max(1, min(4096, most // (k * n)))), k=k, n=n, act=rng.choice(("silu", "gelu", "gelu_tanh", "relu", "sigmoid")))
    else:
        kv = rng.randint(1, 8)
        heads = kv * rng.choice((1, 1, 2, 4, 7))
        width = rng.choice((64, 64, 128, 128, 8 * rng.randint(2, 32), rng.randint(10, 130)))
        v_width = rng.choice((width, width, width, 8 * rng.randint(2, 16)))
        mask = rng.choice(("none", "lengths", "causal", "causal_end"))
        batch = 1 if mask in ("none", "causal") else rng.randint(1, 5)
        m = rng.choice((1, 1, _spread(rng, 2, 4096)))
        most = min(1 << 31, 400_000_000_000 // (width + v_width)) if dtype == "f16" else 1 << 27          # scores
        if width % 8 or v_width % 8:
            most = 1 << 26
        n = m if mask == "causal" and m > 1 else _spread(rng, 1, 65536)
        n = max(1, min(n, most // (m * heads * batch)))
        case.update(batch=batch, m=min(m, n) if mask == "causal" else m, n=n, heads=heads, kv_heads=kv, width=width, v_width=v_width, mask=mask)
    return case


# ---- inputs ---------------------------------------------------------------------------

def _inputs(case, seed):
    """Activations N(0, 1), weights N(0, 0.02) and around one for norms; lengths spread over the range,
    one of them zero where there are several."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = _TYPES[case["dtype"]]
    normal = lambda *shape, std=1.0, mean=0.0, dtype=t: torch.empty(shape, dtype=dtype, device="cuda").normal_(mean, std, generator=g)
    op = case["op"]
    if op == "rotary":
        return {"x": normal(case["m"], case["heads"] * case["width"]), "first": case["first"] + seed % 7}
    if op == "norm":
        norms = 2 if case["after"] else 1
        d = {"x": normal(case["m"], case["n"]), "r": normal(case["m"], case["n"], std=2.0),
             "w": normal(norms, case["n"], std=0.1, mean=1.0), "b": normal(norms, case["n"], std=0.1, dtype=torch.float32)}
        if case["gates"]:
            d["g"] = normal(case["gates"], case["n"], std=0.5)
        return d
    if op == "gated":
        return {"x": normal(case["m"], case["k"]), "w": normal(2 * case["n"], case["k"], std=0.02),
                "b": normal(2 * case["n"], std=0.02, dtype=torch.float32)}
    b, m, n = case["batch"], case["m"], case["n"]
    d = {"q": normal(b * m, case["heads"] * case["width"]), "k": normal(b * n, case["kv_heads"] * case["width"]),
         "v": normal(b * n, case["kv_heads"] * case["v_width"])}
    if case["mask"] in ("lengths", "causal_end"):
        lengths = [n - (n * i * (1 + seed % 3)) // (4 * b) for i in range(b)]
        if b > 1:
            lengths[-1] = 0
        d["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    return d


class _Bound:
    """One operator as a DAG bound to its tensors; `outputs`: where its results are."""

    def __init__(self, session, outputs):
        self.session, self.outputs = session, outputs

    def __del__(self):
        self.session.close()


def _bind(case, d):
    from paper_2312_10351_amd.runtime import Session
    from workloads import Builder, Workload
    b = Builder(case["op"], case["dtype"])
    op, weights = case["op"], {}
    if op == "rotary":
        tensors = [d["x"]]
        x = b.ext(d["x"].shape)
        b.rotary(x, case["heads"], case["width"], rotated=case["rotated"], interleaved=case["pairs"] == "interleaved", first=d["first"],
                 base=case["base"], factor=case["factor"], original=case["original"], low=case["low"], high=case["high"])
    elif op == "norm":
        tensors = [d["x"], d["r"]] + ([d["g"]] if case["gates"] else [])
        x, r = b.ext(d["x"].shape), b.ext(d["r"].shape)
        gate = b.ext(d["g"].shape) if case["gates"] else None
        b.residual_norm(x, r, gate=gate, rms=case["kind"] == "rms", after=case["after"], before=True, alpha=case["alpha"], beta=case["beta"], eps=1e-5)
        weights = {0: {"w": d["w"], "b": d["b"]}}
    elif op == "gated":
        tensors = [d["x"]]
        b.gated(b.ext(d["x"].shape), case["m"], case["k"], case["n"], activation=case["act"])
        weights = {0: {"w": d["w"], "b": d["b"]}}
    else:
        tensors = [d["q"], d["k"], d["v"]] + ([d["lengths"]] if "lengths" in d else [])
        q, k, v = (b.ext(d[name].shape) for name in "qkv")
        lengths = b.ext(d["lengths"].shape) if "lengths" in d else None
        b.attention(q, k, v, heads=case["heads"], kv_heads=case["kv_heads"], width=case["width"], v_width=case["v_width"], batch=case["batch"],
                    lengths=lengths, causal={"causal": "start", "causal_end": "end"}.get(case["mask"]),
                    first=case["n"] - case["m"] if case["mask"] == "causal" else 0, alpha=case["width"] ** -0.5)
    s = Session(Workload(b.name, b.dtype, b.ops, tensors, weights), device="cuda:0")
    return _Bound(s, [s.result(0), s.result(0, second=True)] if op == "norm" else [s.result(0)])


def prepare(case, seed):
    d = _inputs(case, seed)
    return _bind(case, d) if own else (case, d)


# ---- one pass -------------------------------------------------------------------------

def run(state):
    if own:
        state.session.launch()
        return state.outputs
    case, d = state
    return _PLAIN[case["op"]](case, d)


def _turns(case):
    """Turns per position of every pair of a head, as float64."""
    i = torch.arange(case["rotated"] // 2, dtype=torch.float64, device="cuda")
    f = case["base"] ** (-2.0 * i / case["rotated"]) / (2.0 * math.pi)
    if case["high"] > 0.0:
        mix = ((case["original"] * f - case["low"]) / (case["high"] - case["low"])).clamp(0.0, 1.0)
        return f * (mix + (1.0 - mix) / case["factor"])
    return f / case["factor"]


def _plain_rotary(case, d):
    m, h, w, r = case["m"], case["heads"], case["width"], case["rotated"]
    x = d["x"].float().view(m, h, w)
    p = torch.arange(m, dtype=torch.float64, device="cuda") + d["first"]
    a = p[:, None] * _turns(case)
    a = (a - a.floor()) * (2.0 * math.pi)
    c, s = a.cos().float()[:, None], a.sin().float()[:, None]
    y = x.clone()
    if case["pairs"] == "half":
        u, v = x[..., :r // 2], x[..., r // 2:r]
        y[..., :r // 2], y[..., r // 2:r] = u * c - v * s, v * c + u * s
    else:
        u, v = x[..., 0:r:2], x[..., 1:r:2]
        y[..., 0:r:2], y[..., 1:r:2] = u * c - v * s, v * c + u * s
    return [y.view(m, h * w).to(d["x"].dtype)]


def _plain_norm(case, d):
    def norm(x, w, b):
        if case["kind"] == "layer":
            x = x - x.mean(-1, keepdim=True)
        return x / ((x * x).mean(-1, keepdim=True) + 1e-5).sqrt() * w.float() + b
    t = d["x"].dtype
    z = d["x"].float()
    if case["after"]:
        z = norm(z, d["w"][0], d["b"][0])
    if case["gates"]:
        z = (z.view(case["gates"], -1, case["n"]) * d["g"].float()[:, None]).view(case["m"], case["n"])
    s = case["alpha"] * d["r"].float() + case["beta"] * z
    return [norm(s, d["w"][-1], d["b"][-1]).to(t), s.to(t)]


def _act(name, x):
    if name == "silu":
        return x / (1.0 + (-x).exp())
    if name == "gelu":
        return 0.5 * x * (1.0 + (x * math.sqrt(0.5)).erf())
    if name == "gelu_tanh":
        return 0.5 * x * (1.0 + (math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)).tanh())
    return x.clamp(min=0.0) if name == "relu" else 1.0 / (1.0 + (-x).exp())


def _plain_gated(case, d):
    y = d["x"].float() @ d["w"].float().t() + d["b"]
    return [(_act(case["act"], y[:, :case["n"]]) * y[:, case["n"]:]).to(d["x"].dtype)]


def _seen(case, d):
    """[batch, m, n]: which key rows a query row sees; None: all of them."""
    if case["mask"] == "none":
        return None
    b, m, n = case["batch"], case["m"], case["n"]
    i, j = torch.arange(m, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
    if case["mask"] == "causal":
        return (j <= i + (n - m)).expand(b, m, n)
    lengths = d["lengths"].long()[:, None, None]
    inside = (j < lengths).expand(b, m, n)
    return inside if case["mask"] == "lengths" else inside & (j <= i + lengths - m)


def _plain_attention(case, d):
    b, m, n, h, kv, w, vw = (case[name] for name in ("batch", "m", "n", "heads", "kv_heads", "width", "v_width"))
    share = h // kv
    q = d["q"].float().view(b, m, kv, share, w).permute(0, 2, 3, 1, 4).reshape(b, kv, share * m, w)
    k = d["k"].float().view(b, n, kv, w).permute(0, 2, 3, 1).contiguous()
    v = d["v"].float().view(b, n, kv, vw).permute(0, 2, 1, 3).contiguous()
    s = (q @ k).view(b, kv, share, m, n) * case["width"] ** -0.5
    seen = _seen(case, d)
    if seen is None:
        p = (s - s.amax(-1, keepdim=True)).exp()
        p = p / p.sum(-1, keepdim=True)
    else:
        seen = seen[:, None, None]
        s = s.masked_fill(~seen, -math.inf)
        top = s.amax(-1, keepdim=True)
        p = (s - top.masked_fill(top == -math.inf, 0.0)).exp()
        total = p.sum(-1, keepdim=True)
        p = p / total.masked_fill(total == 0.0, 1.0)
    y = p.reshape(b, kv, share * m, n) @ v
    return [y.view(b, kv, share, m, vw).permute(0, 3, 1, 2, 4).reshape(b * m, h * vw).to(d["q"].dtype)]


_PLAIN = {"rotary": _plain_rotary, "norm": _plain_norm, "gated": _plain_gated, "attention": _plain_attention}


# ---- what a pass cannot do without --------------------------------------------------------

def work(case):
    es = 2 if case["dtype"] == "f16" else 4
    if case["op"] == "rotary":
        cells = case["m"] * case["heads"] * case["width"]
        return {"bytes": 2 * cells * es, "flops": 3 * case["m"] * case["heads"] * case["rotated"]}
    if case["op"] == "norm":
        cells, norms = case["m"] * case["n"], 2 if case["after"] else 1
        return {"bytes": (4 * cells + case["gates"] * case["n"]) * es + norms * case["n"] * (es + 4), "flops": (4 + 6 * norms) * cells}
    if case["op"] == "gated":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": (m * k + 2 * n * k + m * n) * es + 8 * n, "flops": 4 * m * n * k}
    b, m, n, h, kv, w, vw = (case[name] for name in ("batch", "m", "n", "heads", "kv_heads", "width", "v_width"))
    rows = [n - (n * i) // (4 * b) for i in range(b)] if case["mask"] in ("lengths", "causal_end") else [n] * b
    if case["mask"] in ("lengths", "causal_end") and b > 1:
        rows[-1] = 0
    pairs = 0
    for length in rows:
        seen = m * length
        if case["mask"] in ("causal", "causal_end"):          # query row i sees length - m + i + 1 rows, none below zero
            few = min(m, length)
            seen = few * length - few * (few - 1) // 2
        pairs += seen
    return {"bytes": (b * m * h * (w + vw) + sum(rows) * kv * (w + vw)) * es, "flops": 2 * pairs * h * (w + vw)}


# ---- the definitions in 64 bits ---------------------------------------------------------

def exact(case, seed):
    d = {name: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for name, v in _inputs(case, seed).items()}
    op = case["op"]
    if op == "rotary":
        # A pair is a complex number; a rotation is a product with exp(i angle).
        m, r = case["m"], case["rotated"]
        x = d["x"].view(m, case["heads"], case["width"])
        turns = []
        for i in range(r // 2):
            f = 1.0 / (2.0 * math.pi * case["base"] ** (2.0 * i / r))
            if case["high"] > 0.0:
                count = case["original"] * f               # turns within the original length
                if count <= case["low"]:
                    f = f / case["factor"]
                elif count < case["high"]:
                    share = (count - case["low"]) / (case["high"] - case["low"])
                    f = f * share + f / case["factor"] * (1.0 - share)
            else:
                f = f / case["factor"]
            turns.append(f)
        angle = torch.tensor(turns, dtype=torch.float64, device="cuda") * (torch.arange(m, device="cuda") + d["first"]).double()[:, None]
        turn = torch.polar(torch.ones_like(angle), 2.0 * math.pi * angle.frac())[:, None]
        head, rest = x[..., :r], x[..., r:]
        if case["pairs"] == "half":
            z = torch.complex(head[..., :r // 2].contiguous(), head[..., r // 2:].contiguous()) * turn
            head = torch.cat([z.real, z.imag], -1)
        else:
            z = torch.view_as_complex(head.reshape(m, case["heads"], r // 2, 2)) * turn
            head = torch.view_as_real(z).reshape(m, case["heads"], r)
        return [torch.cat([head, rest], -1).view(m, -1)]
    if op == "norm":
        def stats(x):
            mean = x.sum(1) / case["n"] if case["kind"] == "layer" else torch.zeros_like(x[:, 0])
            c = x - mean[:, None]
            return c * ((c.square().sum(1) / case["n"] + 1e-5) ** -0.5)[:, None]
        z = d["x"]
        if case["after"]:
            z = stats(z) * d["w"][0] + d["b"][0].double()
        if case["gates"]:
            z = z * d["g"].repeat_interleave(case["m"] // case["gates"], 0)
        s = d["r"] * case["alpha"] + z * case["beta"]
        return [stats(s) * d["w"][-1] + d["b"][-1].double(), s]
    if op == "gated":
        gate, up = d["w"][:case["n"]], d["w"][case["n"]:]
        a, u = torch.addmm(d["b"][:case["n"]], d["x"], gate.t()), torch.addmm(d["b"][case["n"]:], d["x"], up.t())
        act = {"silu": lambda x: x * torch.sigmoid(x), "gelu": lambda x: x * 0.5 * torch.special.erfc(-x / math.sqrt(2.0)),
               "gelu_tanh": lambda x: x * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3)),
               "relu": lambda x: torch.where(x > 0.0, x, torch.zeros_like(x)), "sigmoid": torch.sigmoid}[case["act"]]
        return [act(a) * u]
    b, m, n, h, w, vw = (case[name] for name in ("batch", "m", "n", "heads", "width", "v_width"))
    y = torch.zeros(b * m, h * vw, dtype=torch.float64, device="cuda")
    for i in range(b):
        length = int(d["lengths"][i]) if "lengths" in d else n
        if length == 0:
            continue
        last = {"causal": n - m, "causal_end": length - m}.get(case["mask"])
        for head in range(h):
            g = head * case["kv_heads"] // h
            s = d["q"][i * m:(i + 1) * m, head * w:(head + 1) * w] @ d["k"][i * n:i * n + length, g * w:(g + 1) * w].t() / math.sqrt(w)
            if last is not None:
                s += torch.full_like(s, -math.inf).triu(last + 1)
            p = torch.softmax(s, 1).nan_to_num_(0.0)           # rows that see nothing
            y[i * m:(i + 1) * m, head * vw:(head + 1) * vw] = p @ d["v"][i * n:i * n + length, g * vw:(g + 1) * vw]
    return [y]
