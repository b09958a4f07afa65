"""A decoder's operators on the GPU against their 64-bit forms, at the sizes and masks where they can go wrong."""
import numpy as np
import pytest
import torch

import decoder_util as D
from oracle import executor
from paper_2312_10351_amd import binding as B
from paper_2312_10351_amd.runtime import Session
from util import compare_all, mismatch
from workloads import Builder, Second, Workload, decoder_like

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def run(session):
    session.launch()
    torch.cuda.synchronize()
    return session


def gen(seed):
    return torch.Generator().manual_seed(seed)


# ---- rotary positions ----------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("m, heads, width, rotated, first", [
    (1, 1, 2, 2, 0), (1, 12, 64, 64, 1048575), (7, 3, 80, 32, 100), (33, 5, 96, 96, -20), (5, 4, 130, 66, 70000),
    (3, 2, 37, 10, 9), (200, 9, 128, 128, 0), (2, 70, 256, 254, 2 ** 31 - 3), (1, 2, 4096, 4096, 5)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary(dtype, m, heads, width, rotated, first, interleaved):
    x = D.normal(gen(m * width + heads), (m, heads * width), dtype)
    kw = dict(base=500000.0, factor=8.0, original=512.0, low=1.0, high=4.0, alpha=0.9) if m % 2 else {}
    s = D.bind(lambda b, e: b.rotary(e[0], heads, width, rotated, interleaved, first, **kw), [x], dtype=dtype)
    want, bound = D.rotary(x, heads, width, rotated, interleaved, first + np.arange(m, dtype=np.int64), **kw)
    D.within(run(s).result(0), want, bound, dtype)
    copied = torch.arange(heads * width) % width >= rotated
    assert torch.equal(s.result(0).cpu()[:, copied], x[:, copied])
    s.close()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_rotary_takes_positions_from_memory(dtype):
    """The table of positions is read at every launch: a captured graph follows it."""
    x = D.normal(gen(3), (6, 4 * 64), dtype)
    pos = torch.tensor([0, 5, 5, -7, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    s = D.bind(lambda b, e: b.rotary(e[0], 4, 64, positions=e[1]), [x, pos], dtype=dtype)
    D.within(run(s).result(0), *D.rotary(x, 4, 64, 64, False, pos), dtype)
    exe = s.capture(B.SEQUENTIAL)
    for step in range(3):
        pos = pos // 2 + step
        s.ext_dev[1].copy_(pos)
        torch.cuda.synchronize()
        s.replay(exe)
        D.within(s.result(0), *D.rotary(x, 4, 64, 64, False, pos), dtype)
    s.close()


def eager(op, tensors, dtype):
    """One operator from its records over device tensors."""
    dag = B.opara_build_dag_more([op[0]], [op[1]], [t.data_ptr() for t in tensors])
    B.opara_run_eager(dag, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    B.load().opara_dag_destroy(dag)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("lead, pitch", [(0, 3 * 128 + 8), (1, 3 * 128 + 1)])
def test_rotary_rows_apart_and_unaligned(dtype, lead, pitch):
    m, heads, width = 9, 3, 128
    x = torch.zeros(m * pitch + lead, dtype=D.TORCH[dtype], device=DEV)
    y = torch.full_like(x, 7.0)
    rows = D.normal(gen(1), (m, heads * width), dtype)
    view = lambda t: t[lead:lead + m * pitch].view(m, pitch)[:, :heads * width]
    view(x).copy_(rows)
    table = torch.tensor(np.array(B.opara_rotary_table(width), dtype=np.uint64).view(np.int64), device=DEV)
    d = D.describe(B.ROTARY, dtype, 1, m=m, heads=heads, width=width, rotated=width, alpha=1.0, a_row_stride=pitch, c_row_stride=pitch,
                   weight=table.data_ptr(), out=y[lead:].data_ptr())
    eager(d, [x[lead:]], dtype)
    D.within(view(y), *D.rotary(rows, heads, width, width, False, np.arange(m)), dtype)
    between = y.clone()
    view(between).fill_(7.0)
    assert (between == 7.0).all()                              # nothing written between the rows


# ---- the norms around a residual sum ------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("m, n", D.NORM)
@pytest.mark.parametrize("rms, after, before, gates", [(True, False, True, 0), (False, True, True, 1), (True, True, False, -1), (False, False, True, -1)])
def test_residual_norm(dtype, m, n, rms, after, before, gates):
    g = gen(m * n + after)
    gates = m if gates < 0 else gates
    x, r = D.normal(g, (m, n), dtype, 1.0, 0.5), D.normal(g, (m, n), dtype, 2.0)
    gate = D.normal(g, (gates, n), dtype) if gates else None
    w, b = D.normal(g, (after + before, n), dtype, 0.1, 1.0), D.normal(g, (after + before, n), "f32", 0.1)
    kw = dict(rms=rms, after=after, before=before, alpha=0.75, beta=1.5)
    s = D.bind(lambda bl, e: bl.residual_norm(e[0], e[1], e[2] if gates else None, **kw), [x, r] + ([gate] if gates else []),
               {0: {"w": w, "b": b}}, dtype)
    y, second = D.residual_norm(x, r, gate, w, b, **kw)
    D.within(run(s).result(0), *y, dtype, "result")
    if before:
        D.within(s.result(0, second=True), *second, dtype, "sum")
    s.close()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_residual_norm_without_residual_weights_or_sum(dtype):
    x = D.normal(gen(4), (6, 520), dtype)
    y = torch.zeros(6, 520, dtype=D.TORCH[dtype], device=DEV)
    xd = x.to(DEV)
    d = D.describe(B.RESIDUAL_NORM, dtype, 1, m=6, n=520, eps=1e-6, alpha=5.0, beta=0.5, flags=B.FLAG_NORM_BEFORE | B.FLAG_RMS, out=y.data_ptr())
    eager(d, [xd], dtype)
    D.within(y, *D.residual_norm(x, beta=0.5, eps=1e-6)[0], dtype)
    d[0].params.flags = 0                                         # no norm at all: the scaled block
    eager(d, [xd], dtype)
    D.within(y, *D.residual_norm(x, beta=0.5, before=False)[0], dtype)


def test_residual_norm_gate_rows_serve_runs_of_rows():
    x, r, g = (D.normal(gen(i), s, "f16") for i, s in enumerate([(12, 96), (12, 96), (3, 96)]))
    s = D.bind(lambda b, e: b.residual_norm(e[0], e[1], e[2], before=False, weights=False), [x, r, g])
    D.within(run(s).result(0), *D.residual_norm(x, r, g, before=False)[0], "f16")
    s.close()


def test_residual_norm_rows_of_zeros():
    x = torch.zeros(2, 640, dtype=torch.float16)
    s = D.bind(lambda b, e: b.residual_norm(e[0], e[0], rms=False, after=True, weights=False), [x])
    assert not run(s).result(0).any() and not s.result(0, second=True).any()
    s.close()


# ---- the gated block ------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("i", range(len(D.GATED)))
def test_gated(dtype, i):
    m, k, n = D.GATED[i]
    act = list(B.ACTIVATION_IDS)[i % 5]
    g = gen(i)
    x, w, b = D.normal(g, (m, k), dtype), D.normal(g, (2 * n, k), dtype, 1.0 / np.sqrt(k)), D.normal(g, (2 * n,), "f32", 0.1)
    s = D.bind(lambda bl, e: bl.gated(e[0], m, k, n, act), [x], {0: {"w": w, "b": b}}, dtype)
    D.within(run(s).result(0), *D.gated(*(t.to(DEV) for t in (x, w, b)), act, dtype), dtype, act)
    s.close()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("act", list(B.ACTIVATION_IDS))
@pytest.mark.parametrize("m", [1, 40])
def test_gated_activations_over_their_range(dtype, act, m):
    """One product per result: the gate runs from deep saturation to large values."""
    n = 96
    x = torch.ones(m, 8, dtype=D.TORCH[dtype])
    w = torch.zeros(2 * n, 8, dtype=D.TORCH[dtype])
    w[:n, 0] = torch.linspace(-90, 90, n)
    w[n:, 3] = 1.0
    s = D.bind(lambda b, e: b.gated(e[0], m, 8, n, act), [x], {0: {"w": w, "b": torch.zeros(2 * n)}}, dtype)
    D.within(run(s).result(0), *D.gated(x, w, None, act, dtype), dtype, act)
    s.close()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("m, k, n, lda, ldy, lead", [(3, 64, 40, 72, 48, 0), (20, 128, 33, 131, 35, 1), (90, 256, 64, 264, 72, 0), (140, 512, 256, 520, 264, 0)])
def test_gated_rows_apart_unaligned_and_without_bias(dtype, m, k, n, lda, ldy, lead):
    g = gen(m)
    rows, w = D.normal(g, (m, k), dtype), D.normal(g, (2 * n, k), dtype, 1.0 / np.sqrt(k))
    x = torch.full((lead + m * lda,), float("nan"), dtype=D.TORCH[dtype], device=DEV)   # what lies between the rows is not read
    x[lead:].view(m, lda)[:, :k].copy_(rows)
    y = torch.full((lead + m * ldy,), 7.0, dtype=D.TORCH[dtype], device=DEV)
    wd = torch.zeros(lead + 2 * n * k, dtype=D.TORCH[dtype], device=DEV)
    wd[lead:].view(2 * n, k).copy_(w)
    d = D.describe(B.GATED, dtype, 1, m=m, n=n, k=k, activation=1, a_row_stride=lda, c_row_stride=ldy, weight=wd[lead:].data_ptr(),
                   out=y[lead:].data_ptr())
    eager(d, [x[lead:]], dtype)
    D.within(y[lead:].view(m, ldy)[:, :n], *D.gated(rows, w, None, "gelu", dtype), dtype)
    assert (y[lead:].view(m, ldy)[:, n:] == 7.0).all()


# ---- attention -----------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("i", range(len(D.ATTEND)))
def test_attention(dtype, i):
    batch, m, n, heads, kv, width, v_width, lengths, causal, first = D.ATTEND[i]
    g = gen(i)
    q, k, v = (D.normal(g, s, dtype) for s in [(batch * m, heads * width), (batch * n, kv * width), (batch * n, kv * v_width)])
    ext = [q, k, v]
    if lengths is not None:
        # rows behind a sequence's length hold anything
        for b, length in enumerate(lengths):
            for t, bad in ((k, float("nan")), (v, float("inf"))):
                t.view(batch, n, -1)[b, min(max(length, 0), n):] = bad
        ext.append(torch.tensor(lengths, dtype=torch.int32))
    kw = dict(heads=heads, width=width, kv_heads=kv, v_width=v_width, batch=batch, causal=causal, first=first)
    s = D.bind(lambda b, e: b.attention(*e[:3], lengths=e[3] if lengths is not None else None, **kw), ext, dtype=dtype)
    want, bound = D.attention(*(t.to(DEV) for t in (q, k, v)), dtype, lengths=lengths, **kw)
    first_run = run(s).result(0).clone()
    D.within(first_run, want, bound, dtype)
    assert torch.equal(run(s).result(0), first_run)            # the same bits from launch to launch
    s.close()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("m", [1, 40, 150])
def test_attention_of_large_scores(dtype, m):
    """Scores of hundreds: the running maximum moves in steps of many powers of two."""
    g = gen(m)
    q, k, v = (D.normal(g, (r, 2 * 64), dtype, std) for r, std in ((m, 8.0), (700, 8.0), (700, 1.0)))
    s = D.bind(lambda b, e: b.attention(*e, heads=2, width=64), [q, k, v], dtype=dtype)
    D.within(run(s).result(0), *D.attention(*(t.to(DEV) for t in (q, k, v)), dtype, heads=2, width=64), dtype)
    s.close()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("m, n, scratch", [(1, 3000, True), (1, 3000, False), (130, 200, True)])
def test_attention_through_strides(dtype, m, n, scratch):
    """Heads before rows, rows apart, keys and values in one buffer; nothing else is written."""
    heads, kv, width, batch = 4, 2, 64, 2
    g = gen(n)
    q, k, v = (D.normal(g, s, dtype) for s in [(batch * m, heads * width), (batch * n, kv * width), (batch * n, kv * width)])
    both = torch.full((batch, kv, n, 2 * width + 8), float("nan"), dtype=D.TORCH[dtype], device=DEV)
    both[..., :width] = k.view(batch, n, kv, width).permute(0, 2, 1, 3)
    both[..., width:2 * width] = v.view(batch, n, kv, width).permute(0, 2, 1, 3)
    qd = q.view(batch, m, heads, width).permute(0, 2, 1, 3).contiguous().to(DEV)
    y = torch.full((heads, batch, m, width + 16), 7.0, dtype=D.TORCH[dtype], device=DEV)
    row = 2 * width + 8
    strides = [[heads * m * width, width, m * width], [kv * n * row, row, n * row], [kv * n * row, row, n * row],
               [m * (width + 16), width + 16, batch * m * (width + 16)]]
    d = D.describe(B.ATTENTION, dtype, 3, batch=batch, m=m, n=n, heads=heads, kv_heads=kv, width=width, alpha=0.125, strides=strides, out=y.data_ptr())
    d[1].scratch_bytes = B.opara_scratch_bytes(*d)
    assert d[1].scratch_bytes > 0 or m > 1
    room = torch.zeros(max(d[1].scratch_bytes, 256), dtype=torch.uint8, device=DEV)
    d[1].scratch = room.data_ptr() if scratch else None
    eager(d, [qd, both, both[..., width:]], dtype)
    want, bound = D.attention(*(t.to(DEV) for t in (q, k, v)), dtype, batch=batch, heads=heads, kv_heads=kv, width=width)
    got = y[..., :width].permute(1, 2, 0, 3).reshape(batch * m, heads * width)
    D.within(got, want, bound, dtype)
    assert (y[..., width:] == 7.0).all()


def test_attention_lengths_are_read_at_every_launch():
    """A cache that fills: one captured graph serves every length, and leaves its scratch memory ready for the next."""
    n, heads, kv, width = 4000, 8, 2, 128
    g = gen(8)
    q, k, v = (D.normal(g, s, "f16") for s in [(1, heads * width), (n, kv * width), (n, kv * width)])
    length = torch.tensor([1], dtype=torch.int32)
    s = D.bind(lambda b, e: b.attention(*e[:3], heads=heads, width=width, kv_heads=kv, lengths=e[3]), [q, k, v, length])
    exe = s.capture(B.SEQUENTIAL)
    for now in (1, 0, 31, 32, 33, 700, 4000, 3999, 2):
        s.ext_dev[3].fill_(now)
        torch.cuda.synchronize()
        s.replay(exe)
        captured = s.result(0).clone()
        D.within(captured, *D.attention(*(t.to(DEV) for t in (q, k, v)), "f16", heads=heads, kv_heads=kv, width=width, lengths=[now]), "f16", str(now))
        assert torch.equal(run(s).result(0), captured)
    s.close()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("m, heads, kv, width, causal", [(20, 2, 1, 64, "start"), (1000, 8, 4, 128, "start"), (900, 8, 8, 64, "end"), (70, 2, 2, 37, "start"),
                                                         (33, 1, 1, 256, "end"), (129, 3, 3, 130, "start"), (1000, 24, 8, 64, "start"),
                                                         (1300, 8, 4, 128, "start"), (2000, 8, 4, 64, "end")])
def test_attention_of_rows_that_do_not_see_what_is_not_finite(dtype, m, heads, kv, width, causal):
    """Under a causal mask later keys and values may hold anything: rows before them are as without them."""
    first, second = m // 3, m * 2 // 3
    g = gen(m)
    q, k, v = (D.normal(g, (m, h * width), dtype) for h in (heads, kv, kv))
    v[first, 0::4], v[first, 1::4], v[first, 2::4] = np.inf, -np.inf, np.nan
    k[second:], v[second:] = np.nan, np.inf
    kw = dict(heads=heads, width=width, kv_heads=kv, causal=causal)
    s = D.bind(lambda b, e: b.attention(*e, **kw), [q, k, v], dtype=dtype)
    got = run(s).result(0).clone()
    s.close()
    cut = lambda rows: [t.to(DEV) for t in (q[:rows], k[:rows], v[:rows].nan_to_num(0.0, 0.0, 0.0))]
    head = dict(kw, causal="start")
    D.within(got[:first], *D.attention(*cut(first), dtype, **head), dtype, "before")
    want, bound = D.attention(*cut(second), dtype, **head)
    c = torch.arange(heads * width, device=DEV)
    column = (c // width // (heads // kv) * width + c % width) % 4        # of the values
    D.within(got[first:second, column == 3], want[first:second, column == 3], bound[first:second, column == 3], dtype, "finite columns")
    seen = got[first:second].float()
    assert (seen[:, column == 0] == np.inf).all() and (seen[:, column == 1] == -np.inf).all() and seen[:, column == 2].isnan().all()
    assert got[second:].isnan().all()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("m, n, width, causal", [(1, 3000, 64, None), (50, 700, 128, "end"), (1000, 500, 64, "start"), (9, 100, 33, None)])
@pytest.mark.parametrize("alpha", [-0.4, 0.0])
def test_attention_of_any_factor(dtype, m, n, width, causal, alpha):
    g = gen(n)
    q, k, v = (D.normal(g, (r, 4 * width), dtype) for r in (m, n, n))
    kw = dict(heads=4, width=width, causal=causal, alpha=alpha)
    s = D.bind(lambda b, e: b.attention(*e, **kw), [q, k, v], dtype=dtype)
    D.within(run(s).result(0), *D.attention(*(t.to(DEV) for t in (q, k, v)), dtype, **kw), dtype)
    s.close()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("pitch, scratch", [(8, True), (0, False)])
def test_attention_over_windows_of_one_row(dtype, pitch, scratch):
    """Keys and values that overlap, or are one row for all."""
    n, width = 900, 64
    g = gen(pitch)
    row = D.normal(g, (n * 8 + width,), dtype)
    q = D.normal(g, (2, width), dtype)
    keys = row.as_strided((n, width), (pitch, 1)).contiguous()
    y = torch.zeros(2, width, dtype=D.TORCH[dtype], device=DEV)
    d = D.describe(B.ATTENTION, dtype, 3, m=2, n=n, heads=1, width=width, alpha=0.125, out=y.data_ptr(),
                   strides=[[0] * 3, [0, pitch, 1], [0, pitch, 1], [0] * 3])
    d[1].scratch_bytes = B.opara_scratch_bytes(*d) if scratch else 0
    room = torch.zeros(max(256, d[1].scratch_bytes), dtype=torch.uint8, device=DEV)
    d[1].scratch = room.data_ptr() if scratch else None
    eager(d, [q.to(DEV), row.to(DEV), row.to(DEV)], dtype)
    D.within(y, *D.attention(*(t.to(DEV) for t in (q, keys, keys)), dtype, width=width), dtype)


def test_attention_with_less_scratch_than_asked_for():
    q, k, v = (D.normal(gen(i), (r, 4 * 128), "f16") for i, r in enumerate((1, 20000, 20000)))
    on = [t.to(DEV) for t in (q, k, v)]
    want = D.attention(*on, "f16", heads=4, width=128)
    d = D.describe(B.ATTENTION, "f16", 3, m=1, n=20000, heads=4, width=128, alpha=128 ** -0.5)
    asked = B.opara_scratch_bytes(*d)
    for given in (asked, asked // 2, asked // 7, 256, 0):
        y = torch.zeros(1, 4 * 128, dtype=torch.float16, device=DEV)
        room = torch.zeros(given + 256, dtype=torch.uint8, device=DEV)
        room[given:] = 77
        d[0].out, d[1].scratch, d[1].scratch_bytes = y.data_ptr(), room.data_ptr(), given
        eager(d, on, "f16")
        D.within(y, *want, "f16", str(given))
        assert (room[given:] == 77).all()


def test_attention_over_more_than_four_gigabytes_of_keys():
    """Rows far apart: offsets of the last keys pass 32 bits."""
    n, width, pitch = 2100, 64, 1 << 21
    k = torch.zeros(n * pitch, dtype=torch.float16, device=DEV)
    assert k.numel() * 2 > 2 ** 33
    g = gen(9)
    q, kk, vv = (D.normal(g, (r, width), "f16") for r in (1, n, n))
    k.view(n, pitch)[:, :width] = kk.to(DEV)
    k.view(n, pitch)[:, width:2 * width] = vv.to(DEV)
    y = torch.zeros(1, width, dtype=torch.float16, device=DEV)
    d = D.describe(B.ATTENTION, "f16", 3, m=1, n=n, heads=1, width=width, alpha=0.125, out=y.data_ptr(),
                   strides=[[0] * 3, [n * pitch, pitch, width], [n * pitch, pitch, width], [0] * 3])
    eager(d, [q.to(DEV), k, k[width:]], "f16")
    D.within(y, *D.attention(q.to(DEV), kk.to(DEV), vv.to(DEV), "f16", width=width), "f16")


def test_operators_follow_the_callers_stream():
    """Inputs written on a stream just before, results read on it right after."""
    g = gen(10)
    q, k, v = (D.normal(g, (r, 4 * 64), "f16") for r in (1, 900, 900))
    s = D.bind(lambda b, e: b.attention(*e, heads=4, width=64), [q, k, v])
    want = D.attention(*(t.to(DEV) for t in (q, k, v)), "f16", heads=4, width=64)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(5):
        with torch.cuda.stream(side):
            s.ext_dev[1].zero_()
            s.ext_dev[1].copy_(k.to(DEV, non_blocking=False))
            s.launch()
            got = s.result(0).clone()
        side.synchronize()
        D.within(got, *want, "f16")
    s.close()


# ---- together --------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("kw", [dict(seq=1, states=300, past=40), dict(seq=77, states=130, hidden=384, heads=6, kv_heads=2, ffn=520)])
def test_decoder_through_the_graph_executors(dtype, kw):
    wl = decoder_like(dtype=dtype, **kw)
    ref = executor.run_dag(wl)
    s = Session(wl, device=DEV)
    modes = [B.SEQUENTIAL, B.PARALLEL, B.PARALLEL_PRUNED, B.FUSED]
    exes = [s.capture(m) for m in modes]                       # several executors over one set of buffers
    for turn in range(3):
        for mode, exe in zip(modes, exes):
            s.clear_outputs()
            s.replay(exe)
            assert not compare_all(s, ref), (mode, compare_all(s, ref))
            for op in wl.ops:
                if (op.id, 1) in ref:
                    assert mismatch(s.output(op.id, second=True), ref[(op.id, 1)], dtype) is None
        s.clear_outputs()
        s.run_eager()
        assert not compare_all(s, ref)
    kernels = B.opara_fused_node_kernels(exes[-1], dtype)
    node_of, _ = B.opara_fused_plan(exes[-1], len(wl.ops))
    names = {op.name: op.id for op in wl.ops}
    assert node_of[names["L0.rotary_q"]] == node_of[names["L0.rotary_k"]]
    assert kernels[node_of[names["L0.rotary_q"]]] == f"group_{dtype}_decoder"
    s.close()


def test_fused_groups_of_many_row_wise_operators():
    """Twenty rotations and norms of both results in one wave: more than a group holds."""
    b = Builder("wide", "f16")
    x = b.ext((40, 256))
    n = b.residual_norm(x, x)
    for i in range(10):
        b.rotary(Second(n) if i % 2 else n, 4, 64, first=i)
        b.residual_norm(n, Second(n), alpha=0.5 * i, rms=bool(i % 2))
    g = b.gemm(n, 40, 256, 64)
    wl = b.build(3)
    ref = executor.run_dag(wl)
    s = Session(wl, device=DEV)
    exe = s.capture(B.FUSED)
    for _ in range(3):
        s.clear_outputs()
        s.replay(exe)
        assert not compare_all(s, ref)
    node_of, nodes = B.opara_fused_plan(exe, len(wl.ops))
    assert nodes == 4 and node_of[g] not in (node_of[1], node_of[2])      # two groups, the product and the first norm
    t = s.operator_trace(B.FUSED)
    assert (t >= 0).all()
    s.close()


def test_persistent_and_chained_executors_refuse():
    wl = decoder_like(layers=1, seq=8, states=16, hidden=128, heads=2, kv_heads=1, ffn=64)
    s = Session(wl, device=DEV)
    for capture in (s.capture_persistent, s.capture_chained, s.run_persistent_noalloc):
        with pytest.raises(B.OparaError) as e:
            capture()
        assert e.value.status == B.EUNSUPPORTED
    s.close()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_launches_captured_into_the_callers_graph(dtype):
    """A session's launches among a program's own operations, in a graph that is replayed between eager work."""
    wl = decoder_like(dtype=dtype, layers=1, seq=3, states=900, hidden=256, heads=4, kv_heads=2, ffn=300, past=7)
    s = Session(wl, device=DEV)
    run(s)
    x, last = torch.zeros_like(s.ext_dev[0]), len(wl.ops) - 1
    x.copy_(s.ext_dev[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.ext_dev[0].copy_(x)
        s.launch()
        captured = s.result(last) * 2
    for step in range(4):
        x.mul_(0.5).add_(step)
        graph.replay()
        torch.cuda.synchronize()
        got = captured.clone()
        s.clear_outputs()
        assert torch.equal(run(s).result(last) * 2, got) and got.abs().max() > 0
    s.close()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_attentions_beside_each_other(dtype):
    """Independent ones of a wave run at once, each with its own scratch memory."""
    b = Builder("beside", dtype)
    k, v = b.ext((3000, 128)), b.ext((3000, 128))
    for i in range(5):
        b.attention(b.ext((1 + i, 256)), k, v, heads=4, width=64, kv_heads=2, causal="end" if i % 2 else None)
    b.rowwise("add", [0, 0], 1, 256)
    wl = b.build(4)
    ref = executor.run_dag(wl)
    s = Session(wl, device=DEV)
    assert len({s.descs[i].out for i in range(5)}) == 5
    for mode in (B.PARALLEL, B.FUSED, B.SEQUENTIAL):
        exe = s.capture(mode)
        for _ in range(3):
            s.clear_outputs()
            s.replay(exe)
            assert not compare_all(s, ref), mode
    s.close()


def test_two_sessions_at_once():
    """Operators with scratch memory of their own on two streams."""
    g = gen(12)
    pairs = []
    for i in range(2):
        q, k, v = (D.normal(g, (r, 8 * 64), "f16") for r in (1, 6000, 6000))
        s = D.bind(lambda b, e: b.attention(*e, heads=8, width=64), [q, k, v])
        pairs.append((s, torch.cuda.Stream(), D.attention(*(t.to(DEV) for t in (q, k, v)), "f16", heads=8, width=64)))
    torch.cuda.synchronize()
    for _ in range(20):
        for s, stream, _ in pairs:
            s.launch(stream)
    torch.cuda.synchronize()
    for s, _, want in pairs:
        D.within(s.result(0), *want, "f16")
        s.close()


def test_device_tensors_are_checked():
    with pytest.raises(ValueError):
        x = torch.zeros(4, 8, dtype=torch.float16)             # on the host
        b = Builder("host", "f16")
        b.rotary(b.ext((4, 8)), 1, 8)
        Session(Workload("host", "f16", b.ops, [x], {}), device=DEV)
