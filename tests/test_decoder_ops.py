"""A decoder's operators on the host: the oracle's definitions against values worked out another way, the table of
rotary frequencies, what the library refuses, and how the operators take their place in a DAG."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from decoder_util import ATTEND as ATTEND_SIZES, GATED as GATED_SIZES, NORM as NORM_SIZES, build, describe
from oracle import executor, ops as O
from paper_2312_10351_amd import binding as B
from paper_2312_10351_amd.runtime import Session
from workloads import Builder, Second, Workload, decoder_like


# ---- the oracle ---------------------------------------------------------------------------

@pytest.mark.parametrize("interleaved", [False, True])
def test_oracle_rotary_turns_pairs(interleaved):
    x = np.array([[1.0, 0.0, 0.0, 2.0, 7.0]])
    y = O.rotary(x, 1, 5, 4, interleaved, [3], 100.0, 1.0, 0.0, 1.0, 4.0)
    a, b = 3.0, 0.3                                            # angles of the two pairs
    if interleaved:                                            # (1, 0) and (0, 2)
        want = [math.cos(a), math.sin(a), -2 * math.sin(b), 2 * math.cos(b), 7.0]
    else:                                                      # (x0, x2) = (1, 0), (x1, x3) = (0, 2)
        want = [math.cos(a), -2 * math.sin(b), math.sin(a), 2 * math.cos(b), 7.0]
    np.testing.assert_allclose(y[0], want, atol=1e-14)


def test_oracle_rotary_is_relative():
    """The product of two rotated rows depends on the distance of their positions only."""
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 1, 16))
    turn = lambda x, p: O.rotary(x, 1, 16, 16, False, [p], 10000.0, 4.0, 64.0, 1.0, 4.0)
    assert (turn(q, 5) @ turn(k, 3).T)[0, 0] == pytest.approx((turn(q, 1002) @ turn(k, 1000).T)[0, 0], abs=1e-10)


def test_oracle_residual_norm_by_hand():
    x, r = np.array([[3.0, -1.0]]), np.array([[1.0, 1.0]])
    y, s = O.residual_norm(x, r, np.array([[2.0, 0.5]]), np.array([[1.0, 1.0], [10.0, 10.0]]), np.array([[0.0, 0.0], [1.0, 0.0]]),
                           False, True, True, 0.5, 1.0, 0.0)
    np.testing.assert_allclose(s, [[2.5, 0.0]])                # the norm of (3, -1) is (1, -1)
    np.testing.assert_allclose(y, [[11.0, -10.0]])
    y, s = O.residual_norm(x, None, None, None, None, True, False, False, 1.0, 2.0, 0.0)
    np.testing.assert_allclose(y, [[6.0, -2.0]])
    assert s is None


def test_oracle_gated_by_hand():
    x, w = np.array([[2.0]]), np.array([[1.0, -1.0, 3.0, 0.5]])
    y = O.gated(x, w, np.array([0.0, 0.0, 0.0, 1.0]), "sigmoid")
    np.testing.assert_allclose(y, [[6.0 / (1 + math.exp(-2.0)), 2.0 / (1 + math.exp(2.0))]])
    assert O.gated(x, w, np.zeros(4), "relu")[0, 1] == 0.0
    np.testing.assert_allclose(O.gated(x, w, np.zeros(4), "gelu")[0, 0], 2 * 0.5 * (1 + math.erf(2 / math.sqrt(2))) * 6)


def test_oracle_attention_agrees_with_three_operators():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 6, 8))
    p = O.softmax([O.bgemm_qk(q, k, 2, 0.5).reshape(12, 6)]).reshape(2, 6, 6)
    np.testing.assert_allclose(O.attention(q, k, v, 1, 2, 2, 4, 4, 0.5), O.bgemm_pv(p, v, 2), atol=1e-14)


def test_oracle_attention_masks():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((6, 4)), rng.standard_normal((10, 4)), rng.standard_normal((10, 2))
    y = O.attention(q, k, v, 2, 1, 1, 4, 2, 1.0, lengths=[0, 9], causal="end")
    assert not y[:3].any()                                     # no keys at all
    np.testing.assert_allclose(y[3], O.attention(q[3:4], k[5:8], v[5:8], 1, 1, 1, 4, 2, 1.0)[0])   # length cut to 5; row 0 sees three
    y = O.attention(q, k, v, 2, 1, 1, 4, 2, 1.0, causal="start", first=-1)
    assert not y[0].any() and not y[3].any()
    np.testing.assert_allclose(y[1], v[0])                     # a single visible key


# ---- the table of frequencies --------------------------------------------------------------

@pytest.mark.parametrize("kw", [dict(), dict(base=500000.0, factor=8.0), dict(factor=4.0, original_length=8192.0, low=1.0, high=4.0)])
def test_rotary_table_to_its_last_bits(kw):
    rotated = 64
    table = B.opara_rotary_table(rotated, **kw)
    base, factor, original = kw.get("base", 10000.0), kw.get("factor", 1.0), kw.get("original_length", 0.0)
    two_pi = Fraction(6283185307179586476925286766559, 10 ** 30)
    for i, got in enumerate(table):
        f = Fraction(float(np.longdouble(base) ** (np.longdouble(-2 * i) / rotated))) / two_pi
        if original:
            keep = min(Fraction(1), max(Fraction(0), (Fraction(original) * f - 1) / 3))
            f = f * (keep + (1 - keep) / Fraction(factor))
        else:
            f = f / Fraction(factor)
        assert abs(got - f * 2 ** 64) <= f * 2 ** 64 * Fraction(1, 2 ** 51) + 1, i     # a double's rounding of the power


@pytest.mark.parametrize("kw", [dict(rotated=3), dict(rotated=0), dict(rotated=4098), dict(base=0.0), dict(base=math.inf), dict(factor=-1.0),
                                dict(factor=math.nan), dict(original_length=-1.0), dict(original_length=8.0, low=4.0, high=1.0)])
def test_rotary_table_refuses(kw):
    with pytest.raises(B.OparaError) as e:
        B.opara_rotary_table(**{"rotated": 64, **kw})
    assert e.value.status == B.EINVAL


# ---- refusals ------------------------------------------------------------------------------

ROTARY = dict(m=4, heads=2, width=8, rotated=8, alpha=1.0, weight=0x2000)
NORM = dict(m=4, n=16, eps=1e-5, alpha=1.0, beta=1.0, flags=B.FLAG_NORM_BEFORE)
GATED = dict(m=4, n=16, k=8, weight=0x2000)
ATTEND = dict(m=4, n=9, heads=4, kv_heads=2, width=8, alpha=1.0)


@pytest.mark.parametrize("kind, n_inputs, good, bad", [
    (B.ROTARY, 1, ROTARY, dict(rotated=7)), (B.ROTARY, 1, ROTARY, dict(rotated=10)), (B.ROTARY, 1, ROTARY, dict(rotated=0)),
    (B.ROTARY, 1, ROTARY, dict(width=0)), (B.ROTARY, 1, ROTARY, dict(width=4098)), (B.ROTARY, 1, ROTARY, dict(weight=None)),
    (B.ROTARY, 1, ROTARY, dict(a_row_stride=15)), (B.ROTARY, 1, ROTARY, dict(c_row_stride=-16)), (B.ROTARY, 3, ROTARY, dict()),
    (B.ROTARY, 1, ROTARY, dict(m=0)), (B.ROTARY, 1, ROTARY, dict(heads=1 << 30)), (B.ROTARY, 1, ROTARY, dict(out2=0x900000)),
    (B.RESIDUAL_NORM, 2, NORM, dict(m=0)), (B.RESIDUAL_NORM, 2, NORM, dict(n=-1)), (B.RESIDUAL_NORM, 4, NORM, dict()),
    (B.RESIDUAL_NORM, 3, NORM, dict(batch=3)), (B.RESIDUAL_NORM, 2, NORM, dict(batch=2)), (B.RESIDUAL_NORM, 2, NORM, dict(eps=-1.0)),
    (B.RESIDUAL_NORM, 2, NORM, dict(eps=math.nan)), (B.RESIDUAL_NORM, 2, NORM, dict(flags=0, out2=0x900000)),
    (B.RESIDUAL_NORM, 2, NORM, dict(out2=0x100000)),
    (B.RESIDUAL_NORM, 2, NORM, dict(flags=0, weight=0x2000)),
    (B.GATED, 1, GATED, dict(weight=None)), (B.GATED, 2, GATED, dict()), (B.GATED, 1, GATED, dict(activation=5)),
    (B.GATED, 1, GATED, dict(activation=-1)), (B.GATED, 1, GATED, dict(k=0)), (B.GATED, 1, GATED, dict(a_row_stride=7)),
    (B.GATED, 1, GATED, dict(c_row_stride=15)), (B.GATED, 1, GATED, dict(n=1 << 30)),
    (B.ATTENTION, 3, ATTEND, dict(kv_heads=3)), (B.ATTENTION, 3, ATTEND, dict(width=257)), (B.ATTENTION, 3, ATTEND, dict(v_width=257)),
    (B.ATTENTION, 3, ATTEND, dict(n=0)), (B.ATTENTION, 3, ATTEND, dict(m=0)), (B.ATTENTION, 3, ATTEND, dict(batch=-1)),
    (B.ATTENTION, 2, ATTEND, dict()), (B.ATTENTION, 5, ATTEND, dict()), (B.ATTENTION, 3, ATTEND, dict(flags=B.FLAG_CAUSAL | B.FLAG_CAUSAL_END)),
    (B.ATTENTION, 3, ATTEND, dict(strides=[[0] * 3, [0, -16, 8], [0] * 3, [0] * 3])),
    (B.ATTENTION, 3, ATTEND, dict(strides=[[0] * 3, [0] * 3, [0] * 3, [0, 31, 8]])),     # result rows of 32 elements
    (B.ATTENTION, 3, ATTEND, dict(scratch=0x900080, scratch_bytes=1 << 30)),
])
def test_refuses(kind, n_inputs, good, bad):
    for dtype in ("f16", "f32"):
        if bad:
            build(describe(kind, dtype, n_inputs, **good))
        with pytest.raises(B.OparaError) as e:
            build(describe(kind, dtype, n_inputs, **{**good, **bad}))
        assert e.value.status == B.EINVAL


@pytest.mark.parametrize("kind, n_inputs, good, bad", [
    (B.ROTARY, 1, ROTARY, dict(m=0x7fffffff, width=64)), (B.GATED, 1, GATED, dict(m=0x7fffffff, n=1 << 20)),
    (B.ATTENTION, 3, ATTEND, dict(n=0x7fffffff)), (B.ATTENTION, 3, ATTEND, dict(heads=1 << 17, kv_heads=0)),
])
def test_sizes_past_a_launch_are_refused(kind, n_inputs, good, bad):
    with pytest.raises(B.OparaError) as e:
        build(describe(kind, "f16", n_inputs, **{**good, **bad}))
    assert e.value.status == B.EUNSUPPORTED


def test_second_results_are_named_by_their_readers():
    norm, reader = describe(B.RESIDUAL_NORM, "f16", 2, **NORM, out2=0x900000), describe(B.RESIDUAL_NORM, "f16", 2, **NORM, out=0x200000)
    reader[0].inputs[0], reader[0].inputs[1], reader[1].result_of[1] = 0, 0, 1
    build(norm, reader)

    def refused():
        with pytest.raises(B.OparaError) as e:
            build(norm, reader)
        return e.value.status == B.EINVAL
    for value in (2, -1):                                      # no such result
        reader[1].result_of[1] = value
        assert refused()
    reader[1].result_of[1] = 1
    norm[1].out2 = None                                        # nothing to read
    assert refused()
    norm[1].out2 = 0x900000
    reader[0].inputs[1] = -1                                   # external tensors have one
    assert refused()


def test_operators_that_need_a_record_are_refused_without():
    d, _ = describe(B.GATED, "f16", 1, **GATED)
    with pytest.raises(B.OparaError) as e:
        B.opara_build_dag([d], [0x1000000])
    assert e.value.status == B.EINVAL
    with pytest.raises(ValueError):
        B.opara_build_dag_more([d], [], [0x1000000])


def test_record_layout_matches_header():
    import ctypes
    assert ctypes.sizeof(B.OpMore) == 7 * 4 + 4 + 12 * 8 + 8 + 8 * 4 + 8 + 8


def test_scratch_is_asked_for_where_keys_are_shared_out():
    few = describe(B.ATTENTION, "f16", 3, m=1, n=65536, heads=32, kv_heads=8, width=128, alpha=1.0)
    many = describe(B.ATTENTION, "f16", 3, m=4096, n=4096, heads=32, kv_heads=8, width=128, alpha=1.0)
    short = describe(B.ATTENTION, "f16", 3, m=1, n=60, heads=1, kv_heads=1, width=64, alpha=1.0)
    assert B.opara_scratch_bytes(*few) > 0
    assert B.opara_scratch_bytes(*many) == 0 and B.opara_scratch_bytes(*short) == 0
    assert B.opara_scratch_bytes(describe(B.GATED, "f16", 1, **GATED)[0], None) == 0
    few[1].width = 300
    for more in (few[1], None):
        with pytest.raises(B.OparaError):
            B.opara_scratch_bytes(few[0], more)


def test_norm_sizes_of_the_gpu_tests_reach_every_form():
    every = [B.opara_kernel_info(i)[0] for i in range(B.opara_kernel_count())]
    for dtype in ("f16", "f32"):
        taken = {build(describe(B.RESIDUAL_NORM, dtype, 2, **{**NORM, "m": m, "n": n}))[0] for m, n in NORM_SIZES}
        assert taken == {name for name in every if name.startswith(f"resnorm_{dtype}_")}


def test_gated_sizes_of_the_gpu_tests_reach_every_form():
    for dtype in ("f16", "f32"):
        all_of_them = {B.opara_kernel_info(i)[0] for i in range(B.opara_kernel_count())}
        taken = {build(describe(B.GATED, dtype, 1, m=m, n=n, k=k, weight=0x2000))[0] for m, k, n in GATED_SIZES}
        assert taken == {name for name in all_of_them if name.startswith(f"gated_{dtype}_")}


def test_attention_sizes_of_the_gpu_tests_reach_every_form():
    every = [B.opara_kernel_info(i)[0] for i in range(B.opara_kernel_count())]
    for dtype in ("f16", "f32"):
        taken = {}
        for batch, m, n, heads, kv, width, v_width, _, causal, first in ATTEND_SIZES:
            op = describe(B.ATTENTION, dtype, 3, batch=batch, m=m, n=n, heads=heads, kv_heads=kv, width=width, v_width=v_width,
                          first=first, alpha=1.0, flags={None: 0, "start": B.FLAG_CAUSAL, "end": B.FLAG_CAUSAL_END}[causal])
            op[1].scratch_bytes = B.opara_scratch_bytes(*op)
            op[1].scratch = 0x900000 if op[1].scratch_bytes else None
            taken.setdefault(build(op)[0], set()).add(op[1].scratch_bytes > 0)
        assert set(taken) == {name for name in every if name.startswith(f"attend_{dtype}_")}
        for name in ("rows64", "rows128") + (("wide64", "wide128") if dtype == "f16" else ()):
            assert taken[f"attend_{dtype}_{name}"] == {False, True}, name


@pytest.mark.parametrize("width, v_width, strides, straight", [
    (64, 64, [0, 0, 0], True), (64, 64, [0, 64, 64], True), (64, 64, [0, 8, 0], False), (64, 64, [0, 132, 64], False),
    (60, 64, [0, 128, 64], False), (64, 60, [0, 128, 64], False), (64, 56, [0, 128, 64], True), (64, 64, [0, 1 << 24, 64], False),
    (64, 64, [0, 0, 64], False)])
def test_attention_loads_only_rows_that_it_can_through_buffers(width, v_width, strides, straight):
    """Unaligned, overlapping and far keys take the form that reads them through registers."""
    op = describe(B.ATTENTION, "f16", 3, m=1, n=500, heads=2, kv_heads=2, width=width, v_width=v_width, alpha=1.0,
                  strides=[[0] * 3, strides, [0, 128, 64], [0] * 3])
    assert (build(op) != ["attend_f16_any64"]) == straight


# ---- tensors of a workload ------------------------------------------------------------------

def tensors(**changed):
    """An attention of a batch of two and the gated block and norm after it, over torch tensors (not on a device: host only)."""
    t = dict(q=torch.zeros(6, 32, dtype=torch.float16), k=torch.zeros(10, 32, dtype=torch.float16), lengths=torch.zeros(2, dtype=torch.int32),
             w=torch.zeros(48, 32, dtype=torch.float16), b=torch.zeros(48), g=torch.zeros(1, 24, dtype=torch.float16), nb=torch.zeros(1, 24))
    t.update(changed)
    b = Builder("tensors", "f16")
    e = [b.ext(s) for s in ((6, 32), (10, 32), (2,))]
    a = b.attention(e[0], e[1], e[1], heads=2, width=16, batch=2, lengths=e[2])
    b.residual_norm(b.gated(a, 6, 32, 24))
    return Workload("tensors", "f16", b.ops, [t["q"], t["k"], t["lengths"]], {1: {"w": t["w"], "b": t["b"]}, 2: {"w": t["g"], "b": t["nb"]}})


def test_tensors_used_in_place_are_checked():
    Session(tensors(), device=None)
    Session(tensors(lengths=np.zeros(2, dtype=np.int32)), device=None)
    for bad in (dict(q=torch.zeros(6, 32)), dict(k=torch.zeros(9, 32, dtype=torch.float16)), dict(lengths=torch.zeros(2, dtype=torch.int64)),
                dict(lengths=torch.zeros(1, dtype=torch.int32)), dict(lengths=np.zeros(2, dtype=np.int64)), dict(w=torch.zeros(48, 32)),
                dict(w=torch.zeros(47, 32, dtype=torch.float16)), dict(b=torch.zeros(48, dtype=torch.float16)), dict(b=torch.zeros(24)),
                dict(g=torch.zeros(1, 23, dtype=torch.float16)), dict(nb=torch.zeros(1, 24, dtype=torch.float64))):
        with pytest.raises(ValueError):
            Session(tensors(**bad), device=None)


# ---- in a DAG ------------------------------------------------------------------------------

def test_decoder_is_scheduled_and_its_rotations_share_a_wave():
    wl = decoder_like(layers=2)
    s = Session(wl, device=None)
    so, ns, order, sync = s.schedule()
    assert sorted(order) == list(range(len(wl.ops))) and ns > 2
    wave, _ = B.opara_wave_of(s.dag)
    names = {op.name: op.id for op in wl.ops}
    assert wave[names["L0.rotary_q"]] == wave[names["L0.rotary_k"]]
    assert wave[names["L1.cross_k"]] == 0                      # needs the encoder's states alone
    classes = [d.op_class for d in B.opara_get_demands(s.dag)]
    for op in wl.ops:
        assert classes[op.id] == (B.COMP if op.type in ("gemm", "gated", "attention") else B.MEM), op.name


def test_oracle_carries_second_results():
    b = Builder("two", "f32")
    x = b.ext((3, 8))
    n = b.residual_norm(x, x, alpha=1.0, beta=1.0, weights=False)
    b.residual_norm(n, Second(n), before=False, alpha=2.0, beta=0.0, weights=False)
    wl = b.build(5)
    out = executor.run_dag(wl)
    np.testing.assert_allclose(out[(0, 1)], 2 * wl.ext_inputs[0], rtol=1e-6)
    np.testing.assert_allclose(out[1], 4 * wl.ext_inputs[0], rtol=1e-6)
    assert (1, 1) not in out
