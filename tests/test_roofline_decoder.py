"""The work of a decoder's operators as the roofline counts it."""
import numpy as np
import pytest

from paper_2312_10351_amd.roofline import dag_roofline
from workloads import Builder, decoder_like


def work(add, dtype="f16", **ext):
    b = Builder("work", dtype)
    add(b)
    return dag_roofline(b.build(1))["per_op"]


def test_gated_block_counts_both_products_and_weights():
    (flops, nbytes), = work(lambda b: b.gated(b.ext((3, 40)), 3, 40, 16))
    assert flops == 2 * 2 * 3 * 40 * 16
    assert nbytes == 2 * (3 * 40 + 2 * 40 * 16 + 3 * 16)


@pytest.mark.parametrize("causal, first, lengths", [(None, 0, None), ("start", 0, None), ("start", -2, None), ("start", 4, [7, 2]),
                                                    ("end", 0, None), ("end", 0, [9, 3]), (None, 0, [0, 50])])
def test_attention_counts_what_its_rows_see(causal, first, lengths):
    m, n, batch, heads, kv, w, vw = 5, 9, 2, 6, 3, 8, 4

    def add(b):
        l = None if lengths is None else b.ext((batch,), lengths)
        b.attention(b.ext((batch * m, heads * w)), b.ext((batch * n, kv * w)), b.ext((batch * n, kv * vw)), heads, w, kv, vw, batch=batch,
                    lengths=l, causal=causal, first=first)
    (flops, nbytes), = work(add, "f32")
    pairs = rows = 0
    for b in range(batch):
        length = n if lengths is None else min(n, lengths[b])
        rows += length
        for i in range(m):
            for j in range(length):
                pairs += causal is None or j <= i + (first if causal == "start" else length - m)
    assert flops == 2 * pairs * heads * (w + vw)
    assert nbytes == 4 * (batch * m * heads * (w + vw) + rows * kv * (w + vw)) + (4 * batch if lengths else 0)


def test_row_wise_operators_count_their_bytes():
    def add(b):
        x = b.ext((6, 32))
        b.rotary(x, 2, 16, positions=b.ext((6,), range(6)))
        b.residual_norm(x, x, after=True)
        b.residual_norm(x, before=False, weights=False)
    rotary, two, none = work(add)
    cells = 6 * 32
    assert rotary == (0, 2 * cells * 2 + 6 * 4)
    assert two == (0, 4 * cells * 2 + 2 * 32 * (2 + 4))        # two inputs, the norm and the sum, two rows of weights
    assert none == (0, 2 * cells * 2)


def test_bound_of_a_decoder_holds_its_weights_and_products():
    wl = decoder_like(layers=2, seq=77, hidden=768, heads=12, kv_heads=4, ffn=2048)
    r = dag_roofline(wl)
    gated = [op for op in wl.ops if op.type == "gated"]
    assert r["flops"] > sum(4 * op.params["m"] * op.params["n"] * op.params["k"] for op in gated)
    assert r["bytes"] > sum(w["w"].nbytes for w in wl.weights.values())
    assert np.isfinite(r["t_roof_us"]) and r["t_roof_us"] > 0
