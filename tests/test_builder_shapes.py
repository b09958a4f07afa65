"""Shapes that do not fit together are refused where a decoder's operators are added, not read as something else."""
import pytest

from workloads import Builder, Second, decoder_like


@pytest.fixture
def b():
    return Builder("shapes", "f16")


def test_rotary(b):
    x = b.ext((6, 128))
    b.rotary(x, 2, 64)
    b.rotary(x, 2, 64, positions=b.ext((6,)))
    for heads, width in ((1, 64), (2, 32), (4, 64)):
        with pytest.raises(ValueError):
            b.rotary(x, heads, width)
    b.rotary(b.ext((6, 2, 64)), 2, 64, positions=b.ext((6, 1)))      # heads as an axis
    for positions in (b.ext((5,)), b.ext((7,)), b.ext((6, 2)), b.gemm(x, 6, 128, 1)):
        with pytest.raises(ValueError):
            b.rotary(x, 2, 64, positions=positions)


def test_residual_norm(b):
    x = b.ext((6, 32))
    n = b.residual_norm(x, x)
    b.residual_norm(x, Second(n), gate=b.ext((3, 32)))
    for r in (b.ext((5, 32)), b.ext((6, 33)), b.ext((6, 64))):
        with pytest.raises(ValueError):
            b.residual_norm(x, r)
    for g in (b.ext((4, 32)), b.ext((1, 16)), b.ext((12, 32))):
        with pytest.raises(ValueError):
            b.residual_norm(x, x, gate=g)


def test_gated(b):
    x = b.ext((6, 32))
    b.gated(x, 6, 32, 8)
    b.gated(x, 4, 32, 8)                                       # the first rows
    b.gated(x, 3, 64, 8)                                       # the same elements in another shape
    b.gated(b.ext((32, 2, 3)), 1, 192, 8)
    for m, k in ((7, 32), (6, 33), (6, 16), (4, 40)):
        with pytest.raises(ValueError):
            b.gated(x, m, k, 8)


def test_attention(b):
    q, k, v = b.ext((6, 64)), b.ext((10, 32)), b.ext((10, 16))
    ok = dict(heads=4, width=16, kv_heads=2, v_width=8)
    b.attention(q, k, v, **ok)
    b.attention(q, k, v, **ok, batch=2, lengths=b.ext((2,)))
    b.attention(b.ext((6, 4, 16)), b.ext((10, 2, 16)), b.ext((10, 2, 8)), **ok)
    with pytest.raises(ValueError):                            # sequences as an axis of their own
        b.attention(b.ext((2, 3, 64)), b.ext((2, 5, 32)), b.ext((2, 5, 16)), **ok, batch=2)
    for bad in (dict(batch=4), dict(batch=5), dict(batch=0), dict(heads=2), dict(width=8), dict(v_width=16), dict(kv_heads=1)):
        with pytest.raises(ValueError):
            b.attention(q, k, v, **{**ok, **bad})
    with pytest.raises(ValueError):                            # as many values as keys
        b.attention(q, k, b.ext((12, 16)), **ok)
    for lengths in (b.ext((1,)), b.ext((3,)), b.gemm(q, 2, 64, 1)):
        with pytest.raises(ValueError):
            b.attention(q, k, v, **ok, batch=2, lengths=lengths)


@pytest.mark.parametrize("kw", [dict(), dict(seq=1, states=300, past=40), dict(hidden=384, heads=6, kv_heads=2, ffn=520)])
def test_the_decoder_fits_together(kw):
    decoder_like(**kw)
