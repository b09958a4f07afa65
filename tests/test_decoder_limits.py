"""Sizes that the kernels of a decoder's operators cannot count or launch are refused when the DAG is built."""
import pytest

from decoder_util import build, describe
from paper_2312_10351_amd import binding as B

INT = 2 ** 31 - 1
NORM = dict(m=4, n=8, eps=1e-5, alpha=1.0, beta=1.0, flags=B.FLAG_NORM_AFTER | B.FLAG_NORM_BEFORE)


def refused(kind, n_inputs, dtype="f16", **fields):
    with pytest.raises(B.OparaError) as e:
        build(describe(kind, dtype, n_inputs, **fields))
    return e.value.status == B.EUNSUPPORTED


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("n", [8, 7, 512, 4096])
def test_rows_that_a_norm_counts(dtype, n):
    """The counter of a workgroup passes the last row by up to 4096 before it stops."""
    build(describe(B.RESIDUAL_NORM, dtype, 2, **{**NORM, "m": INT - 4096, "n": n}))
    for m in (INT - 4095, INT):
        assert refused(B.RESIDUAL_NORM, 2, dtype, **{**NORM, "m": m, "n": n})


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_columns_that_a_norm_counts(dtype):
    """The second norm's weights follow the first's: column n + j is a 32-bit number."""
    build(describe(B.RESIDUAL_NORM, dtype, 2, **{**NORM, "n": 2 ** 30}))
    for n in (2 ** 30 + 1, 2 ** 30 + 8, INT):
        assert refused(B.RESIDUAL_NORM, 2, dtype, **{**NORM, "n": n})


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("m", [1, 3])
def test_row_lengths_that_a_gated_block_counts(dtype, m):
    """One row: a wavefront looks two of its vectors (2 * 512 elements in fp16) past where it is."""
    shape = dict(m=m, n=16, weight=0x2000)
    build(describe(B.GATED, dtype, 1, k=INT - 2048, **shape))
    for k in (INT - 2047, INT - 1000, INT - 64, INT):
        assert refused(B.GATED, 1, dtype, k=k, **shape)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_threads_that_a_launch_counts(dtype):
    """Workgroups times threads along an axis stay below 2^32."""
    attend = dict(n=1, heads=1, kv_heads=1, width=1, alpha=1.0)
    build(describe(B.ATTENTION, dtype, 3, m=2 ** 27, **attend))
    assert refused(B.ATTENTION, 3, dtype, m=2 ** 28, **attend)           # sixteen rows, 256 threads
    gated = dict(k=1, weight=0x2000)
    build(describe(B.GATED, dtype, 1, m=2 ** 29, n=1, **gated))
    assert refused(B.GATED, 1, dtype, m=2 ** 30, n=1, **gated)           # 64 rows
    build(describe(B.GATED, dtype, 1, m=1, n=2 ** 25, **gated))
    assert refused(B.GATED, 1, dtype, m=1, n=2 ** 26, **gated)           # four columns
