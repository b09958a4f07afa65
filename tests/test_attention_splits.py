"""Into how many workgroups attention shares its keys out, by how they can be loaded."""
import pytest

from decoder_util import describe
from paper_2312_10351_amd import binding as B


def workgroups(dtype, width, m, n, heads, kv):
    op = describe(B.ATTENTION, dtype, 3, m=m, n=n, heads=heads, kv_heads=kv, width=width, alpha=1.0)
    op[1].scratch_bytes = B.opara_scratch_bytes(*op)
    op[1].scratch = 0x900000 if op[1].scratch_bytes else None
    dag = B.opara_build_dag_more([op[0]], [op[1]], [0x1000000 * (i + 1) for i in range(3)])
    d = B.opara_get_demands(dag)[0]
    B.load().opara_dag_destroy(dag)
    return B.opara_kernel_info(d.kernel_id)[0], d.grid_blocks


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("odd, even", [(37, 40), (101, 104), (201, 208)])
@pytest.mark.parametrize("m, n, heads, kv", [(1, 65536, 32, 8), (1, 16384, 32, 8), (1, 16384, 12, 12), (8, 16384, 12, 12)])
def test_keys_that_go_through_registers_are_shared_out_further(dtype, odd, even, m, n, heads, kv):
    """One workgroup walks them 5 to 22 times slower than keys that are loaded directly, so that more of them pay; two
    (of the widest: one) fit on each of 256 compute units."""
    kernel, groups = workgroups(dtype, odd, m, n, heads, kv)
    assert kernel.startswith(f"attend_{dtype}_any")
    assert groups >= workgroups(dtype, even, m, n, heads, kv)[1]
    assert groups >= (160 if odd > 128 else 300)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("width", [37, 101, 201])
def test_short_and_many_rows_are_not_shared_out(dtype, width):
    for m, n, heads, kv in ((1, 60, 4, 4), (4096, 300, 16, 16)):
        assert workgroups(dtype, width, m, n, heads, kv)[1] == -(-m * heads // kv // 16) * kv
