"""What fp16 attention keeps of small softmax weights: one key far above all others, whose value row is zero, so that
the result is the weight of the long tail."""
import math

import pytest
import torch

import decoder_util as D
from paper_2312_10351_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LOG2 = math.log(2.0)

SHAPES = [                                                       # m, n, heads, kv heads, width, form
    (1, 65536, 32, 32, 64, "rows64"), (1, 65536, 8, 2, 128, "rows128"), (3, 30000, 1, 1, 256, "rows256"), (1, 1500, 12, 12, 64, "deep64"),
    (2, 20001, 1, 1, 37, "any64"), (1, 5000, 1, 1, 101, "any128"), (700, 16384, 8, 8, 128, "wide128"), (1000, 20000, 8, 4, 64, "wide64")]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("m, n, heads, kv, width, form", SHAPES)
def test_a_long_tail_keeps_its_weight(dtype, m, n, heads, kv, width, form):
    """Weights 2^-gap beside one of 1: in fp16 rounded relative to themselves down to 2^-25, below that to multiples of
    2^-35 of the largest."""
    at = n * 2 // 3
    q, k, v = (torch.zeros(r, h * width, dtype=D.TORCH[dtype]) for r, h in ((m, heads), (n, kv), (n, kv)))
    q[:, ::width] = 1.0
    v[:] = 1.0
    v[at] = 0.0
    s = D.bind(lambda b, e: b.attention(*e, heads=heads, kv_heads=kv, width=width, alpha=LOG2), [q, k, v], dtype=dtype)
    if dtype == "f16":
        assert B.opara_kernel_info(B.opara_get_demands(s.dag)[0].kernel_id)[0] == f"attend_f16_{form}"
    for gap in (12.375, 17.375, 23.625, 24.5, 25.125, 27.875, 33.0):
        s.ext_dev[1].zero_()
        s.ext_dev[1][at, ::width] = gap
        s.launch()
        torch.cuda.synchronize()
        tail = (n - 1) * 2.0 ** -gap
        want = torch.full((m, heads * width), tail / (1.0 + tail), dtype=torch.float64)
        # roundings: the score's and its power's (gap * 3 * 2^-24 * ln 2 twice, 2^-21), n / 64 + 64 of each fp32 sum, in
        # fp16 the weight's own, and half a multiple of 2^-35 per key where that is more than the weight's own
        relative = 4.0 * D.U * gap + 2.0 ** -21 + 2.0 * (n / 64 + 64) * D.U + (2.0 ** -11 if dtype == "f16" else 0.0)
        step = (n - 1) * 2.0 ** -36 if dtype == "f16" else 0.0
        D.within(s.result(0), want, relative * want + step, dtype, f"gap {gap}")
    s.close()
