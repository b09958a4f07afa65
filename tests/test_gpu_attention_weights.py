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
    2^-35 of the largest (few rows: cut off to such multiples, with at least one)."""
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
        # fp16 the weight's own, and half a multiple (cut off: one) of 2^-35 per key where that is more than the weight's own
        relative = 4.0 * D.U * gap + 2.0 ** -21 + 2.0 * (n / 64 + 64) * D.U + (2.0 ** -11 if dtype == "f16" else 0.0)
        step = (n - 1) * 2.0 ** (-36 if form.startswith("wide") else -35) if dtype == "f16" else 0.0
        D.within(s.result(0), want, relative * want + step, dtype, f"gap {gap}")
    s.close()


@pytest.mark.parametrize("m, n, heads, kv, width, form", [
    (300, 512, 12, 12, 64, "rows64"), (1, 1500, 2, 2, 128, "rows128"), (50, 300, 1, 1, 256, "rows256"), (1, 1500, 12, 12, 64, "deep64"),
    (1, 512, 32, 8, 128, "deep128"), (9, 70, 2, 2, 37, "any64"), (40, 300, 4, 2, 101, "any128"), (12, 150, 1, 1, 130, "any256")])
def test_few_rows_are_off_by_the_rounding_of_their_result(m, n, heads, kv, width, form):
    """Scores that are exact and values of one size and either sign, so that results are small beside what they are
    summed from: nothing but the result itself may be rounded to fp16."""
    g = torch.Generator().manual_seed(n)
    q, k = torch.zeros(m, heads * width, dtype=torch.float16), torch.zeros(n, kv * width, dtype=torch.float16)
    q[:, ::width] = 1.0
    k[:, ::width] = torch.randint(0, 512, (n, kv), generator=g) / 8.0
    v = (torch.randint(0, 2, (n, kv * width), generator=g) * 2 - 1).to(torch.float16)
    s = D.bind(lambda b, e: b.attention(*e, heads=heads, kv_heads=kv, width=width, alpha=LOG2), [q, k, v], dtype="f16")
    assert B.opara_kernel_info(B.opara_get_demands(s.dag)[0].kernel_id)[0] == f"attend_f16_{form}"
    s.launch()
    torch.cuda.synchronize()
    p = torch.softmax(LOG2 * k[:, ::width].double(), 0).repeat_interleave(heads // kv, 1)            # [n, heads]
    values = v.double().view(n, kv, width).repeat_interleave(heads // kv, 1)
    want = (p[:, :, None] * values).sum(0).view(1, -1).expand(m, -1)
    # values have size one, so the weights' errors count whole: scores up to 64 and their powers, a weight cut off in two
    # parts of eleven bits (2^-10 of 2^-10), the sums, and a multiple of 2^-35 of the largest weight per key
    bound = 4.0 * D.U * 64 * LOG2 + 2.0 ** -21 + 2.0 ** -20 + 2.0 * (n / 64 + 64) * D.U + n * 2.0 ** -35
    D.within(s.result(0), want, torch.full_like(want, bound), "f16")
    s.close()


@pytest.mark.parametrize("m, n, width", [(1, 1500, 64), (40, 300, 33), (3, 200, 256), (200, 700, 128)])
def test_a_factor_of_zero_counts_keys_alike_whatever_their_scores(m, n, width):
    """Products of queries and keys near fp32's largest numbers times zero are zero."""
    g = torch.Generator().manual_seed(n)
    q = torch.full((m, width), 1e18)
    k = 1e18 * torch.rand(n, width, generator=g)
    v = torch.randn(n, width, generator=g)
    s = D.bind(lambda b, e: b.attention(*e, heads=1, width=width, alpha=0.0), [q, k, v], dtype="f32")
    s.launch()
    torch.cuda.synchronize()
    want = v.double().mean(0, keepdim=True).expand(m, -1)
    D.within(s.result(0), want, (v.abs().double().mean(0) * (n / 64 + 64) * 3 * D.U).expand(m, -1), "f32")
    s.close()


@pytest.mark.parametrize("width", [64, 37, 128, 200])
@pytest.mark.parametrize("m, n", [(1, 1), (1, 3), (40, 2)])
def test_large_values_stay_in_fp32s_range(m, n, width):
    """Results are sums of weights of at most one times values until they are divided by the weights' sum."""
    g = torch.Generator().manual_seed(n)
    q, k = torch.randn(m, width, generator=g), torch.randn(n, width, generator=g)
    v = 1e38 * (torch.rand(n, width, generator=g) * 2 - 1)
    s = D.bind(lambda b, e: b.attention(*e, heads=1, width=width), [q, k, v], dtype="f32")
    s.launch()
    torch.cuda.synchronize()
    D.within(s.result(0), *D.attention(q, k, v, "f32", width=width), "f32")
    s.close()
