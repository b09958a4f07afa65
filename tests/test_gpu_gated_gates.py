"""Gates of a gated block that are not finite: every form gives what the activation's formula gives for them."""
import math

import pytest
import torch

import decoder_util as D
from paper_2312_10351_amd import binding as B

pytestmark = pytest.mark.gpu

GATES = [math.nan, math.inf, -math.inf]
WANT = {"silu": [math.nan, math.inf, math.nan], "gelu": [math.nan, math.inf, math.nan], "gelu_tanh": [math.nan, math.inf, math.nan],
        "relu": [math.nan, math.inf, 0.0], "sigmoid": [math.nan, 1.0, 0.0]}
SHAPES = [(1, 64, 33), (1, 768, 2048), (3, 1027, 100), (17, 40, 31), (64, 64, 64), (77, 768, 2048), (512, 2048, 1024), (2040, 1032, 4090)]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("act", list(B.ACTIVATION_IDS))
def test_gates_that_are_not_finite(dtype, act):
    for m, k, n in SHAPES:
        x = torch.ones(m, k, dtype=D.TORCH[dtype])
        w = torch.zeros(2 * n, k, dtype=D.TORCH[dtype])
        for i, gate in enumerate(GATES):                       # every column's gate is one product; its value is one
            w[i:n:5, k // 2] = gate
        w[n:, k - 1] = 1.0
        s = D.bind(lambda b, e: b.gated(e[0], m, k, n, act), [x], {0: {"w": w, "b": torch.zeros(2 * n)}}, dtype)
        s.launch()
        got = s.result(0).double().cpu()
        s.close()
        for i, want in enumerate(WANT[act] + [{"sigmoid": 0.5}.get(act, 0.0)] * 2):
            column = got[:, i::5]
            ok = column.isnan() if math.isnan(want) else column == want
            assert ok.all(), (act, (m, k, n), i, want, column[~ok][:3])
