"""Host arrays of a workload that an operator would read past their end, or as another type, are refused."""
import numpy as np
import pytest
import torch

from paper_2312_10351_amd.runtime import Session
from workloads import Builder


def workload(dtype="f16"):
    """A convolution and pooling, and the blocks of a decoder."""
    b = Builder("arrays", dtype)
    b.conv(b.ext((8, 6, 6)), 16, 3, 1, 1)
    x = b.ext((6, 32))
    p = b.rotary(x, 2, 16, positions=b.ext((6,), range(6)))
    a = b.attention(p, p, p, 2, 16, lengths=b.ext((1,), [5]))
    n = b.residual_norm(a, x)
    b.gemm(b.gated(n, 6, 32, 24), 6, 24, 8)
    return b.build(1, random_bias=True)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_arrays_have_the_size_and_type_that_is_read(dtype):
    wl = workload(dtype)
    Session(wl, device=None)
    for v, w in wl.weights.items():                            # biases are converted
        w["b"] = w["b"].astype(np.float64)
    Session(wl, device=None)
    other = np.float32 if dtype == "f16" else np.float16
    for slot, values in enumerate(list(wl.ext_inputs)):
        for bad in (values.reshape(-1)[:-1], values.astype(other), values.astype(np.float64)):
            wl.ext_inputs[slot] = bad
            with pytest.raises(ValueError):
                Session(wl, device=None)
        wl.ext_inputs[slot] = values
    for v, w in wl.weights.items():
        for key in ("w", "b"):
            values = w[key]
            for bad in (values.reshape(-1)[:-1],) + ((values.astype(other),) if key == "w" else ()):
                w[key] = bad
                with pytest.raises(ValueError):
                    Session(wl, device=None)
            w[key] = values
    Session(wl, device=None)


def test_host_arrays_of_three_axes_are_images():
    """They are stored with their channels last, so that rows read from them would be others."""
    b = Builder("axes", "f16")
    b.rotary(b.ext((6, 2, 16)), 2, 16)
    with pytest.raises(ValueError):
        Session(b.build(1), device=None)
    wl = b.build(1)
    wl.ext_inputs[0] = torch.from_numpy(wl.ext_inputs[0])      # tensors are used as they are
    Session(wl, device=None)
    b = Builder("pixel", "f16")
    b.gated(b.ext((32, 1, 1)), 1, 32, 8)                       # one pixel: the same in either order
    Session(b.build(1), device=None)
