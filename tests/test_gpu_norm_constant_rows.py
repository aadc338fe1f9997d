"""Layer norm of rows whose elements are all alike: nothing is left of them about their mean, whatever it is, and the result is the bias."""
import numpy as np
import pytest

import paper_2505_21594_amd as ee
from tests.device import Dev
from tests.test_gpu_head_operators import Rows, Space, empty

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [1, 3, 7, 100, 384, 1000, 1025, 1536, 5120, 9999, 16383])
def test_rows_of_one_value(dim, kind):
    """Values of 8 and 11 bits: up to 2^16 and 2^13 of them add up to numbers of fp32's 24 bits, and the sum by their number is the value itself.  (30000 and 0.1 have 11 bits in fp16.)"""
    value = np.array([0.0, 1.0, -3.0, 0.10009765625, 1000.0, -640.0, 30000.0, 7.0, 96.0])
    if kind == "fp16" and dim > 1 << 13:
        value = value[[0, 1, 2, 4, 5, 7, 8]]
    x, y = Rows(np.repeat(value[:, None], dim, 1), kind), empty(len(value), dim, "fp32")
    rng = np.random.default_rng(dim)
    gain, bias = (np.float32(rng.standard_normal(dim)) for _ in range(2))
    ee.ee_norm(x.view, y.view, gain=Dev(gain), bias=Dev(bias), eps=1e-5, center=True)
    got = y.result()
    assert (got == bias[None].astype(np.float64)).all(), f"rows {np.unique(np.argwhere(got != bias)[:, 0])}: up to {np.abs(got - bias).max()}"
    dy, dx = Rows(rng.standard_normal(x.values().shape), "fp32"), empty(len(value), dim, "fp32")
    dg = Dev(np.ones(dim, np.float32))
    ee.ee_norm_grad(x.view, dy.view, dx=dx.view, gain=Dev(gain), d_gain=dg, eps=1e-5, center=True, workspace=Space(ee.ee_norm_grad_workspace(x.view)).view)
    assert (dg.numpy() == 0).all()
    u = dy.values() * gain
    want = (u - u.mean(1, keepdims=True)) / np.sqrt(1e-5)
    assert (np.abs(dx.result() - want) <= 100 * 2.0 ** -24 * (np.abs(u) + np.abs(u).mean(1, keepdims=True)) / np.sqrt(1e-5)).all()
