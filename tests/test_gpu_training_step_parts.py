"""A training step of an exit head, call by call: what each one wrote against the 64-bit form of what it was given, with the operators' own tolerances, so that a call that is given
something else than the step means (another row, weight, temperature, an older buffer) is outside of them."""
import numpy as np
import pytest

import paper_2505_21594_amd as ee
from tests import head_ref as ref
from tests.device import HALF_STEP
from tests.test_gpu_head_operators import Step, close

pytestmark = pytest.mark.gpu

B, U = HALF_STEP["bf16"], ref.U


@pytest.mark.parametrize("seed", [3, 8])
def test_every_call_of_a_training_step(seed):
    s = Step(seed)
    s.run()
    v = {k: x.result() for k, x in s.e.items()}
    o = {k: x.numpy().astype(np.float64) for k, x in s.o.items()}
    s.ws.check()
    ids, lps = s.ids.numpy(), s.lps.numpy()
    hb, h, down, up, head = (x.values() for x in (s.hb, s.h, s.down, s.up, s.head))
    lists = ref.score(s.target.values(), None, s.TOP, s.T)
    assert (ids == lists["top_ids"]).all()
    close(lps.astype(np.float64), lists["top_logprobs"], "the target's list")
    t, pre = ref.linear(hb, down, s.b_down, None, ee.ACT_SILU, B, B)
    close(v["t"], t, "down")
    close(v["pre"], pre, "what down keeps for its gradient")
    close(v["a"], ref.linear(v["t"], up, s.b_up, h, ee.ACT_NONE, U, 0)[0], "up and residual")
    close(v["n"], ref.norm(v["a"], s.gain, None, 1e-5, 0, B), "norm")
    close(v["z"], ref.linear(v["n"], head, None, None, ee.ACT_NONE, B, 0)[0], "head")
    weight = np.full(s.ROWS, 1.0 / s.ROWS, np.float32)
    loss, dz = ref.distill(v["z"], ids, lps, s.T, True, weight, B)
    close(o["loss"], loss, "loss")
    close(v["dz"], dz, "the loss's gradient")
    dn, d_head, _ = ref.linear_grad(v["n"], head, v["dz"], None, ee.ACT_NONE, U, U, 0, 0)
    close(v["dn"], dn, "gradient of the norm's result")
    close(v["d_head"], d_head, "head's gradient")
    da, d_gain, _ = ref.norm_grad(v["a"], v["dn"], s.gain, 1e-5, 0, B)
    close(v["da"], da, "gradient of the adapters' result")
    close(o["d_gain"], d_gain, "gains' gradient")
    dt, d_up, d_b_up = ref.linear_grad(v["t"], up, v["da"], None, ee.ACT_NONE, B, U, 0, 0)
    close(v["dt"], dt, "gradient of down's result")
    close(v["d_up"], d_up, "up's gradient")
    close(o["d_b_up"], d_b_up, "up's bias")
    _, d_down, d_b_down = ref.linear_grad(hb, down, v["dt"], v["pre"], ee.ACT_SILU, 0, U, 0, 2.0 ** -24)
    close(v["d_down"], d_down, "down's gradient")
    close(o["d_b_down"], d_b_down, "down's bias")


def test_a_planted_mistake_is_outside_the_tolerances():
    """Made in the 64-bit forms: the weight of another step size, an older result of the norm, the neighbour's row of the residual."""
    s = Step(3)
    s.run()
    v = {k: x.result() for k, x in s.e.items()}
    ids, lps = s.ids.numpy(), s.lps.numpy()
    for wrong, got in ((ref.distill(v["z"], ids, lps, s.T, True, np.full(s.ROWS, 1.02 / s.ROWS, np.float32), B)[1], v["dz"]),
                       (ref.linear(v["t"], s.up.values(), s.b_up, np.roll(s.h.values(), 1, 0), ee.ACT_NONE, U, 0)[0], v["a"]),
                       (ref.linear(np.roll(v["n"], 1, 0), s.head.values(), None, None, ee.ACT_NONE, B, 0)[0], v["z"])):
        with pytest.raises(AssertionError):
            close(got, wrong, "planted")
