"""Rows of logits masked with the type's lowest finite value, whose products with log2(e) / T pass fp32, and other logits beyond that, against 64-bit forms."""
import numpy as np
import pytest

from tests import head_ref as ref
from tests.device import decode, encode
from tests.test_gpu_head_operators import close, logits, run_score

pytestmark = pytest.mark.gpu

LOWEST = {"bf16": -3.3895313892515355e38, "fp16": -65504.0, "fp32": -3.4028234663852886e38}


def masked(rng, rows, V, kind):
    z, low = logits(rng, rows, V, kind), LOWEST[kind]
    at = np.arange(V)
    for r in range(rows):
        z[r] = [lambda x: np.where(rng.random(V) < 0.9, low, x),                 # a tenth of the tokens is allowed
                lambda x: np.where((at - V // 2) // 3 == 0, x, low),             # three are: whole threads and waves have none
                lambda x: np.full(V, low),                                       # none: all are alike
                lambda x: np.where(at == V - 1, 1.5, low),
                lambda x: np.where(at < V // 2, low, x),
                lambda x: np.where(at % 2 == 0, low, -np.inf),                   # none, and some of no weight at all
                lambda x: np.where(at == V // 3, -low, x),                       # one far above the others
                lambda x: np.where(at == 0, np.nan if V > 1 else low, low)][r % 8](z[r])
    return decode(encode(z.astype(np.float32), kind))


def in_fp32(want):
    """The value as fp32 holds it: what is beyond its numbers is infinite."""
    value, tol = want
    with np.errstate(over="ignore"):
        return np.where(np.abs(value) > 3.4028235677973366e38, np.float32(value).astype(np.float64), value), tol


@pytest.mark.parametrize("T", [1.0, 0.7, 2.5, 1e-8])
@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,V,top", [(8, 1, 1), (8, 700, 8), (16, 5000, 20), (8, 40000, 64), (8, 100003, 5), (264, 1500, 4), (520, 9000, 64)])
def test_score_of_rows_masked_with_the_lowest_value(rows, V, top, kind, T):
    rng = np.random.default_rng(rows + V)
    z = masked(rng, rows, V, kind)
    tokens = np.where(np.arange(rows) % 3 == 0, V // 2, np.argmax(np.nan_to_num(z, nan=-np.inf), 1))
    lp, h, ids, tl = run_score(z, kind, tokens, top, T)
    want = ref.score(z, tokens, top, T)
    assert (ids == want["top_ids"]).all(), f"lists differ in rows {np.unique(np.argwhere(ids != want['top_ids'])[:, 0])[:8]}"
    close(lp.astype(np.float64), in_fp32(want["logprob"]), "logprob")
    close(h.astype(np.float64), in_fp32(want["entropy"]), "entropy")
    close(tl.astype(np.float64), in_fp32(want["top_logprobs"]), "top_logprobs")
