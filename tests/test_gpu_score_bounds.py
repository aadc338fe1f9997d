"""ee_score_tokens where the bound of a row's candidates says little: vocabularies whose last wave has a chunk or two, rows whose logits are near each other beside what they are offset by."""
import numpy as np
import pytest

from tests.device import decode, encode
from tests.test_gpu_head_operators import check_score, logits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,V", [(40, 1), (40, 63), (40, 257), (40, 511), (40, 513), (40, 520), (40, 769), (600, 1040), (40, 1100), (40, 1544), (9, 4104), (300, 8200), (3, 33000)])
def test_vocabularies_that_end_in_a_wave(rows, V, kind):
    rng = np.random.default_rng(rows + V)
    z = logits(rng, rows, V, kind, special=True)
    for top in (1, 33, 64):
        check_score(z, kind, rng.integers(0, V, rows), top, 1.0)
    z[:] = np.sort(z, 1)                                        # the largest ones in the last wave
    check_score(z, kind, rng.integers(0, V, rows), 64, 1.0)


@pytest.mark.parametrize("rows,V", [(9, 700), (300, 5000), (5, 32000), (3, 100003)])
def test_rows_that_are_near_each_other_beside_their_offset(rows, V):
    rng = np.random.default_rng(V)
    for offset in (1e3, -1e3, 1e5):
        z = decode(encode((offset + 2 * rng.standard_normal((rows, V))).astype(np.float32), "fp32"))
        for top in (1, 20, 64):
            check_score(z, "fp32", rng.integers(0, V, rows), top, 1.0)
