"""Lists of a teacher that are out of the ordinary, against 64-bit forms."""
import numpy as np
import pytest

from tests import head_ref as ref
from tests.test_gpu_head_operators import check_distill, close, logits, run_distill

pytestmark = pytest.mark.gpu

SIZES = [(3, 40), (64, 1024), (300, 700), (257, 33000), (3, 140001)]


def log_softmax(z):
    z = z - z.max(1, keepdims=True)
    return z - np.log(np.exp(z).sum(1, keepdims=True))


@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("rows,V", SIZES)
def test_a_token_named_twice_is_the_token_with_both_probabilities(rows, V, rest):
    """Lists with tokens in two and three pieces: loss and gradient of the lists that name each once."""
    rng = np.random.default_rng(rows + V)
    z = logits(rng, rows, V, "fp32")
    once = np.argsort(-z, 1)[:, :5].astype(np.int32)
    p = rng.uniform(0.05, 0.19, (rows, 5))
    split = np.stack([p[:, 0] * 0.25, p[:, 1], p[:, 0] * 0.75, p[:, 2] / 2, p[:, 3], p[:, 4], p[:, 2] / 4, p[:, 2] / 4], 1)
    twice = once[:, [0, 1, 0, 2, 3, 4, 2, 2]]
    lp = np.log(split).astype(np.float32)
    both = np.exp(lp.astype(np.float64))
    lp_once = np.log(np.stack([both[:, 0] + both[:, 2], both[:, 1], both[:, 3] + both[:, 6] + both[:, 7], both[:, 4], both[:, 5]], 1))
    want = ref.distill(z, once, lp_once, 1.0, rest)
    for kw in (dict(), dict(want_grad=False)):
        loss, grad = run_distill(z, "fp32", twice, lp, 1.0, rest, "fp32", **kw)
        close(loss, want[0], "loss")
        if grad is not None:
            close(grad, want[1], "gradient")


def test_a_student_equal_to_a_teacher_of_split_tokens_has_no_loss():
    rng = np.random.default_rng(4)
    z = logits(rng, 40, 500, "fp32")
    ids = np.argsort(-z, 1)[:, [0, 1, 2, 0]].astype(np.int32)
    lp = np.take_along_axis(log_softmax(z), ids, 1)
    lp[:, [0, 3]] -= np.log(2)
    lp = lp.astype(np.float32)
    # each log-probability is rounded to 2^-24 of it: a divergence of its square; and of the sums' share what the differences leave, by 64-bit arithmetic on the same list
    for rest in (True, False):
        merged = np.stack([np.logaddexp(lp[:, 0].astype(np.float64), lp[:, 3].astype(np.float64)), lp[:, 1].astype(np.float64), lp[:, 2].astype(np.float64)], 1)
        want, tol = ref.distill(z, ids[:, :3], merged, 1.0, rest)[0]
        loss, _ = run_distill(z, "fp32", ids, lp, 1.0, rest, "fp32", want_grad=False)
        close(loss, (want, tol), "loss")
        if rest:
            assert (np.abs(want) < 1e-6).all() and (np.abs(loss) < 2e-6).all()


@pytest.mark.parametrize("rows,V", SIZES)
def test_lists_below_every_number_are_divided_by_their_sum(rows, V):
    """rest = 0: log-probabilities from -700 to -3e4, whose exponentials are 0 in 64 bits, and above 0: only their differences count."""
    rng = np.random.default_rng(rows + 2 * V)
    z = logits(rng, rows, V, "fp32")
    ids = np.argsort(-z, 1)[:, :6].astype(np.int32)
    near = np.log(rng.uniform(0.05, 0.3, (rows, 6)))
    lp = (near + rng.choice([-700.0, -746.0, -1000.0, -3e4, 900.0], (rows, 1))).astype(np.float32)
    lp[::4, 3] = -np.inf
    shifted = lp.astype(np.float64) - np.where(np.isfinite(lp), lp.astype(np.float64), -np.inf).max(1, keepdims=True)
    want = ref.distill(z, ids, shifted, 1.0, False)
    for kw in (dict(), dict(want_grad=False)):
        loss, grad = run_distill(z, "fp32", ids, lp, 1.0, False, "fp32", **kw)
        close(loss, want[0], "loss")
        if grad is not None:
            close(grad, want[1], "gradient")


def test_a_label_with_any_log_probability_is_cross_entropy():
    rng = np.random.default_rng(2)
    z = logits(rng, 6, 900, "fp32")
    label = rng.integers(0, 900, (6, 1)).astype(np.int32)
    lp = np.array([0, -3, -740, -800, -1e5, -1e30], np.float32)[:, None]
    loss, grad = run_distill(z, "fp32", label, lp, 1.0, False, "fp32")
    want = ref.distill(z, label, np.zeros((6, 1)), 1.0, False)
    close(loss, want[0], "loss")
    close(grad, want[1], "gradient")
    check_distill(z, "fp32", label, np.zeros((6, 1), np.float32), 1.0, False, "fp32")
