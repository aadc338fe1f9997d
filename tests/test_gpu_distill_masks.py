"""ee_distill with rows of logits masked with the type's lowest finite value, and others whose products with log2(e) / T pass fp32, against the 64-bit form."""
import numpy as np
import pytest

from tests import head_ref as ref
from tests.device import HALF_STEP
from tests.test_gpu_head_masks import in_fp32, masked
from tests.test_gpu_head_operators import SUBNORMAL, close, run_distill

pytestmark = pytest.mark.gpu


def spread(z, named, T):
    """The softmax over the tokens that the list does not name, relative to the largest of them: beside logits of 1e38 the logarithm of their number is lost in a difference of log q."""
    out = np.zeros(z.shape)
    for x, n, o in zip(z, named, out):
        if not np.isnan(x).any() and np.isfinite(x[~n]).any():
            w = np.exp((x[~n] - x[~n].max()) / float(np.float32(T)))
            o[~n] = w / w.sum()
    return out


@pytest.mark.parametrize("T", [1.0, 0.7, 2.5, 1e-8])
@pytest.mark.parametrize("kind,out", [("bf16", "bf16"), ("fp32", "fp32"), ("fp16", "fp32")])
@pytest.mark.parametrize("rows,V", [(8, 1), (16, 700), (16, 5000), (8, 40000), (8, 140001), (264, 1500), (264, 33000), (260, 9000)])
def test_distillation_of_rows_masked_with_the_lowest_value(rows, V, kind, out, T):
    """The teacher names tokens that are allowed, and in some rows one that is masked; in the others nothing but masked tokens are left."""
    rng = np.random.default_rng(rows * 3 + V)
    z, top = masked(rng, rows, V, kind), min(V, 5)
    ids = np.argsort(-np.nan_to_num(z, nan=-np.inf), 1, kind="stable")[:, :top].astype(np.int32)
    for r in range(0, rows, 3):
        ids[r, -1] = ids[r, -1] if V // 5 in ids[r] else V // 5
    p = rng.uniform(0.05, 0.15, (rows, top))
    lp = np.log(p).astype(np.float32)
    weight = np.where(np.arange(rows) % 5 == 4, 0, rng.standard_normal(rows)).astype(np.float32)
    for rest in (True, False):
        (want_loss, loss_tol), (want, tol) = ref.distill(z, ids, lp, T, rest, weight, HALF_STEP[out], SUBNORMAL[out])
        # masked tokens are nothing beside the others, or all alike: no exponent of theirs is rounded, and of what is spread over all of them each has one part
        far, named = ~(np.abs(z) < 1e30), np.zeros(z.shape, bool)
        np.put_along_axis(named, ids, True, 1)
        if rest:
            m = np.where(np.isnan(z), -np.inf, z).max(1, keepdims=True)
            e = np.exp((z - m) / float(np.float32(T)))
            pi = 1 - np.array([np.exp(l[np.unique(i, return_index=True)[1]].astype(np.float64)).sum() for i, l in zip(ids, lp)])[:, None]
            others = (e / e.sum(1, keepdims=True) - np.where(named.all(1, keepdims=True), 0, pi) * spread(z, named, T)) * (weight / np.float64(np.float32(T)))[:, None]
            want = np.where(named | np.isnan(z).any(1, keepdims=True), want, others)
        part = np.where(named, 2.0, 2.0 / np.maximum((far & ~named & np.isfinite(z)).sum(1, keepdims=True), 1))
        parts = np.where(far, np.abs(weight / T)[:, None] * part * (2 * ref.SUM + 6 * ref.U) + HALF_STEP[out] * np.abs(want) + SUBNORMAL[out] + 1e-37, tol)
        for kw in (dict(), dict(want_grad=False), dict(in_place=True)) if out == kind else (dict(), dict(want_grad=False)):
            # (in place the rows' surroundings are compared as values: without the rows that hold NaN)
            at = ~np.isnan(z).any(1) if kw.get("in_place") and kind != "bf16" else np.ones(rows, bool)
            loss, grad = run_distill(z[at], kind, ids[at], lp[at], T, rest, out, weight[at], **kw)
            close(loss, in_fp32((want_loss[at], loss_tol[at])), f"loss, rest {rest}")
            if grad is not None:
                close(grad, (want[at], np.minimum(tol, parts)[at]), f"gradient, rest {rest}")
