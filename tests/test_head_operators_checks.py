"""Refusals of the operators around the LM head (argument checks run before anything touches a GPU), their reference forms, and mistakes planted in these."""
import ctypes

import numpy as np
import pytest

import paper_2505_21594_amd as ee
from paper_2505_21594_amd import binding
from paper_2505_21594_amd.binding import DistillArgsC, LinearArgsC, LinearGradArgsC, NormArgsC, NormGradArgsC, ScoreArgsC
from tests import head_ref as ref
from tests.device import Dev

P = 1 << 20   # an address that nothing reads
Q = 2 << 20


def filled(c, values, **kw):
    a = c(*values)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def score_args(**kw):
    return filled(ScoreArgsC, (0, ee.FP32, 6, 100, 4, 1.0, P, 100, P, P, P, P, P), **kw)


def distill_args(**kw):
    return filled(DistillArgsC, (0, ee.FP32, ee.BF16, 6, 100, 4, 1, 1.0, P, 100, P, P, P, P, Q, 100), **kw)


def norm_args(**kw):
    return filled(NormArgsC, (0, ee.BF16, ee.FP32, 5, 64, 0, 1e-5, 0, P, P, P, Q, 64, 64), **kw)


def norm_grad_args(**kw):
    return filled(NormGradArgsC, (0, ee.BF16, ee.FP32, ee.BF16, 5, 64, 1, 1e-5, P, 3 * P, P, Q, P, P, 64, 64, 64), **kw)


def linear_args(**kw):
    return filled(LinearArgsC, (0, ee.BF16, ee.FP32, ee.FP32, ee.ACT_SILU, 5, 64, 32, P, 3 * P, P, 4 * P, Q, 5 * P, 64, 64, 32, 32, 32), **kw)


def linear_grad_args(**kw):
    return filled(LinearGradArgsC, (0, ee.BF16, ee.FP32, ee.FP32, ee.ACT_SILU, 5, 64, 32, P, 3 * P, 4 * P, 5 * P, Q, 6 * P, P, 64, 64, 32, 32, 64, 64), **kw)


def refused(rc, word):
    assert rc == ee.EE_EINVAL
    assert word in ee.load_library().ee_last_error().decode()


BIG = 1 << 40


@pytest.mark.parametrize("kw,word", [(dict(device=-1), "device"), (dict(dtype=3), "type"), (dict(vocab=0), "vocab"), (dict(vocab=(1 << 24) + 1), "vocab"), (dict(n_rows=-1), "n_rows"),
                                     (dict(n_rows=(1 << 20) + 1), "n_rows"), (dict(top=65), "top"), (dict(top=-1), "top"), (dict(temperature=0.0), "temperature"),
                                     (dict(temperature=float("nan")), "temperature"), (dict(temperature=float("inf")), "temperature"), (dict(temperature=1e-40), "temperature"),
                                     (dict(logits=0), "null"), (dict(tokens=0), "tokens"), (dict(top_ids=0), "null"), (dict(top_logprobs=0), "null"), (dict(logits_stride=99), "stride"),
                                     (dict(logits_stride=BIG), "stride"), (dict(logits=P + 2), "aligned"), (dict(entropy=P + 2), "4-byte")])
def test_score_is_checked(kw, word):
    refused(ee.load_library().ee_score_tokens(ctypes.byref(score_args(**kw)), P, 1 << 30, None), word)


@pytest.mark.parametrize("kw,word", [(dict(device=-1), "device"), (dict(dtype=-1), "type"), (dict(grad_dtype=3), "type"), (dict(vocab=0), "vocab"), (dict(n_rows=-1), "n_rows"),
                                     (dict(top=0), "top"), (dict(top=65), "top"), (dict(rest=2), "rest"), (dict(temperature=-1.0), "temperature"), (dict(logits=0), "null"),
                                     (dict(ids=0), "null"), (dict(logprobs=0), "null"), (dict(logits_stride=99), "stride"), (dict(d_logits_stride=99), "stride"),
                                     (dict(d_logits=P), "same type"), (dict(d_logits=Q + 1), "aligned"), (dict(loss=P + 1), "4-byte")])
def test_distill_is_checked(kw, word):
    refused(ee.load_library().ee_distill(ctypes.byref(distill_args(**kw)), P, 1 << 30, None), word)


NORM = [(dict(device=-1), "device"), (dict(dtype=3), "type"), (dict(n_rows=-1), "n_rows"), (dict(n_rows=(1 << 21) + 1), "n_rows"), (dict(dim=0), "dim"), (dict(dim=16385), "dim"),
        (dict(center=2), "center"), (dict(eps=-1e-5), "eps"), (dict(eps=float("nan")), "eps"), (dict(x=0), "null"), (dict(x_stride=63), "stride"), (dict(x=P + 1), "aligned"),
        (dict(gain=P + 2), "4-byte")]


@pytest.mark.parametrize("kw,word", NORM + [(dict(out_dtype=-1), "type"), (dict(y=0), "null"), (dict(y_stride=BIG), "stride"), (dict(y=P), "same type"), (dict(bias=P + 2), "4-byte")])
def test_norm_is_checked(kw, word):
    refused(ee.load_library().ee_norm(ctypes.byref(norm_args(**kw)), None), word)


@pytest.mark.parametrize("kw,word", NORM + [(dict(dy_dtype=5), "type"), (dict(dx_dtype=5), "type"), (dict(dy=0), "null"), (dict(dx=P, dx_stride=80), "same type"), (dict(dx=3 * P), "same type"),
                                            (dict(dy_stride=2), "stride"), (dict(d_gain=P + 2), "4-byte")])
def test_norm_grad_is_checked(kw, word):
    refused(ee.load_library().ee_norm_grad(ctypes.byref(norm_grad_args(**kw)), P, 1 << 30, None), word)


LINEAR = [(dict(device=-1), "device"), (dict(dtype=ee.FP32), "bf16 or fp16"), (dict(act=3), "activation"), (dict(n_rows=-1), "n_rows"), (dict(n_in=0), "n_in"), (dict(n_out=(1 << 22) + 1), "n_out"),
          (dict(x=P + 8), "16-byte"), (dict(weight=P + 2), "16-byte"), (dict(x_stride=60), "alignment"), (dict(weight_stride=56), "smaller"), (dict(pre_stride=24), "smaller"), (dict(pre=5 * P + 4), "16-byte")]


@pytest.mark.parametrize("kw,word", LINEAR + [(dict(out_dtype=4), "type"), (dict(residual_dtype=4), "type"), (dict(x=0), "null"), (dict(weight=0), "null"), (dict(y=0), "null"), (dict(y_stride=34), "alignment"),
                                              (dict(residual_stride=28), "smaller"), (dict(y=P), "their own"), (dict(pre=Q), "their own"), (dict(pre=3 * P), "their own"), (dict(pre=4 * P), "their own"), (dict(residual=Q, residual_stride=36), "residual"), (dict(bias=P + 2), "4-byte")])
def test_linear_is_checked(kw, word):
    refused(ee.load_library().ee_linear(ctypes.byref(linear_args(**kw)), P, 1 << 30, None), word)


@pytest.mark.parametrize("kw,word", LINEAR + [(dict(dx_dtype=4), "type"), (dict(dw_dtype=-1), "type"), (dict(dy=0), "dy"), (dict(pre=0), "pre"), (dict(weight=0), "weight"), (dict(x=0), "needs x"),
                                              (dict(dx=P), "their own"), (dict(d_weight=Q), "their own"), (dict(dw_stride=60), "smaller"), (dict(dx_stride=66), "alignment"), (dict(d_bias=P + 2), "4-byte")])
def test_linear_grad_is_checked(kw, word):
    refused(ee.load_library().ee_linear_grad(ctypes.byref(linear_grad_args(**kw)), P, 1 << 30, None), word)


def test_workspaces_are_checked():
    lib, n = ee.load_library(), ctypes.c_size_t()
    for name, call, args in (("score", lib.ee_score_tokens, score_args(vocab=100003, logits_stride=100003)),
                             ("distill", lib.ee_distill, distill_args(vocab=100003, logits_stride=100003, d_logits_stride=100003)),
                             ("norm_grad", lib.ee_norm_grad, norm_grad_args()), ("linear_grad", lib.ee_linear_grad, linear_grad_args())):
        size = getattr(lib, f"ee_{name}_workspace")
        assert size(ctypes.byref(args), ctypes.byref(n)) == ee.EE_OK and n.value > 0, name
        refused(call(ctypes.byref(args), P, n.value - 1, None), "workspace")
        refused(call(ctypes.byref(args), P + 128, n.value, None), "workspace")
        refused(call(ctypes.byref(args), None, n.value, None), "workspace")
        assert size(ctypes.byref(args), None) == ee.EE_EINVAL
        refused(size(None, ctypes.byref(n)), "null")
    assert lib.ee_linear_workspace(ctypes.byref(linear_args()), ctypes.byref(n)) == ee.EE_OK
    refused(lib.ee_linear_workspace(ctypes.byref(linear_args(dtype=ee.FP32)), ctypes.byref(n)), "bf16")


def test_workspaces_of_no_rows():
    lib, n = ee.load_library(), ctypes.c_size_t()
    for name, args in (("score", score_args(n_rows=0)), ("distill", distill_args(n_rows=0)), ("norm_grad", norm_grad_args(n_rows=0)), ("linear", linear_args(n_rows=0)),
                       ("linear_grad", linear_grad_args(n_rows=0))):
        assert getattr(lib, f"ee_{name}_workspace")(ctypes.byref(args), ctypes.byref(n)) == ee.EE_OK


def test_nothing_to_do_is_fine():
    lib = ee.load_library()
    assert lib.ee_score_tokens(ctypes.byref(score_args(n_rows=0)), None, 0, None) == ee.EE_OK
    assert lib.ee_distill(ctypes.byref(distill_args(n_rows=0)), None, 0, None) == ee.EE_OK
    assert lib.ee_distill(ctypes.byref(distill_args(loss=0, d_logits=0)), None, 0, None) == ee.EE_OK
    assert lib.ee_norm(ctypes.byref(norm_args(n_rows=0)), None) == ee.EE_OK
    assert lib.ee_norm_grad(ctypes.byref(norm_grad_args(dx=0, d_gain=0, d_bias=0)), None, 0, None) == ee.EE_OK
    assert lib.ee_linear(ctypes.byref(linear_args(n_rows=0)), None, 0, None) == ee.EE_OK
    assert lib.ee_linear_grad(ctypes.byref(linear_grad_args(dx=0, d_weight=0, d_bias=0)), None, 0, None) == ee.EE_OK
    for call in (lib.ee_score_tokens, lib.ee_distill, lib.ee_norm_grad, lib.ee_linear, lib.ee_linear_grad):
        refused(call(None, None, 0, None), "null")
    refused(lib.ee_norm(None, None), "null")


def test_struct_layouts_match_header():
    sizes = {ScoreArgsC: 6 * 4 + 7 * 8, DistillArgsC: 8 * 4 + 8 * 8, NormArgsC: 8 * 4 + 6 * 8, NormGradArgsC: 8 * 4 + 9 * 8, LinearArgsC: 8 * 4 + 11 * 8, LinearGradArgsC: 8 * 4 + 13 * 8}
    packs = (binding._SCORE_PACK, binding._DISTILL_PACK, binding._NORM_PACK, binding._NORM_GRAD_PACK, binding._LINEAR_PACK, binding._LINEAR_GRAD_PACK)
    for (c, size), fmt in zip(sizes.items(), packs):
        assert ctypes.sizeof(c) == size
        kinds = [f[1] for f in c._fields_]
        values = [0.5 + i if k is ctypes.c_float else i + 1 for i, k in enumerate(kinds)]
        got = c.from_buffer_copy(fmt(*values))
        assert [getattr(got, f[0]) for f in c._fields_] == values


def test_binding_checks_shapes():
    z, w = Dev(np.zeros((4, 32), np.float32)), Dev(np.zeros((8, 32), np.uint16))
    x, ints, fl = Dev(np.zeros((4, 32), np.uint16)), Dev(np.zeros(4, np.int32)), Dev(np.zeros(4, np.float32))
    ids, lps = Dev(np.zeros((4, 3), np.int32)), Dev(np.zeros((4, 3), np.float32))
    y = Dev(np.zeros((4, 8), np.uint16))
    for call in (lambda: ee.ee_score_tokens(z, fl, logprob=fl), lambda: ee.ee_score_tokens(z, ints, logprob=Dev(np.zeros(3, np.float32))), lambda: ee.ee_score_tokens(ints, ints),
                 lambda: ee.ee_score_tokens(z, top_ids=ids, top_logprobs=Dev(np.zeros((4, 2), np.float32))), lambda: ee.ee_score_tokens(z.view((4, 16), (32, 2))),
                 lambda: ee.ee_distill(z, ids, ids), lambda: ee.ee_distill(z, Dev(np.zeros((3, 3), np.int32)), lps), lambda: ee.ee_distill(z, ids, lps, d_logits=y),
                 lambda: ee.ee_norm(z, y), lambda: ee.ee_norm(z, z, gain=fl), lambda: ee.ee_norm_grad(z, y), lambda: ee.ee_norm_grad(z, z, d_gain=ints),
                 lambda: ee.ee_linear(x, Dev(np.zeros((8, 16), np.uint16)), y), lambda: ee.ee_linear(x, w, z), lambda: ee.ee_linear(x, Dev(np.zeros((8, 32), np.float16)), y),
                 lambda: ee.ee_linear(x, w, y, pre=Dev(np.zeros((4, 8), np.float32))), lambda: ee.ee_linear_grad(x, w, z), lambda: ee.ee_linear_grad(x, w, y, dx=y),
                 lambda: ee.ee_linear_grad(x, w, y, d_weight=x), lambda: ee.ee_linear_grad(x, w, y, d_bias=fl)):
        with pytest.raises(ValueError):
            call()


# ---------------------------------------------------------------- the reference forms

def test_gradients_of_the_reference_agree_with_differences():
    rng = np.random.default_rng(5)
    z = rng.standard_normal((3, 20)) * 2
    ids = np.array([[3, 5, 5, 19], [0, -1, 7, 8], [4, 4, 4, 30]])
    lp = np.log(np.array([[0.3, 0.2, 0.1, 0.1], [0.5, 0.2, 0.2, 0.05], [0.2, 0.3, 0.1, 0.4]]))
    for rest in (True, False):
        for T in (1.0, 1.7):
            (_, _), (g, _) = ref.distill(z, ids, lp, T, rest)
            h = 1e-6
            for i in range(20):
                up, down = z.copy(), z.copy()
                up[:, i] += h
                down[:, i] -= h
                d = (ref.distill(up, ids, lp, T, rest)[0][0] - ref.distill(down, ids, lp, T, rest)[0][0]) / (2 * h)
                assert np.allclose(d, g[:, i], atol=1e-8)
    x, dy, gain = rng.standard_normal((4, 9)), rng.standard_normal((4, 9)), rng.standard_normal(9)
    for center in (0, 1):
        (dx, _), (dg, _), _ = ref.norm_grad(x, dy, gain, 1e-3, center)
        value = lambda x, gain: (ref.norm(x, gain, None, 1e-3, center)[0] * dy).sum()
        for i in range(9):
            e = np.zeros((4, 9))
            e[2, i] = 1e-6
            assert abs((value(x + e, gain) - value(x - e, gain)) / 2e-6 - dx[2, i]) < 1e-7
            f = e[2]
            assert abs((value(x, gain + f) - value(x, gain - f)) / 2e-6 - dg[i]) < 1e-7
    x, w, dy, b = rng.standard_normal((4, 6)), rng.standard_normal((5, 6)), rng.standard_normal((4, 5)), rng.standard_normal(5)
    for kind in (0, 1, 2):
        value = lambda x, w, b: (ref.linear(x, w, b, None, kind, 0, 0)[0][0] * dy).sum()
        pre = x @ w.T + b
        (dx, _), (dw, _), (db, _) = ref.linear_grad(x, w, dy, pre, kind, 0, 0, 0, 0)
        for _ in range(5):
            ex, ew, eb = (1e-6 * rng.standard_normal(a.shape) for a in (x, w, b))
            d = (value(x + ex, w + ew, b + eb) - value(x - ex, w - ew, b - eb)) / 2
            assert abs(d - (dx * ex).sum() - (dw * ew).sum() - (db * eb).sum()) < 1e-11


def test_planted_mistakes_are_outside_the_tolerances():
    """What a wrong kernel would give, formed by the reference: each is further off than the tolerance."""
    rng = np.random.default_rng(6)
    z = np.float32(2 * rng.standard_normal((4, 1000))).astype(np.float64)
    tokens = rng.integers(0, 1000, 4)
    want = ref.score(z, tokens, 8, 0.7)
    for wrong in (ref.score(z[:, :999], np.minimum(tokens, 998), 8, 0.7), ref.score(z, tokens, 8, 0.7001)):   # the last token left out; another temperature
        assert (np.abs(wrong["entropy"][0] - want["entropy"][0]) > want["entropy"][1]).any()
        assert (np.abs(wrong["logprob"][0] - want["logprob"][0]) > want["logprob"][1]).any()
    ids = np.argsort(-z, 1)[:, :8]
    lp = np.log(np.full((4, 8), 0.1))
    (loss, tol), (grad, grad_tol) = ref.distill(z, ids, lp, 1.0, True)
    moved = z.copy()
    moved[:, 17] -= 0.05                                                                # one of a thousand tokens slightly off
    (l2, _), (g2, _) = ref.distill(moved, ids, lp, 1.0, True)
    assert (np.abs(l2 - loss) > tol).any() and (np.abs(g2 - grad) > grad_tol).sum() > 100
    for half in (2.0 ** -24, 2.0 ** -8):
        (_, _), (g3, t3) = ref.distill(z, ids, lp, 1.0, True, half=half)
        g4 = ref.distill(z, ids, lp, 1.0, False)[1][0]
        assert (np.abs(g4 - g3) > t3).mean() > 0.5
    x, dy, gain = rng.standard_normal((3, 700)), rng.standard_normal((3, 700)), 1 + 0.1 * rng.standard_normal(700)
    y, tol = ref.norm(x, gain, None, 1e-5, 1, 2.0 ** -8)
    assert (np.abs(ref.norm(x, gain, None, 1e-5, 0)[0] - y) > tol).any()
    (dx, tol), _, _ = ref.norm_grad(x, dy, gain, 1e-5, 1)
    assert (np.abs(ref.norm_grad(x, dy, gain, 1e-5, 0)[0][0] - dx) > tol).mean() > 0.5
    x, w = rng.standard_normal((5, 300)), rng.standard_normal((7, 300))
    (y, tol), _ = ref.linear(x, w, None, None, 1, 2.0 ** -8, 2.0 ** -8)
    x[:, 299] = 0                                                                       # the last element of the sums left out
    assert (np.abs(ref.linear(x, w, None, None, 1, 0, 0)[0][0] - y) > tol).any()


def test_more_parts_than_a_grid_are_refused():
    """2^20 rows of 2^24 tokens: refused before anything is launched (a workspace of any size is claimed, none is touched)."""
    lib = ee.load_library()
    size = dict(n_rows=1 << 20, vocab=1 << 24, logits_stride=1 << 24)
    refused(lib.ee_score_tokens(ctypes.byref(score_args(**size)), P, 1 << 60, None), "too many rows")
    refused(lib.ee_distill(ctypes.byref(distill_args(d_logits_stride=1 << 24, **size)), P, 1 << 60, None), "too many rows")
