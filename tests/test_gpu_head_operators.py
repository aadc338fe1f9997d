"""The operators around the LM head against plain 64-bit forms: ee_score_tokens, ee_distill, ee_norm, ee_linear and their gradients."""
import ctypes

import numpy as np
import pytest

import paper_2505_21594_amd as ee
from tests import head_ref as ref
from tests.device import Dev, FLOATS, HALF_STEP, decode, encode, hip, ok

pytestmark = pytest.mark.gpu

GUARD = 0x5A
FILL = 7.5
SUBNORMAL = {"bf16": 0.0, "fp32": 0.0, "fp16": 2.0 ** -25}


class Space:
    """A workspace with a guard behind it."""

    def __init__(self, n):
        self.n, self.all = n, Dev(np.full(n + 256, GUARD, np.uint8))
        self.view = self.all.view((n,), (1,))

    def check(self):
        assert (self.all.numpy()[self.n:] == GUARD).all()


class Rows:
    """[rows][width] of a type in rows of `stride` elements; what lies between them is filled with a value that a check finds again."""

    def __init__(self, x, kind, stride=None, shift=0):
        rows, width = x.shape
        self.kind, self.rows, self.width, self.stride, self.shift = kind, rows, width, stride or width, shift
        fill = encode(np.full(1, FILL, np.float32), kind)[0]
        self.host = np.full(rows * self.stride + shift + 16, fill, FLOATS[kind])
        self.inside()[:] = encode(np.asarray(x, np.float32), kind)
        self.dev = Dev(self.host)
        self.view = self.dev.view((rows, width), (self.stride, 1), shift)

    def inside(self, a=None):
        a = self.host if a is None else a
        return np.lib.stride_tricks.as_strided(a[self.shift:], (self.rows, self.width), (self.stride * a.itemsize, a.itemsize))

    def values(self):
        """As the call reads them."""
        return decode(np.ascontiguousarray(self.inside()))

    def result(self):
        got = self.dev.numpy()
        out = np.ascontiguousarray(self.inside(got)).copy()
        self.inside(got)[:] = self.inside()
        assert (got == self.host).all(), "elements outside the rows were written"
        return decode(out)


def empty(rows, width, kind, stride=None, shift=0):
    return Rows(np.full((rows, width), FILL, np.float32), kind, stride, shift)


def close(got, want, what):
    want, tol = want
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        bad = ~(same | (np.abs(got - want) <= tol))
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]} +- {np.broadcast_to(tol, got.shape)[bad][0]}"


def logits(rng, rows, V, kind, special=False):
    z = 2 * rng.standard_normal((rows, V))
    z[np.arange(rows), rng.integers(0, V, rows)] += 6
    z = decode(encode(z.astype(np.float32), kind))
    if special and rows >= 8:
        z[0, rng.random(V) < 0.9] = -np.inf                     # few tokens are allowed
        z[1] = -np.inf
        z[1, V // 2] = 1.0                                      # one is
        z[2] = -np.inf                                          # none
        z[3, V - 1] = np.inf
        z[4, 0] = np.nan
        z[5] = 0.0                                              # all alike ...
        z[5, ::3] = -0.0
        z[6] = np.round(z[6])                                   # ... or many
        z[7] = np.where(np.arange(V) < V - 3, -3e4, 3e4)        # far apart
    return decode(encode(z.astype(np.float32), kind))


# ---------------------------------------------------------------- ee_score_tokens

def run_score(z, kind, tokens, top, T, stride=None, shift=0, stream=0):
    rows, V = z.shape
    d = Rows(z, kind, stride, shift)
    lp, h = (Dev(np.full(rows, FILL, np.float32)) for _ in range(2))
    ids, tl = Dev(np.full((rows, top), -77, np.int32)), Dev(np.full((rows, top), FILL, np.float32))
    ws = Space(ee.ee_score_workspace(d.view, top=top))
    lists = dict(top_ids=ids, top_logprobs=tl) if top else {}
    ee.ee_score_tokens(d.view, Dev(np.asarray(tokens, np.int32)), logprob=lp, entropy=h, temperature=T, workspace=ws.view, stream=stream, **lists)
    got = [a.numpy() for a in (lp, h, ids, tl)]
    ws.check()
    return got


def check_score(z, kind, tokens, top, T, **kw):
    lp, h, ids, tl = run_score(z, kind, tokens, top, T, **kw)
    want = ref.score(z, tokens, top, T)
    assert (ids == want["top_ids"]).all(), f"lists differ in rows {np.unique(np.argwhere(ids != want['top_ids'])[:, 0])[:8]}"
    close(lp.astype(np.float64), want["logprob"], "logprob")
    close(h.astype(np.float64), want["entropy"], "entropy")
    close(tl.astype(np.float64), want["top_logprobs"], "top_logprobs")


SCORE = [(1, 1, 1), (1, 5, 8), (5, 1024, 4), (3, 2047, 64), (9, 4097, 20), (5, 32000, 5), (8, 8193, 33), (2, 100003, 64), (40, 300, 64), (600, 1100, 7), (520, 9000, 64), (514, 33000, 20)]


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,V,top", SCORE)
def test_score(rows, V, top, kind):
    rng = np.random.default_rng(rows * 7 + V)
    z = logits(rng, rows, V, kind, special=True)
    tokens = rng.integers(0, V, rows)
    tokens[-1:] = V                                             # (outside the vocabulary)
    if rows > 2:
        tokens[1] = -100
    pad = rows % 3
    check_score(z, kind, tokens, top, [1.0, 0.7, 2.5][V % 3], stride=V + pad, shift=pad)


def test_score_without_lists_and_numbers():
    rng = np.random.default_rng(3)
    z = logits(rng, 6, 3000, "fp32")
    check_score(z, "fp32", rng.integers(0, 3000, 6), 0, 1.0)
    d = Rows(z, "fp32")
    ids, tl = Dev(np.zeros((6, 4), np.int32)), Dev(np.zeros((6, 4), np.float32))
    ee.ee_score_tokens(d.view, top_ids=ids, top_logprobs=tl, workspace=Space(ee.ee_score_workspace(d.view, top=4)).view)
    assert (ids.numpy() == ref.score(z, None, 4, 1.0)["top_ids"]).all()


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_score_ties_and_orders(kind):
    """Rows sorted up, down, in blocks of equal ones, and one large token after another in the same thread's place."""
    V = 5000
    ramp = np.arange(V, dtype=np.float64)
    z = np.stack([ramp % 200, -(ramp % 200), np.floor(ramp / 40), -np.floor(ramp / 40), np.where(ramp % 1000 < 8, 5.0, -ramp / V), np.zeros(V) - 4,
                  np.where(ramp == 4999, 1.0, -np.inf), np.where(ramp < 64, 2.0, 1.0)] * 70)
    z = decode(encode(z.astype(np.float32), kind))
    for rows in (8, 560):
        check_score(z[:rows], kind, np.arange(rows) * 3, 64, 1.0)
        check_score(z[:rows], kind, np.arange(rows) * 3, 5, 1.0)


def test_score_many_parts():
    """More parts than a wave of the second launch takes at once, and lists beyond its room for one step."""
    rng = np.random.default_rng(11)
    z = logits(rng, 2, 700001, "bf16")
    check_score(z, "bf16", [700000, 3], 64, 1.0)


# ---------------------------------------------------------------- ee_distill

def teacher(rng, z, top, T, kind="near"):
    rows, V = z.shape
    t = np.where(np.isfinite(z), z, 0) / T + 0.5 * rng.standard_normal(z.shape)
    t -= np.log(np.exp(t - t.max(1, keepdims=True)).sum(1, keepdims=True)) + t.max(1, keepdims=True)
    ids = np.argsort(-t, 1, kind="stable")[:, :top].astype(np.int32)
    lp = np.take_along_axis(t, ids, 1).astype(np.float32)
    if ids.shape[1] < top:                                       # as ee_score_tokens ends a list
        ids = np.concatenate([ids, np.full((rows, top - V), -1, np.int32)], 1)
        lp = np.concatenate([lp, np.full((rows, top - V), -np.inf, np.float32)], 1)
    if kind == "odd":
        lp -= np.float32(0.4)
        for r in range(rows):
            if r % 5 == 1:
                ids[r, -1] = ids[r, 0]                           # a token twice
            if r % 5 == 2:
                ids[r, 0], ids[r, -1] = V, -5                    # tokens that are none
            if r % 5 == 3:
                lp[r, :] = -np.inf                               # no list at all
            if r % 5 == 4:
                lp[r, top // 2] = -np.inf
    return ids, lp


def run_distill(z, kind, ids, lp, T, rest, out, weight=None, stride=None, shift=0, want_loss=True, want_grad=True, in_place=False, stream=0):
    rows, V = z.shape
    d = Rows(z, kind, stride, shift)
    g = d if in_place else empty(rows, V, out, stride, shift)
    loss = Dev(np.full(rows, FILL, np.float32))
    ws = Space(ee.ee_distill_workspace(d.view, top=ids.shape[1]))
    ee.ee_distill(d.view, Dev(ids), Dev(lp), loss=loss if want_loss else None, d_loss=None if weight is None else Dev(np.asarray(weight, np.float32)),
                  d_logits=g.view if want_grad else None, rest=rest, temperature=T, workspace=ws.view, stream=stream)
    a = loss.numpy().astype(np.float64)
    b = g.result() if want_grad else None
    ws.check()
    return a, b


def check_distill(z, kind, ids, lp, T, rest, out, weight=None, **kw):
    (loss, grad), (want_loss, want_grad) = run_distill(z, kind, ids, lp, T, rest, out, weight, **kw), ref.distill(z, ids, lp, T, rest, weight, HALF_STEP[out], SUBNORMAL[out])
    if kw.get("want_loss", True):
        close(loss, want_loss, "loss")
    if grad is not None:
        close(grad, want_grad, "gradient")


DISTILL = [(1, 1, 1), (1, 5, 8), (64, 1024, 8), (3, 2047, 64), (9, 4097, 20), (5, 32000, 5), (2, 100003, 64), (300, 300, 33), (260, 9000, 64), (257, 33000, 7), (256, 70001, 16)]


@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("kind,out", [("bf16", "bf16"), ("fp16", "fp32"), ("fp32", "fp32"), ("fp32", "bf16")])
@pytest.mark.parametrize("rows,V,top", DISTILL)
def test_distill(rows, V, top, kind, out, rest):
    rng = np.random.default_rng(rows * 3 + V)
    z = logits(rng, rows, V, kind, special=True)
    T = [1.0, 0.7, 2.5][V % 3]
    ids, lp = teacher(rng, z, top, T, "odd" if rows > 4 else "near")
    weight = np.where(rng.random(rows) < 0.3, 0, rng.standard_normal(rows)).astype(np.float32)
    pad = rows % 3
    check_distill(z, kind, ids, lp, T, rest, out, weight, stride=V + pad, shift=pad)


@pytest.mark.parametrize("rows,V", [(7, 5000), (300, 700), (270, 40000), (3, 40000)])
def test_distill_one_result_and_in_place(rows, V):
    rng = np.random.default_rng(V)
    z = logits(rng, rows, V, "bf16")
    ids, lp = teacher(rng, z, 16, 1.0)
    for kw in (dict(want_grad=False), dict(want_loss=False), dict(in_place=True)):
        check_distill(z, "bf16", ids, lp, 1.0, True, "bf16", **kw)


@pytest.mark.parametrize("T", [2.5, 0.7, 1.0])
def test_log_probabilities_of_far_tokens(T):
    """A far token's log-probability is rounded once, at 2^-24 of it: the factor log2(e) / T in fp32 (0.82 of that off for T = 2.5) has no part in it."""
    rng = np.random.default_rng(31)
    rows, V = 64, 300
    z = 2 * rng.standard_normal((rows, V))
    z[:, 7] = -np.exp(rng.uniform(np.log(1e2), np.log(6e4), rows))
    z = decode(encode(z.astype(np.float32), "fp32"))
    check_score(z, "fp32", np.full(rows, 7), 8, T)
    ids, lp = np.full((rows, 1), 7, np.int32), np.zeros((rows, 1), np.float32)
    check_distill(z, "fp32", ids, lp, T, False, "fp32")
    far = decode(encode((z[:, 7:8] + np.arange(9)[None] / 4).astype(np.float32), "fp32"))
    far[:, 4] = 3.0                                              # the one token that the teacher names, with half its probability; the others are far
    check_distill(far, "fp32", np.full((rows, 1), 4, np.int32), np.full((rows, 1), np.log(0.5), np.float32), T, True, "fp32")


@pytest.mark.parametrize("T", [2.5, 0.7, 2.0])
@pytest.mark.parametrize("rows,V", [(64, 1024), (5, 32000), (300, 9000), (3, 140001)])
def test_small_divergences_keep_their_digits(rows, V, T):
    """A teacher that is nearly the student: what the sums are off by cancels, and the loss is off by 2^-24 of it and of what the teacher differs by."""
    rng = np.random.default_rng(rows + V)
    z = logits(rng, rows, V, "fp32")
    other = z + 1e-3 * rng.standard_normal(z.shape)
    t = float(np.float32(T))
    ids = np.argsort(-z, 1)[:, :32].astype(np.int32)
    lse = other.max(1, keepdims=True) / t + np.log(np.exp((other - other.max(1, keepdims=True)) / t).sum(1, keepdims=True))
    lp = (np.take_along_axis(other, ids, 1) / t - lse).astype(np.float32)
    check_distill(z, "fp32", ids, lp, T, True, "fp32", want_grad=False)
    check_distill(z, "fp32", ids, lp, T, False, "fp32")


@pytest.mark.parametrize("rows,V,kind", [(2, 140001, "bf16"), (2, 70001, "fp32"), (260, 140001, "bf16")])
def test_distill_in_place_in_parts(rows, V, kind):
    """Rows too long for a workgroup: the second launch reads logits where the first parts of the same row hold gradients already."""
    rng = np.random.default_rng(V + rows)
    z = logits(rng, rows, V, kind, special=True)
    ids, lp = teacher(rng, z, 64, 0.7, "near")
    ids[:, 0], ids[:, 1] = 0, V - 1
    weight = np.where(np.arange(rows) % 2, 0, 1.5).astype(np.float32)
    check_distill(z, kind, ids, lp, 0.7, True, kind, weight, in_place=True)


def test_distill_label_is_cross_entropy():
    rng = np.random.default_rng(2)
    z = logits(rng, 5, 900, "fp32")
    label = rng.integers(0, 900, (5, 1)).astype(np.int32)
    loss, grad = run_distill(z, "fp32", label, np.zeros((5, 1), np.float32), 1.0, False, "fp32")
    p = np.exp(z - z.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    assert np.allclose(loss, -np.log(p[np.arange(5), label[:, 0]]), atol=2 * ref.SUM)
    p[np.arange(5), label[:, 0]] -= 1
    assert np.abs(grad - p).max() < 4 * ref.SUM


def test_distill_extreme_students():
    """A student with next to nothing, or nothing, for the tokens that the list does not name, or for one that it does."""
    V = 600
    z = np.full((6, V), -50.0)
    z[:, :4] = [1.0, 2.0, 0.5, 1.5]
    z[1, 4:] = -180.0                                            # below the numbers of fp32
    z[2, 4:] = -np.inf
    z[3, 2] = -np.inf
    z[4, 2] = 300.0
    z[5, 4:] = 300.0
    ids = np.tile(np.arange(4, dtype=np.int32), (6, 1))
    lp = np.log(np.tile(np.array([[0.1, 0.5, 0.1, 0.2]]), (6, 1))).astype(np.float32)
    for rest in (True, False):
        check_distill(z, "fp32", ids, lp, 1.0, rest, "fp32")
    # a list that names every token leaves nothing over, whatever its rounding
    z = logits(np.random.default_rng(1), 4, 8, "fp32")
    ids = np.tile(np.arange(8, dtype=np.int32), (4, 1))
    lp = np.log(np.full((4, 8), 0.12)).astype(np.float32)
    check_distill(z, "fp32", ids, lp, 1.0, True, "fp32")


@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("rows,V", [(3, 3000), (300, 500)])
def test_distill_gradient_agrees_with_differences(rows, V, rest):
    rng = np.random.default_rng(V)
    z = logits(rng, rows, V, "fp32")
    ids, lp = teacher(rng, z, 12, 1.5)
    _, grad = run_distill(z, "fp32", ids, lp, 1.5, rest, "fp32")
    along = np.float32(rng.standard_normal(z.shape)).astype(np.float64)
    h = 2.0 ** -5
    up, down = (np.float32(z + s * h * along).astype(np.float64) for s in (1, -1))
    lu, ld = (run_distill(x, "fp32", ids, lp, 1.5, rest, "fp32", want_grad=False)[0] for x in (up, down))
    wu, wd = (ref.distill(x, ids, lp, 1.5, rest)[0][0] for x in (up, down))
    # the differences' own error (third derivatives) is what the reference's differences have
    slope = (grad * (up - down)).sum(1)
    third = np.abs((wu - wd) - (ref.distill(z, ids, lp, 1.5, rest)[1][0] * (up - down)).sum(1))
    assert (np.abs((lu - ld) - slope) <= 2 * third + 8 * ref.SUM).all()


# ---------------------------------------------------------------- ee_norm

NORM = [(1, 1), (3, 7), (5, 64), (9, 256), (2, 1000), (5, 1025), (4, 4096), (3, 5120), (2, 8191), (2, 16384), (1030, 24), (700, 1536), (520, 2048), (300, 10000)]


@pytest.mark.parametrize("center", [False, True])
@pytest.mark.parametrize("kind,out", [("bf16", "bf16"), ("fp32", "bf16"), ("fp16", "fp32"), ("fp32", "fp32")])
@pytest.mark.parametrize("rows,dim", NORM)
def test_norm(rows, dim, kind, out, center):
    rng = np.random.default_rng(rows + dim)
    x = rng.standard_normal((rows, dim)) * rng.uniform(0.1, 3, (rows, 1)) + 0.5
    x[0] = 0 if dim > 1 else x[0]                               # (a row of zeros: eps alone)
    gain, bias = (np.float32(rng.standard_normal(dim)) for _ in range(2))
    gain, bias = (gain, bias) if dim % 3 else (None, None) if dim % 2 else (gain, None)
    pad = (rows + dim) % 3
    d, y = Rows(x, kind, dim + pad, pad), empty(rows, dim, out, dim + 2 * pad)
    ee.ee_norm(d.view, y.view, gain=None if gain is None else Dev(gain), bias=None if bias is None else Dev(bias), eps=1e-5, center=center)
    close(y.result(), ref.norm(d.values(), gain, bias, 1e-5, center, HALF_STEP[out]), "y")
    dy, dx = Rows(rng.standard_normal((rows, dim)), out, dim + pad), empty(rows, dim, kind, dim + 2 * pad, pad)
    dg, db = (Dev(np.full(dim + 1, FILL, np.float32)) for _ in range(2))
    ws = Space(ee.ee_norm_grad_workspace(d.view))
    ee.ee_norm_grad(d.view, dy.view, dx=dx.view, gain=None if gain is None else Dev(gain), d_gain=dg, d_bias=db, eps=1e-5, center=center, workspace=ws.view)
    ws.check()
    want = ref.norm_grad(d.values(), dy.values(), gain, 1e-5, center, HALF_STEP[kind])
    close(dx.result(), (want[0][0], want[0][1] + SUBNORMAL[kind]), "dx")
    for got, w, what in ((dg, want[1], "d_gain"), (db, want[2], "d_bias")):
        got = got.numpy().astype(np.float64)
        close(got[:dim], w, what)
        assert got[dim] == FILL


def test_norm_parts_and_places():
    rng = np.random.default_rng(8)
    for rows, dim in ((6, 300), (5, 4096)):
        x, dy = Rows(rng.standard_normal((rows, dim)), "bf16"), Rows(rng.standard_normal((rows, dim)), "bf16")
        xv, dyv = x.values(), dy.values()
        want = ref.norm_grad(xv, dyv, None, 1e-6, 1, HALF_STEP["bf16"])
        dx = empty(rows, dim, "bf16")
        ee.ee_norm_grad(x.view, dy.view, dx=dx.view, eps=1e-6, center=True)          # no sums wanted: no workspace
        close(dx.result(), want[0], "dx alone")
        db = Dev(np.zeros(dim, np.float32))
        ws = Space(ee.ee_norm_grad_workspace(x.view))
        ee.ee_norm_grad(x.view, dy.view, d_bias=db, eps=1e-6, center=True, workspace=ws.view)
        close(db.numpy().astype(np.float64), want[2], "d_bias alone")
        ee.ee_norm_grad(x.view, dy.view, dx=dy.view, eps=1e-6, center=True)
        close(dy.result(), want[0], "dx in dy's place")
        ee.ee_norm(x.view, x.view, eps=1e-6, center=True)
        close(x.result(), ref.norm(xv, None, None, 1e-6, 1, HALF_STEP["bf16"]), "y in x's place")


def test_norm_of_no_rows_and_special_values():
    x = Rows(np.ones((4, 128)), "fp32")
    none = x.dev.view((0, 128), (128, 1))
    dg, db = (Dev(np.full(128, FILL, np.float32)) for _ in range(2))
    ws = Space(max(ee.ee_norm_grad_workspace(none), 256))
    ee.ee_norm_grad(none, none, dx=none, d_gain=dg, d_bias=db, workspace=ws.view)
    assert (dg.numpy() == 0).all() and (db.numpy() == 0).all()
    v = np.random.default_rng(0).standard_normal((4, 128))
    v[1, 5], v[2, 7] = np.nan, np.inf
    x, y = Rows(v, "fp32"), empty(4, 128, "fp32")
    ee.ee_norm(x.view, y.view)
    got = y.result()
    assert np.isfinite(got[[0, 3]]).all() and np.isnan(got[1]).all() and np.isnan(got[2, 7]) and (np.delete(got[2], 7) == 0).all()


def test_norm_far_from_zero():
    """A mean that is large beside the spread: the squares are taken about it."""
    x = Rows(np.random.default_rng(4).standard_normal((3, 5000)) + 3000, "fp32")
    y = empty(3, 5000, "fp32")
    ee.ee_norm(x.view, y.view, center=True)
    close(y.result(), ref.norm(x.values(), None, None, 1e-5, 1), "y")


# ---------------------------------------------------------------- ee_linear

def up8(n):
    return -(-n // 8) * 8


def matrix(rng, rows, width, kind, scale=1.0, pad=0):
    return Rows(scale * rng.standard_normal((rows, width)), kind, up8(width) + 8 * pad, 8 * pad)


LINEAR = [(1, 1, 1), (1, 64, 32), (5, 256, 688), (16, 100, 17), (17, 33, 130), (48, 96, 64), (3, 1000, 300), (129, 65, 127), (130, 512, 256), (257, 40, 384), (64, 384, 129), (300, 264, 520)]


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,n_in,n_out", LINEAR)
def test_linear(rows, n_in, n_out, kind):
    rng = np.random.default_rng(rows + n_in * 3 + n_out)
    pad = rows % 2
    x, w = matrix(rng, rows, n_in, kind, pad=pad), matrix(rng, n_out, n_in, kind, 0.2, pad)
    for act, out, with_bias, res in ((ee.ACT_NONE, kind, False, None), (ee.ACT_SILU, kind, True, None), (ee.ACT_GELU, "fp32", True, "fp32"), (ee.ACT_SILU, "fp32", False, kind), (ee.ACT_NONE, kind, True, "fp32")):
        bias = np.float32(rng.standard_normal(n_out)) if with_bias else None
        residual = matrix(rng, rows, n_out, res, pad=pad) if res else None
        y = empty(rows, n_out, out, up8(n_out) + 8 * pad, 8 * pad)
        pre = empty(rows, n_out, kind, up8(n_out)) if act else None
        ws = Space(ee.ee_linear_workspace(x.view, w.view))
        ee.ee_linear(x.view, w.view, y.view, bias=None if bias is None else Dev(bias), act=act, residual=residual and residual.view, pre=pre and pre.view, workspace=ws.view)
        ws.check()
        want_y, want_pre = ref.linear(x.values(), w.values(), bias, residual.values() if residual else None, act, HALF_STEP[out], HALF_STEP[kind])
        close(y.result(), (want_y[0], want_y[1] + SUBNORMAL[out]), f"y, activation {act}, {out}")
        if pre:
            close(pre.result(), (want_pre[0], want_pre[1] + SUBNORMAL[kind]), "pre")


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,n_in,n_out", LINEAR)
def test_linear_grad(rows, n_in, n_out, kind):
    rng = np.random.default_rng(rows + n_in * 5 + n_out)
    pad = rows % 2
    x, w = matrix(rng, rows, n_in, kind, pad=pad), matrix(rng, n_out, n_in, kind, 0.2)
    dy, pre = matrix(rng, rows, n_out, kind), matrix(rng, rows, n_out, kind, 1.5, pad)
    for act, out_x, out_w in ((ee.ACT_NONE, kind, "fp32"), (ee.ACT_SILU, kind, kind), (ee.ACT_GELU, "fp32", kind), (ee.ACT_SILU, kind, "fp32")):
        dx, dw = empty(rows, n_in, out_x, up8(n_in) + 8 * pad), empty(n_out, n_in, out_w, up8(n_in), 8 * pad)
        db = Dev(np.full(n_out + 1, FILL, np.float32))
        ws = Space(ee.ee_linear_grad_workspace(x.view, w.view, act=act))
        ee.ee_linear_grad(x.view, w.view, dy.view, pre=pre.view if act else None, act=act, dx=dx.view, d_weight=dw.view, d_bias=db, workspace=ws.view)
        ws.check()
        # dz is rounded once for 16-bit results; to 2^-24 (three terms of bf16), 2^-22 (two of fp16, or half its smallest number) for fp32
        step = {out: (2.0 ** -22 if kind == "fp16" else 2.0 ** -24) if out == "fp32" else HALF_STEP[kind] for out in (out_x, out_w)} if act else {out_x: 0, out_w: 0}
        want = ref.linear_grad(x.values(), w.values(), dy.values(), pre.values(), act, HALF_STEP[out_x], HALF_STEP[out_w], step[out_x], step[out_w])
        small = 2.0 ** -25 if kind == "fp16" and act else 0.0                          # of dz
        close(dx.result(), (want[0][0], want[0][1] + SUBNORMAL[out_x] + small * np.abs(w.values()).sum(0)), f"dx, activation {act}")
        close(dw.result(), (want[1][0], want[1][1] + SUBNORMAL[out_w] + small * np.abs(x.values()).sum(0)), f"d_weight, activation {act}")
        got = db.numpy().astype(np.float64)
        close(got[:n_out], want[2], "d_bias")
        assert got[n_out] == FILL


class Large:
    """Matrices for products that fill the chip, made of few different rows so that the 64-bit form is quick: row i is row i % 37 of a small one."""

    def __init__(self, rng, rows, width, kind, scale=1.0):
        self.small = Rows(scale * rng.standard_normal((37, width)), kind, up8(width))
        self.index = np.arange(rows) % 37
        self.all = Rows(np.zeros((1, 1)), kind)
        host = np.ascontiguousarray(self.small.inside())[self.index]
        wide = np.full((rows, up8(width) + 8), encode(np.full(1, np.nan, np.float32), kind)[0])
        wide[:, :width] = host
        self.dev = Dev(wide)
        self.view = self.dev.view((rows, width), (up8(width) + 8, 1))

    def values(self):
        return self.small.values()


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,n_in,n_out", [(2600, 96, 2100), (2050, 133, 2433), (4100, 64, 1025), (40000, 40, 72), (72, 8200, 40), (5, 72, 26000), (20, 40, 26003), (16, 2100, 13000)])
def test_linear_that_fills_the_chip(rows, n_in, n_out, kind):
    """Every result, by the large tiles or in parts of the sum."""
    rng = np.random.default_rng(rows)
    x, w = Large(rng, rows, n_in, kind), Large(rng, n_out, n_in, kind, 0.2)
    bias = np.float32(rng.standard_normal(n_out))
    y, pre = empty(rows, n_out, "fp32", up8(n_out)), empty(rows, n_out, kind, up8(n_out))
    ws = Space(ee.ee_linear_workspace(x.view, w.view))
    ee.ee_linear(x.view, w.view, y.view, bias=Dev(bias), act=ee.ACT_SILU, pre=pre.view, workspace=ws.view)
    ws.check()
    z = (x.values() @ w.values().T)[x.index][:, w.index] + bias
    size = (np.abs(x.values()) @ np.abs(w.values()).T)[x.index][:, w.index]
    tol_z = (n_in + 2) * ref.U * size + 2 * ref.U * np.abs(z)
    value = ref.act(z, 1)
    close(y.result(), (value, 1.13 * tol_z + ref.ACT * (np.abs(z) + np.abs(value)) + ref.U * np.abs(value)), "y")
    close(pre.result(), (z, tol_z + HALF_STEP[kind] * np.abs(z) * (1 + 2.0 ** -8) + SUBNORMAL[kind]), "pre")
    # backward: dy of 37 kinds of rows as well, by columns of 37 kinds
    d = rng.standard_normal((37, 37))
    dy = Rows(d[x.index][:, w.index], kind, up8(n_out) + 8)
    dv = decode(encode(d.astype(np.float32), kind))
    dx, dw, db = empty(rows, n_in, "fp32", up8(n_in)), empty(n_out, n_in, "fp32", up8(n_in)), Dev(np.zeros(n_out, np.float32))
    ws = Space(ee.ee_linear_grad_workspace(x.view, w.view))
    ee.ee_linear_grad(x.view, w.view, dy.view, dx=dx.view, d_weight=dw.view, d_bias=db, workspace=ws.view)
    ws.check()
    nx, nw = np.bincount(x.index, minlength=37).astype(float), np.bincount(w.index, minlength=37).astype(float)
    want = (dv * nw) @ w.values()
    close(dx.result(), (want[x.index], ((n_out + 2) * ref.U * ((np.abs(dv) * nw) @ np.abs(w.values())))[x.index]), "dx")
    want = (dv.T * nx) @ x.values()
    close(dw.result(), (want[w.index], ((rows + 2) * ref.U * ((np.abs(dv).T * nx) @ np.abs(x.values())))[w.index]), "d_weight")
    close(db.numpy().astype(np.float64), ((dv.T @ nx)[w.index], (rows * ref.U * (np.abs(dv).T @ nx))[w.index]), "d_bias")


def test_linear_one_result_at_a_time_and_no_rows():
    rng = np.random.default_rng(9)
    x, w, dy = matrix(rng, 70, 96, "bf16"), matrix(rng, 40, 96, "bf16"), matrix(rng, 70, 40, "bf16")
    want = ref.linear_grad(x.values(), w.values(), dy.values(), None, 0, HALF_STEP["bf16"], HALF_STEP["bf16"], 0, 0)
    ws = Space(ee.ee_linear_grad_workspace(x.view, w.view))
    dx, dw, db = empty(70, 96, "bf16"), empty(40, 96, "bf16"), Dev(np.full(40, FILL, np.float32))
    ee.ee_linear_grad(x.view, w.view, dy.view, dx=dx.view, workspace=ws.view)
    close(dx.result(), want[0], "dx alone")
    ee.ee_linear_grad(x.view, w.view, dy.view, d_weight=dw.view, workspace=ws.view)
    close(dw.result(), want[1], "d_weight alone")
    ee.ee_linear_grad(x.view, w.view, dy.view, d_bias=db, workspace=ws.view)
    close(db.numpy().astype(np.float64), want[2], "d_bias alone")
    none_x, none_y = x.dev.view((0, 96), (96, 1)), dy.dev.view((0, 40), (40, 1))
    ee.ee_linear_grad(none_x, w.view, none_y, dx=dx.dev.view((0, 96), (96, 1)), d_weight=dw.view, d_bias=db, workspace=ws.view)
    assert (dw.result() == 0).all() and (db.numpy() == 0).all()


def test_linear_residual_in_place():
    rng = np.random.default_rng(12)
    x, w, h = matrix(rng, 37, 64, "bf16"), matrix(rng, 56, 64, "bf16"), matrix(rng, 37, 56, "fp32")
    want = ref.linear(x.values(), w.values(), None, h.values(), 0, HALF_STEP["fp32"], 0)[0]
    ws = Space(ee.ee_linear_workspace(x.view, w.view))
    ee.ee_linear(x.view, w.view, h.view, residual=h.view, workspace=ws.view)
    close(h.result(), want, "y in the residual's place")


def test_linear_does_not_read_behind_rows():
    """NaN between the rows and behind the last element of an odd length."""
    for rows, n_in, n_out in ((20, 77, 45), (150, 131, 133)):
        rng = np.random.default_rng(n_in)

        def poisoned(r, c):
            m = Rows(rng.standard_normal((r, c)), "bf16", up8(c) + 8)
            keep = m.inside().copy()
            m.host[:] = 0x7FC0
            m.inside()[:] = keep
            m.dev.write(m.host)
            return m

        x, w, dy = poisoned(rows, n_in), poisoned(n_out, n_in), poisoned(rows, n_out)
        y, dx, dw = empty(rows, n_out, "fp32", up8(n_out)), empty(rows, n_in, "fp32", up8(n_in)), empty(n_out, n_in, "fp32", up8(n_in))
        ws = Space(max(ee.ee_linear_workspace(x.view, w.view), ee.ee_linear_grad_workspace(x.view, w.view)))
        ee.ee_linear(x.view, w.view, y.view, workspace=ws.view)
        close(y.result(), ref.linear(x.values(), w.values(), None, None, 0, 2.0 ** -24, 0)[0], "y")
        ee.ee_linear_grad(x.view, w.view, dy.view, dx=dx.view, d_weight=dw.view, workspace=ws.view)
        want = ref.linear_grad(x.values(), w.values(), dy.values(), None, 0, 2.0 ** -24, 2.0 ** -24, 0, 0)
        close(dx.result(), want[0], "dx")
        close(dw.result(), want[1], "d_weight")


# ---------------------------------------------------------------- far apart

class far_rows:
    """Rows so far apart that offsets pass 32 bits."""

    def __init__(self, x, kind, stride):
        self.host = np.ascontiguousarray(encode(np.asarray(x, np.float32), kind))
        self._stride, item = stride, self.host.itemsize
        self._p = ctypes.c_void_p()
        ok(hip().hipMalloc(ctypes.byref(self._p), ((len(x) - 1) * stride + x.shape[1]) * item + 256))
        for r in range(len(x)):
            ok(hip().hipMemcpy(self._p.value + r * stride * item, self.host[r].ctypes.data, x.shape[1] * item, 1))
        like = Dev(self.host[:1])
        self.shape, self.dtype, self.device = x.shape, like.dtype, like.device

    def data_ptr(self):
        return self._p.value

    def stride(self):
        return (self._stride, 1)

    def result(self):
        out = np.empty_like(self.host)
        ok(hip().hipDeviceSynchronize())
        for r in range(len(out)):
            ok(hip().hipMemcpy(out[r].ctypes.data, self._p.value + r * self._stride * out.itemsize, out.shape[1] * out.itemsize, 2))
        return decode(out)

    def __del__(self):
        hip().hipFree(self._p)


def test_rows_beyond_32_bits():
    rng = np.random.default_rng(0)
    far = (1 << 31) + 8                                            # elements from row to row
    z = logits(rng, 3, 700, "bf16")
    d, g = far_rows(z, "bf16", far), far_rows(z, "bf16", far)
    ids, tl = Dev(np.zeros((3, 5), np.int32)), Dev(np.zeros((3, 5), np.float32))
    ee.ee_score_tokens(d, top_ids=ids, top_logprobs=tl, workspace=Space(ee.ee_score_workspace(d, top=5)).view)
    want = ref.score(z, None, 5, 1.0)
    assert (ids.numpy() == want["top_ids"]).all()
    ee.ee_distill(d, ids, tl, d_logits=g, workspace=Space(ee.ee_distill_workspace(d, top=5)).view)
    close(g.result(), ref.distill(z, want["top_ids"], tl.numpy(), 1.0, True, None, HALF_STEP["bf16"])[1], "gradient")
    x = decode(encode(rng.standard_normal((3, 64)).astype(np.float32), "bf16"))
    d, y, dy = far_rows(x, "bf16", far), far_rows(0 * x, "bf16", far), far_rows(x[::-1], "bf16", far)
    ee.ee_norm(d, y)
    close(y.result(), ref.norm(x, None, None, 1e-5, 0, HALF_STEP["bf16"]), "norm")
    ee.ee_norm_grad(d, dy, dx=y)
    close(y.result(), ref.norm_grad(x, x[::-1], None, 1e-5, 0, HALF_STEP["bf16"])[0], "norm's gradient")
    w = matrix(rng, 40, 64, "bf16")
    y, dx, dw = far_rows(np.zeros((3, 40)), "bf16", far), far_rows(0 * x, "bf16", far), empty(40, 64, "fp32")
    v = decode(encode(rng.standard_normal((3, 40)).astype(np.float32), "bf16"))
    dy = far_rows(v, "bf16", far)
    ws = Space(max(ee.ee_linear_workspace(d, w.view), ee.ee_linear_grad_workspace(d, w.view)))
    ee.ee_linear(d, w.view, y, workspace=ws.view)
    close(y.result(), ref.linear(x, w.values(), None, None, 0, HALF_STEP["bf16"], 0)[0], "linear")
    ee.ee_linear_grad(d, w.view, dy, dx=dx, d_weight=dw.view, workspace=ws.view)
    want = ref.linear_grad(x, w.values(), v, None, 0, HALF_STEP["bf16"], 2.0 ** -24, 0, 0)
    close(dx.result(), want[0], "dx")
    close(dw.result(), want[1], "d_weight")


def test_linear_rows_beyond_offsets_of_a_tile():
    """Rows of operands farther apart than 32-bit offsets within a tile allow."""
    rng = np.random.default_rng(1)
    for rows in (5, 70):
        x = decode(encode(rng.standard_normal((rows, 96)).astype(np.float32), "bf16"))
        d, w, y = far_rows(x, "bf16", (1 << 22) + 8), matrix(rng, 72, 96, "bf16"), empty(rows, 72, "fp32")
        ws = Space(ee.ee_linear_workspace(d, w.view))
        ee.ee_linear(d, w.view, y.view, workspace=ws.view)
        close(y.result(), ref.linear(x, w.values(), None, None, 0, 2.0 ** -24, 0)[0], "y")


# ---------------------------------------------------------------- a run of them together

class Step:
    """A training step of an exit head: its adapters (down, SiLU, up, residual), norm and head matrix, against the target's most likely tokens."""
    ROWS, D, A, V, TOP, T = 40, 256, 24, 1024, 12, 1.5

    def __init__(self, seed):
        self.rng = rng = np.random.default_rng(seed)
        R, D, A, V = self.ROWS, self.D, self.A, self.V
        self.h, self.target = matrix(rng, R, D, "fp32"), Rows(logits(rng, R, V, "fp32"), "fp32")
        self.hb = Rows(self.h.values(), "bf16")
        self.down, self.up, self.head = matrix(rng, A, D, "bf16", 0.06), matrix(rng, D, A, "bf16", 0.2), matrix(rng, V, D, "bf16", 0.05)
        self.b_down, self.b_up, self.gain = (np.float32(0.1 * rng.standard_normal(n)) for n in (A, D, D))
        self.gain += 1
        self.dev = {k: Dev(getattr(self, k)) for k in ("b_down", "b_up", "gain")}
        e = {k: empty(R, n, kind) for k, n, kind in (("t", A, "bf16"), ("pre", A, "bf16"), ("a", D, "fp32"), ("n", D, "bf16"), ("z", V, "bf16"), ("dz", V, "bf16"), ("dn", D, "fp32"),
                                                     ("da", D, "bf16"), ("dt", A, "bf16"))}
        e.update({k: empty(n, m, "fp32") for k, n, m in (("d_head", V, D), ("d_up", D, A), ("d_down", A, D))})
        self.e = e
        self.o = {k: Dev(np.zeros(n, np.float32)) for k, n in (("loss", R), ("d_gain", D), ("d_b_up", D), ("d_b_down", A))}
        self.ids, self.lps = Dev(np.zeros((R, self.TOP), np.int32)), Dev(np.zeros((R, self.TOP), np.float32))
        self.weight = Dev(np.full(R, 1.0 / R, np.float32))
        v = {k: x.view for k, x in e.items()}
        sizes = [ee.ee_score_workspace(self.target.view, top=self.TOP), ee.ee_distill_workspace(v["z"], top=self.TOP), ee.ee_norm_grad_workspace(v["a"])]
        for x, w, act in ((self.hb.view, self.down.view, 1), (v["t"], self.up.view, 0), (v["n"], self.head.view, 0)):
            sizes += [ee.ee_linear_workspace(x, w), ee.ee_linear_grad_workspace(x, w, act=act)]
        self.ws = Space(max(sizes))

    def run(self, stream=0):
        v, kw = {k: x.view for k, x in self.e.items()}, dict(workspace=self.ws.view, stream=stream)
        ee.ee_score_tokens(self.target.view, top_ids=self.ids, top_logprobs=self.lps, temperature=self.T, **kw)
        ee.ee_linear(self.hb.view, self.down.view, v["t"], bias=self.dev["b_down"], act=ee.ACT_SILU, pre=v["pre"], **kw)
        ee.ee_linear(v["t"], self.up.view, v["a"], bias=self.dev["b_up"], residual=self.h.view, **kw)
        ee.ee_norm(v["a"], v["n"], gain=self.dev["gain"], stream=stream)
        ee.ee_linear(v["n"], self.head.view, v["z"], **kw)
        ee.ee_distill(v["z"], self.ids, self.lps, loss=self.o["loss"], d_loss=self.weight, d_logits=v["dz"], temperature=self.T, **kw)
        ee.ee_linear_grad(v["n"], self.head.view, v["dz"], dx=v["dn"], d_weight=v["d_head"], **kw)
        ee.ee_norm_grad(v["a"], v["dn"], dx=v["da"], gain=self.dev["gain"], d_gain=self.o["d_gain"], **kw)
        ee.ee_linear_grad(v["t"], self.up.view, v["da"], dx=v["dt"], d_weight=v["d_up"], d_bias=self.o["d_b_up"], **kw)
        ee.ee_linear_grad(self.hb.view, self.down.view, v["dt"], pre=v["pre"], act=ee.ACT_SILU, d_weight=v["d_down"], d_bias=self.o["d_b_down"], **kw)

    def results(self):
        out = {k: self.o[k].numpy().astype(np.float64) for k in self.o}
        return dict(out, **{k: self.e[k].result() for k in ("d_head", "d_up", "d_down", "z")}, ids=self.ids.numpy(), lps=self.lps.numpy())

    def reference(self, move=None):
        """In 64 bits without any rounding in between; `move`: what is added to the weights, to take differences."""
        w = {k: getattr(self, k).values() for k in ("down", "up", "head")}
        w.update(b_down=self.b_down.astype(np.float64), b_up=self.b_up.astype(np.float64), gain=self.gain.astype(np.float64))
        if move:
            w = {k: w[k] + move.get(k, 0) for k in w}
        lists = ref.score(self.target.values(), None, self.TOP, self.T)
        hb, h = self.hb.values(), self.h.values()
        pre = hb @ w["down"].T + w["b_down"]
        t = ref.act(pre, 1)
        a = h + t @ w["up"].T + w["b_up"]
        n = ref.norm(a, w["gain"], None, 1e-5, 0)[0]
        z = n @ w["head"].T
        R = self.ROWS
        (loss, _), (dz, _) = ref.distill(z, lists["top_ids"], lists["top_logprobs"][0], self.T, True, np.full(R, 1.0 / R))
        (dn, _), (d_head, _), _ = ref.linear_grad(n, w["head"], dz, None, 0, 0, 0, 0, 0)
        (da, _), (d_gain, _), _ = ref.norm_grad(a, dn, w["gain"], 1e-5, 0)
        (dt, _), (d_up, _), (d_b_up, _) = ref.linear_grad(t, w["up"], da, None, 0, 0, 0, 0, 0)
        _, (d_down, _), (d_b_down, _) = ref.linear_grad(hb, w["down"], dt, pre, 1, 0, 0, 0, 0)
        return dict(loss=loss, d_head=d_head, d_gain=d_gain, d_up=d_up, d_b_up=d_b_up, d_down=d_down, d_b_down=d_b_down, z=z, ids=lists["top_ids"], lps=lists["top_logprobs"][0])


GRADS = ("d_head", "d_gain", "d_up", "d_b_up", "d_down", "d_b_down")


def test_training_step():
    s = Step(3)
    s.run()
    got, want = s.results(), s.reference()
    s.ws.check()
    assert (got["ids"] == want["ids"]).all()
    assert np.allclose(got["lps"], want["lps"], atol=ref.SUM * 2)
    # Between the operators values are rounded to bf16: t, n and z on the way there, dz and da (and dt) on the way back, each by 2^-8 of itself at most.  Every gradient
    # is linear in what comes from behind; six of these roundings reach the last one, and z's moves q by as much as z is off (|z| 2^-8 in a logit of which softmax takes the difference).
    zoff = 2.0 ** -8 * np.abs(want["z"]).max()
    assert np.abs(got["loss"] - want["loss"]).max() < 2 * zoff + 0.05
    for k in GRADS:
        off = np.linalg.norm(got[k] - want[k]) / np.linalg.norm(want[k])
        assert off < 6 * 2.0 ** -8 + 2 * zoff, f"{k}: {off}"


def test_training_step_reference_agrees_with_differences():
    s = Step(3)
    want, rng = s.reference(), np.random.default_rng(0)
    for k in GRADS:
        move = rng.standard_normal(want[k].shape)
        h = 1e-6
        d = (s.reference({k[2:]: h * move})["loss"].mean() - s.reference({k[2:]: -h * move})["loss"].mean()) / (2 * h)
        assert abs(d - (want[k] * move).sum()) < 1e-6 * max(1, abs(d)), k


def test_training_steps_captured_and_replayed():
    """Two captured steps that share one workspace, replayed in turn with eager steps between, on inputs that change from replay to replay: the bits of the eager results."""
    h = hip()
    A, B, eager = Step(3), Step(4), Step(3)
    B.ws = A.ws
    eager.run()
    want_a = eager.results()
    eager_b = Step(4)
    eager_b.run()
    want_b = eager_b.results()
    other = Step(5)
    s = ctypes.c_void_p()
    ok(h.hipStreamCreate(ctypes.byref(s)))
    ok(h.hipDeviceSynchronize())
    execs = []
    for step in (A, B):
        graph, ex = ctypes.c_void_p(), ctypes.c_void_p()
        ok(h.hipStreamBeginCapture(s, 0))
        step.run(s.value)
        ok(h.hipStreamEndCapture(s, ctypes.byref(graph)))
        ok(h.hipGraphInstantiate(ctypes.byref(ex), graph, None, None, ctypes.c_size_t(0)))
        execs.append((graph, ex))
    for rep in range(4):
        if rep == 2:                                            # A's inputs become another step's
            A.target.dev.write(other.target.host)
            A.h.dev.write(other.h.host)
            A.hb.dev.write(other.hb.host)
            for x in (eager,):
                x.target.dev.write(other.target.host)
                x.h.dev.write(other.h.host)
                x.hb.dev.write(other.hb.host)
            eager.run()
            want_a = eager.results()
        for (_, ex), step, want in zip(execs, (A, B), (want_a, want_b)):
            for k in GRADS:
                x = step.e[k].dev if k in step.e else step.o[k]
                x.write(np.zeros(x.shape, np.float32) if k in step.o else step.e[k].host)
            ok(h.hipGraphLaunch(ex, s))
            ok(h.hipStreamSynchronize(s))
            got = step.results()
            for k in got:
                assert np.array_equal(got[k], want[k]), f"replay {rep}: {k}"
        eager.run()
        got = eager.results()
        assert all(np.array_equal(got[k], want_a[k]) for k in got)
    for graph, ex in execs:
        ok(h.hipGraphExecDestroy(ex))
        ok(h.hipGraphDestroy(graph))
    ok(h.hipStreamDestroy(s))


def test_results_do_not_depend_on_timing():
    s = Step(7)
    s.run()
    first = s.results()
    for _ in range(5):
        s.run()
        again = s.results()
        assert all(np.array_equal(first[k], again[k]) for k in first)


def test_infinities_and_far_arguments_of_activations():
    """The slope of an activation far out is 0 or 1, of pre = +-infinity (z beyond the type) too; an infinite dy stays infinite in every number of terms."""
    rng = np.random.default_rng(21)
    x, w = matrix(rng, 40, 16, "fp16"), matrix(rng, 24, 16, "fp16")
    dyv = rng.standard_normal((40, 24))
    prev = rng.standard_normal((40, 24))
    prev[3, 5], prev[4, 6], prev[5, 7], prev[6, 8] = np.inf, -np.inf, 6e4, -6e4
    for out in ("fp16", "fp32"):
        for act in (ee.ACT_SILU, ee.ACT_GELU):
            dy, pre, dx, dw = Rows(dyv, "fp16"), Rows(prev, "fp16"), empty(40, 16, out), empty(24, 16, out)
            ws = Space(ee.ee_linear_grad_workspace(x.view, w.view, act=act))
            ee.ee_linear_grad(x.view, w.view, dy.view, pre=pre.view, act=act, dx=dx.view, d_weight=dw.view, workspace=ws.view)
            limit = np.where(np.abs(prev) > 1e3, np.copysign(100, prev), pre.values())
            step = 2.0 ** -22 if out == "fp32" else HALF_STEP["fp16"]
            want = ref.linear_grad(x.values(), w.values(), dy.values(), limit, act, HALF_STEP[out], HALF_STEP[out], step, step)
            small = 2.0 ** -25
            close(dx.result(), (want[0][0], want[0][1] + SUBNORMAL[out] + small * np.abs(w.values()).sum(0)), "dx")
            close(dw.result(), (want[1][0], want[1][1] + SUBNORMAL[out] + small * np.abs(x.values()).sum(0)), "d_weight")
    for kind in ("bf16", "fp16"):
        x, w = matrix(rng, 4, 8, kind), matrix(rng, 8, 8, kind)
        w = Rows(np.eye(8) * 2, kind)
        dyv = rng.standard_normal((4, 8))
        dyv[1, 3] = np.inf
        dx = empty(4, 8, "fp32")
        ws = Space(ee.ee_linear_grad_workspace(x.view, w.view, act=ee.ACT_SILU))
        ee.ee_linear_grad(x.view, w.view, Rows(dyv, kind).view, pre=Rows(np.full((4, 8), 2.0), kind).view, act=ee.ACT_SILU, dx=dx.view, workspace=ws.view)
        got = dx.result()
        assert got[1, 3] == np.inf and np.isfinite(got[[0, 2, 3]]).all()
