"""ee_linear and ee_linear_grad by every tile that a product may be taken in, whole and in parts of the sum, in one and in several terms, against 64-bit forms."""
import ctypes

import numpy as np
import pytest

import paper_2505_21594_amd as ee
from tests import head_ref as ref
from tests.device import HALF_STEP, Dev, decode, encode, hip, ok
from tests.test_gpu_head_operators import SUBNORMAL, Large, Space, close, empty, up8
from tests.test_linear_plans import CASES

pytestmark = pytest.mark.gpu

U = ref.U


class Kinds:
    """[rows][width] whose element depends on the row's and the column's kind alone, so that the 64-bit form is quick; NaN behind the rows' ends."""

    def __init__(self, rng, row_kinds, column_kinds, kind, scale=1.0):
        small = encode((scale * rng.standard_normal((37, 37))).astype(np.float32), kind)
        rows, width = len(row_kinds), len(column_kinds)
        wide = np.full((rows, up8(width) + 8), encode(np.full(1, np.nan, np.float32), kind)[0])
        wide[:, :width] = small[np.ix_(row_kinds, column_kinds)]
        self.dev, self.small = Dev(wide), decode(small)
        self.view = self.dev.view((rows, width), (up8(width) + 8, 1))


class Layer:
    def __init__(self, rows, n_in, n_out, kind):
        rng = np.random.default_rng(rows + n_in + n_out)
        self.kind, self.rows, self.n_in, self.n_out = kind, rows, n_in, n_out
        self.x, self.w = Large(rng, rows, n_in, kind), Large(rng, n_out, n_in, kind, 0.2)
        self.bias = np.float32(rng.standard_normal(n_out))
        self.dy, self.pre = (Kinds(rng, self.x.index, self.w.index, kind, s) for s in (1.0, 1.5))
        self.bias_dev = Dev(self.bias)

    def forward(self, out, ws, stream=0):
        y, pre = empty(self.rows, self.n_out, out, up8(self.n_out)), empty(self.rows, self.n_out, self.kind, up8(self.n_out))
        ee.ee_linear(self.x.view, self.w.view, y.view, bias=self.bias_dev, act=ee.ACT_SILU, pre=pre.view, workspace=ws.view, stream=stream)
        return y, pre

    def check_forward(self, out):
        ws = Space(ee.ee_linear_workspace(self.x.view, self.w.view))
        y, pre = self.forward(out, ws)
        xv, wv, xi, wi, kind = self.x.values(), self.w.values(), self.x.index, self.w.index, self.kind
        z = (xv @ wv.T)[np.ix_(xi, wi)] + self.bias
        tol = (self.n_in + 2) * U * (np.abs(xv) @ np.abs(wv).T)[np.ix_(xi, wi)] + 2 * U * np.abs(z)
        value = ref.act(z, 1)
        close(y.result(), (value, 1.13 * tol + ref.ACT * (np.abs(z) + np.abs(value)) + HALF_STEP[out] * np.abs(value) * (1 + 2.0 ** -8) + SUBNORMAL[out]), "y")
        close(pre.result(), (z, tol + HALF_STEP[kind] * np.abs(z) * (1 + 2.0 ** -8) + SUBNORMAL[kind]), "pre")
        ws.check()

    def backward(self, act, out_x, out_w, ws, stream=0):
        dx, dw, db = empty(self.rows, self.n_in, out_x, up8(self.n_in)), empty(self.n_out, self.n_in, out_w, up8(self.n_in)), Dev(np.zeros(self.n_out, np.float32))
        ee.ee_linear_grad(self.x.view, self.w.view, self.dy.view, pre=self.pre.view if act else None, act=act, dx=dx.view, d_weight=dw.view, d_bias=db, workspace=ws.view, stream=stream)
        return dx, dw, db

    def check_backward(self, act, out_x, out_w):
        ws = Space(ee.ee_linear_grad_workspace(self.x.view, self.w.view, act=act))
        dx, dw, db = self.backward(act, out_x, out_w, ws)
        xv, wv, xi, wi, kind = self.x.values(), self.w.values(), self.x.index, self.w.index, self.kind
        nx, nw = (np.bincount(i, minlength=37).astype(float) for i in (xi, wi))
        dz = self.dy.small * (ref.slope(self.pre.small, act) if act else 1.0)
        off = ref.ACT * np.abs(self.dy.small) * (1 + np.abs(self.pre.small)) if act else 0 * dz
        # dz is rounded once for 16-bit results; to 2^-24 (three terms of bf16), 2^-22 or 2^-36 (two of fp16) for fp32
        exact = (2.0 ** -22, 2.0 ** -36) if kind == "fp16" else (2.0 ** -24, 0.0)
        coarse = (HALF_STEP[kind], SUBNORMAL[kind])
        n = 3 if act else 1                                      # terms that a result may be summed in

        def tolerance(want, size, off_size, all_of_it, out, K):
            step, small = (exact if out == "fp32" else coarse) if act else (0.0, 0.0)
            return (n * (K + 2) * U + step) * size + off_size + small * all_of_it + HALF_STEP[out] * np.abs(want) * (1 + 2.0 ** -8) + SUBNORMAL[out]

        want = (dz * nw) @ wv
        tol = tolerance(want, (np.abs(dz) * nw) @ np.abs(wv), (off * nw) @ np.abs(wv), nw @ np.abs(wv), out_x, self.n_out)
        close(dx.result(), (want[xi], tol[xi]), f"dx, activation {act}, {out_x}")
        want = (dz.T * nx) @ xv
        tol = tolerance(want, (np.abs(dz).T * nx) @ np.abs(xv), (off.T * nx) @ np.abs(xv), nx @ np.abs(xv), out_w, self.rows)
        close(dw.result(), (want[wi], tol[wi]), f"d_weight, activation {act}, {out_w}")
        close(db.numpy().astype(np.float64), ((dz.T @ nx)[wi], (self.rows * U * (np.abs(dz).T @ nx) + off.T @ nx)[wi]), "d_bias")
        ws.check()


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("sizes", [sizes for sizes, _ in CASES])
def test_every_tile(sizes, kind):
    layer = Layer(*sizes, kind)
    layer.check_forward("fp32")
    layer.check_forward(kind)
    for act, out_x, out_w in ((ee.ACT_NONE, "fp32", kind), (ee.ACT_SILU, "fp32", "fp32"), (ee.ACT_GELU, kind, kind), (ee.ACT_SILU, kind, "fp32")):
        layer.check_backward(act, out_x, out_w)


def test_large_tiles_captured_and_replayed():
    """The tiles whose LDS a launch has to ask for, in a graph: the bits of the eager results, replay after replay with eager work between."""
    h, s = hip(), ctypes.c_void_p()
    layer = Layer(1501, 2050, 8011, "fp16")
    assert ee.ee_debug_linear_plan(1501, 2050, 8011, 2)[:2] == (256, 128) and ee.ee_debug_linear_plan(1501, 2050, 8011, 0)[:2] == (192, 128)
    ws = Space(max(ee.ee_linear_workspace(layer.x.view, layer.w.view), ee.ee_linear_grad_workspace(layer.x.view, layer.w.view, act=ee.ACT_SILU)))
    ok(h.hipStreamCreate(ctypes.byref(s)))
    ok(h.hipDeviceSynchronize())
    graph, ex = ctypes.c_void_p(), ctypes.c_void_p()
    y, pre = empty(layer.rows, layer.n_out, "fp16", up8(layer.n_out)), empty(layer.rows, layer.n_out, "fp16", up8(layer.n_out))
    dx, dw, db = empty(layer.rows, layer.n_in, "fp32", up8(layer.n_in)), empty(layer.n_out, layer.n_in, "fp32", up8(layer.n_in)), Dev(np.zeros(layer.n_out, np.float32))
    ok(h.hipStreamBeginCapture(s, 0))
    ee.ee_linear(layer.x.view, layer.w.view, y.view, bias=layer.bias_dev, act=ee.ACT_SILU, pre=pre.view, workspace=ws.view, stream=s.value)
    ee.ee_linear_grad(layer.x.view, layer.w.view, layer.dy.view, pre=pre.view, act=ee.ACT_SILU, dx=dx.view, d_weight=dw.view, d_bias=db, workspace=ws.view, stream=s.value)
    ok(h.hipStreamEndCapture(s, ctypes.byref(graph)))
    ok(h.hipGraphInstantiate(ctypes.byref(ex), graph, None, None, ctypes.c_size_t(0)))
    want = None
    for replay in range(3):
        for r in (y, pre, dx, dw):
            r.dev.write(r.host)
        ok(h.hipGraphLaunch(ex, s))
        ok(h.hipStreamSynchronize(s))
        got = [r.result() for r in (y, pre, dx, dw)] + [db.numpy()]
        eager_y, eager_pre = layer.forward("fp16", ws)
        layer.pre.view, keep = eager_pre.view, layer.pre.view
        eager = [r.result() for r in (eager_y, eager_pre)]
        gx, gw, gb = layer.backward(ee.ACT_SILU, "fp32", "fp32", ws)
        eager += [gx.result(), gw.result(), gb.numpy()]
        layer.pre.view = keep
        for a, b in zip(got, eager):
            assert np.array_equal(a, b), f"replay {replay}"
        assert want is None or all(np.array_equal(a, b) for a, b in zip(got, want))
        want = got
    ws.check()
    ok(h.hipGraphExecDestroy(ex))
    ok(h.hipGraphDestroy(graph))
    ok(h.hipStreamDestroy(s))
