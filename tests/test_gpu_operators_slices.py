"""A slice of a batch: rows in front of row_start[0] belong to no sequence of the call and stay as they are."""
import numpy as np
import pytest

import paper_2505_21594_amd as ee
from tests import operators_ref as ref
from tests.device import Dev, bf16_values, decode, encode, hip
from tests.test_gpu_operators import cache_of, close, drafted, rope_table, run_attend

pytestmark = pytest.mark.gpu

SLICES = [
    # rows in front, rows, lens, heads, kv_heads, dim, terms, kind, out, groups, shared pages
    (1, [1], [1], 4, 4, 64, 1, "bf16", "bf16", (), ()),                                       # one part
    (3, [1], [1999], 4, 1, 128, 1, "bf16", "bf16", (), ()),                                   # parts of a single row
    (17, [5, 2], [900, 700], 4, 4, 64, 2, "fp32", "fp32", (), ()),
    (40, [200], [1500], 4, 4, 128, 1, "bf16", "fp16", (), ()),                                # parts of many rows
    (5, [2, 0, 2], [3000, 40, 2050], 4, 2, 128, 1, "bf16", "fp32", [(0, 3)], [2]),
    (9, [2, 2], [3000, 2050], 4, 2, 128, 1, "fp16", "fp16", [(0, 2)], [120]),                 # parts of common pages
    (2, [1] * 80, [600 + i for i in range(80)], 2, 2, 64, 1, "bf16", "bf16", [(0, 40), (40, 80)], [30, 20]),   # more members than lanes
]


@pytest.mark.parametrize("i", range(len(SLICES)))
def test_attend_leaves_rows_in_front(i):
    """The workspace comes filled with bytes that make no sense as counts of parts."""
    front, rows, lens, heads, kv_heads, dim, terms, kind, out_kind, groups, shared = SLICES[i]
    c = ref.Case(800 + i, rows, lens, kv_heads, dim, terms, groups, shared, pad=i % 3).fill_fast()
    c.row_start = c.row_start + np.int32(front)
    c.T, c.cap = c.T + front, c.cap + front
    got, want, tol = run_attend(c, heads, kind, out_kind)
    close(got[front:], want[front:], tol[front:], "attention")
    assert (got[:front] == 7.5).all(), "rows in front of the first sequence's were written"


def test_append_leaves_rows_in_front():
    front, rows, lens, heads, kv_heads, dim = 6, [3, 20], [40, 33], 4, 2, 64
    c = ref.Case(820, rows, lens, kv_heads, dim, 1).fill()
    T = sum(rows)
    x = c.rng.standard_normal((front + T, heads + 2 * kv_heads, dim)).astype(np.float32)
    q, k, v = (np.ascontiguousarray(x[:, a:b]) for a, b in ((0, heads), (heads, heads + kv_heads), (heads + kv_heads, heads + 2 * kv_heads)))
    q[:front], k[:front], v[:front] = np.nan, np.nan, np.nan
    kp, vp, table = cache_of(c)
    rope = rope_table(64, dim)
    out, keep = Dev(np.full((front + T, heads, dim), 7.5, np.float32)), [Dev(a) for a in (c.row_start + np.int32(front), c.kv_len, q, k, v, rope)]
    ee.ee_kv_append(ee.PagedCache(kp, vp, table), keep[0], keep[1], keep[2], keep[3], keep[4], out, rope=keep[5])
    got = out.numpy()
    want, tol, places = ref.append(c, q[front:], k[front:], v[front:], None, None, 1e-5, rope, False, "fp32")
    assert (got[:front] == 7.5).all()
    close(got[front:].astype(np.float64), want, tol, "q_out")
    values = bf16_values(kp.numpy()).astype(np.float64).sum(3)
    for (page, slot), (wk, tk, _) in places.items():
        close(values[page, :, slot], wk, tk, "key")
    rest = np.ones(kp.shape[:3], bool)
    for page, slot in places:
        rest[page, :, slot] = False
    assert (kp.numpy()[rest] == c.k_pool[rest]).all()


def test_accept_of_a_slice():
    """Two of a batch's four sequences, over the whole batch's rows."""
    rng = np.random.default_rng(30)
    rows, V = [4, 3, 5, 2], 5000
    z, p, x, u, v = drafted(rng, sum(rows), V)
    temp = (0.5 + rng.random(4)).astype(np.float32)
    rs = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    z[: rs[1]], z[rs[3]:] = np.nan, np.inf
    d = [Dev(a) for a in (z, rs[1:4].copy(), x, p, u, v, temp[1:3].copy())]
    acc, tok = Dev(np.full(2, -9, np.int32)), Dev(np.full(2, -9, np.int32))
    n = ee.ee_accept_workspace(d[0], d[1])
    ee.ee_accept_drafts(*d[:2], d[2], d[3], d[4], d[5], d[6], acc, tok, workspace=Dev(np.full(n, 0x5A, np.uint8)))
    wa, wt, margin = ref.accept(rs[1:4], z.astype(np.float64), x, p, u, v, temp[1:3])
    assert margin > 1e-11 and (acc.numpy() == wa).all() and (tok.numpy() == wt).all()


def test_slices_of_one_batch_in_turn():
    """A batch attended to in two calls over the same queries, results and workspace, the second slice last: both calls' rows are there."""
    rows, lens, heads, kv_heads, dim = [3, 2, 4], [700, 1300, 900], 4, 2, 64
    c = ref.Case(821, rows, lens, kv_heads, dim, 1).fill_fast()
    q = c.rng.standard_normal((c.T, heads, dim)).astype(np.float32)
    enc = encode(q, "bf16")
    kp, vp, table = cache_of(c)
    dq, out = Dev(enc), Dev(np.full(q.shape, 7.5, np.float32))
    keep, ws = [], None
    for lo, hi in ((0, 1), (1, 3)):
        cache = ee.PagedCache(kp, vp, Dev(np.ascontiguousarray(c.table[lo:hi])))
        rs, kl = Dev(c.row_start[lo: hi + 1].copy()), Dev(c.kv_len[lo:hi].copy())
        keep += [cache, rs, kl]
        if ws is None:
            ws = Dev(np.full(1 << 22, 0x5A, np.uint8))
        assert ee.ee_attend_workspace(cache, rs, dq, max_kv=max(lens)) <= 1 << 22
        ee.ee_attend(cache, rs, kl, dq, out, scale=dim ** -0.5, max_kv=max(lens), workspace=ws)
    want, tol = ref.attend(c, decode(enc), dim ** -0.5, "bf16", "fp32")
    close(out.numpy().astype(np.float64), want, tol, "two slices")
    hip().hipDeviceSynchronize()
