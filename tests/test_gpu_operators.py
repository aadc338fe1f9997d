"""The operators on device memory against plain 64-bit forms: ee_kv_append, ee_attend, ee_accept_drafts."""
import copy
import ctypes

import numpy as np
import pytest

import paper_2505_21594_amd as ee
from tests import operators_ref as ref
from tests.device import Dev, HALF_STEP, bf16_values, decode, encode, hip, ok

pytestmark = pytest.mark.gpu

GUARD = 0x5A


def cache_of(c):
    return c.far if hasattr(c, "far") else (Dev(c.k_pool), Dev(c.v_pool), Dev(c.table))


class Far:
    """A pool of n pages in device memory of which the last ones are `pages`."""

    def __init__(self, pages, n):
        self.shape, self.dtype = (n,) + pages.shape[1:], "bfloat16"
        self._last = Dev(pages[:1])                              # (its device)
        self.device, self._count, self._page = self._last.device, len(pages), pages[0].nbytes
        self._p = ctypes.c_void_p()
        ok(hip().hipMalloc(ctypes.byref(self._p), n * self._page))
        ok(hip().hipMemcpy(self._p.value + (n - self._count) * self._page, pages.ctypes.data, pages.nbytes, 1))

    def data_ptr(self):
        return self._p.value

    def stride(self):
        return tuple(int(np.prod(self.shape[i + 1:])) for i in range(5))

    def pages(self):
        out = np.empty((self._count,) + self.shape[1:], np.uint16)
        ok(hip().hipDeviceSynchronize())
        ok(hip().hipMemcpy(out.ctypes.data, self._p.value + (self.shape[0] - self._count) * self._page, out.nbytes, 2))
        return out

    def __del__(self):
        hip().hipFree(self._p)


def workspace(n):
    """With a guard behind it, so that writes past its end show."""
    return Dev(np.full(n + 256, GUARD, np.uint8))


def rope_table(n, dim, base=10000.0):
    angle = np.arange(n)[:, None] * base ** (-np.arange(0, dim, 2) / dim)
    return np.stack([np.cos(angle), np.sin(angle)], -1).astype(np.float32)


def close(got, want, tol, what):
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, e.g. {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]} +- {tol[bad][0]}"


# ---------------------------------------------------------------- ee_attend

def run_attend(c, heads, kind, out_kind, groups=True, scale=None, layout="plain", max_kv=None, hint_shared=None, stream=0, weight_step=0.0):
    """weight_step: how far one term of a softmax weight may be off, relative to it, where that is more than the tolerance of ref.attend has."""
    q = np.zeros((c.cap, heads, c.dim), np.float32)
    q[:] = c.rng.standard_normal(q.shape)
    enc = encode(q, kind)
    if c.cap > c.T:
        enc[c.T:] = encode(np.full((1,), np.nan, np.float32), kind)[0]
    fill = encode(np.full((1,), 7.5, np.float32), out_kind)[0]
    if layout == "plain":
        dq, base = Dev(enc), np.full((c.cap, heads, c.dim), fill)
        dout = Dev(base)
        vq, vout = dq, dout
    else:   # rows and heads apart, heads outermost
        wide = np.zeros((heads, c.cap, c.dim + 16), enc.dtype)
        wide[:, :, : c.dim] = enc.transpose(1, 0, 2)
        dq = Dev(wide)
        vq = dq.view((c.cap, heads, c.dim), (c.dim + 16, c.cap * (c.dim + 16), 1))
        base = np.full((c.cap, heads + 3, c.dim), fill)
        dout = Dev(base)
        vout = dout.view((c.cap, heads, c.dim), ((heads + 3) * c.dim, c.dim, 1), c.dim)
    k, v, table = cache_of(c)
    cache = ee.PagedCache(k, v, table)
    rs, kl = Dev(c.row_start), Dev(c.kv_len)
    g = {}
    if groups and c.group_start is not None:
        g = dict(group_start=Dev(c.group_start), group_pages=Dev(c.group_pages), max_shared=int(max(c.group_pages)) * 16 if hint_shared is None else hint_shared)
    max_kv = max(list(c.lens) + [1]) if max_kv is None else max_kv
    n = ee.ee_attend_workspace(cache, rs, vq, max_kv=max_kv, **g)
    ws = workspace(n)
    scale = c.dim ** -0.5 if scale is None else scale
    ee.ee_attend(cache, rs, kl, vq, vout, scale=scale, max_kv=max_kv, workspace=ws.view((n,), (1,)), stream=stream, **g)
    out = dout.numpy()
    assert (ws.numpy()[n:] == GUARD).all()
    if layout != "plain":
        assert (out[:, 0] == fill).all() and (out[:, heads + 1:] == fill).all()
        out = out[:, 1: heads + 1]
    assert (out[c.T:] == fill).all(), "padding rows were written"
    want, tol = ref.attend(c, decode(enc)[: c.T], scale, kind, out_kind)
    if weight_step:
        magnitudes = copy.copy(c)
        magnitudes.values = lambda s: np.abs(c.values(s))
        tol = tol + weight_step * ref.attend(magnitudes, decode(enc)[: c.T], scale, kind, out_kind)[0]
    return decode(out)[: c.T], want, tol


ATTEND = [
    # rows, lens, heads, kv_heads, dim, terms, kind, out
    ([1], [1], 4, 4, 64, 1, "bf16", "bf16"),
    ([5], [69], 4, 4, 64, 2, "fp32", "fp32"),
    ([1], [17], 2, 2, 128, 1, "bf16", "bf16"),
    ([3], [16], 3, 1, 128, 1, "fp16", "fp16"),
    ([1, 4, 2], [33, 64, 5], 8, 2, 128, 1, "bf16", "fp32"),
    ([17, 1, 0, 5], [40, 300, 12, 5], 6, 2, 64, 1, "fp32", "fp32"),
    ([2, 0, 3], [0, 0, 2], 4, 2, 64, 2, "fp32", "bf16"),           # rows in front of position 0
    ([70], [131], 3, 3, 128, 2, "fp32", "fp32"),
    ([33], [500], 5, 1, 64, 2, "bf16", "fp32"),
    ([1], [1999], 4, 1, 128, 1, "bf16", "bf16"),
    ([9] * 5, [100, 9, 400, 33, 1000], 32, 32, 64, 1, "fp16", "bf16"),
    ([1] * 70, list(range(1, 141, 2)), 2, 1, 64, 1, "bf16", "fp32"),  # more sequences than lanes
    ([3], [50], 40, 1, 64, 1, "bf16", "fp32"),                     # 40 query heads on one key head
]


@pytest.mark.parametrize("layout", ["plain", "strided"])
@pytest.mark.parametrize("i", range(len(ATTEND)))
def test_attend(i, layout):
    rows, lens, heads, kv_heads, dim, terms, kind, out_kind = ATTEND[i]
    c = ref.Case(100 + i, rows, lens, kv_heads, dim, terms, pad=i % 3).fill_fast()
    got, want, tol = run_attend(c, heads, kind, out_kind, layout=layout)
    close(got, want, tol, "attention")


MANY = [
    # rows, lens, heads, kv_heads, dim, terms, kind, out, groups, shared pages: more than 32 lines of a key head a sequence
    ([33], [33], 1, 1, 64, 1, "bf16", "bf16", (), ()),
    ([128], [128], 4, 4, 64, 1, "bf16", "bf16", (), ()),
    ([200], [1500], 4, 4, 128, 1, "bf16", "bf16", (), ()),                 # parts
    ([300], [120], 2, 2, 64, 1, "bf16", "bf16", (), ()),                   # rows in front of position 0
    ([65, 0, 100, 3], [65, 10, 900, 400], 8, 2, 128, 1, "bf16", "fp16", (), ()),
    ([40, 30], [300, 31], 2, 1, 64, 1, "fp16", "fp16", (), ()),
    ([129], [2049], 2, 2, 128, 1, "fp16", "fp32", (), ()),
    ([40] * 3, [100, 500, 3001], 4, 4, 128, 1, "fp32", "fp32", (), ()),
    ([50, 1], [1600, 1700], 3, 1, 64, 1, "bf16", "fp32", (), ()),
    ([150], [150], 2, 2, 64, 2, "fp32", "fp32", (), ()),
    ([70, 70, 70], [2000, 71, 500], 2, 2, 128, 2, "fp32", "bf16", (), ()),
    ([66, 70, 1], [300, 290, 220], 4, 4, 128, 1, "bf16", "bf16", [(0, 3)], [13]),
    ([90, 66], [700, 90], 2, 2, 64, 2, "fp32", "fp32", [(0, 2)], [1]),
    ([40] * 66, [40 + 7 * i for i in range(66)], 1, 1, 64, 1, "bf16", "fp32", (), ()),      # more sequences than lanes
]


@pytest.mark.parametrize("layout", ["plain", "strided"])
@pytest.mark.parametrize("i", range(len(MANY)))
def test_attend_many_rows(i, layout):
    """For bf16 queries and results of one-term caches a weight is one bf16 term, off by half a step: 2^-8 of it."""
    rows, lens, heads, kv_heads, dim, terms, kind, out_kind, groups, shared = MANY[i]
    c = ref.Case(600 + i, rows, lens, kv_heads, dim, terms, groups, shared, pad=i % 3).fill_fast()
    got, want, tol = run_attend(c, heads, kind, out_kind, layout=layout, weight_step=2.0 ** -8 if (kind, out_kind, terms) == ("bf16", "bf16", 1) else 0)
    close(got, want, tol, "many rows")


GROUPS = [
    # rows, lens, groups, shared pages, heads, kv_heads, dim, terms, kind
    ([5] * 8, [100 + 7 * i for i in range(8)], [(0, 8)], [5], 4, 4, 128, 2, "fp32"),
    ([1, 2, 3, 1, 1], [70, 80, 90, 200, 33], [(0, 3), (3, 5)], [4, 1], 8, 2, 128, 1, "bf16"),
    ([1, 2, 3, 1, 1], [70, 80, 90, 200, 33], [(1, 3)], [4], 6, 2, 64, 1, "fp16"),              # some sequences in no group
    ([4, 0, 20, 1], [64, 64, 84, 65], [(0, 4)], [4], 4, 1, 64, 1, "fp32"),                     # the common pages end among new rows
    ([1] * 80, [48 + i for i in range(80)], [(0, 40), (40, 80)], [3, 2], 2, 2, 64, 1, "bf16"),  # more members than lanes
    ([2, 2], [3000, 2050], [(0, 2)], [120], 4, 2, 128, 1, "bf16"),
    ([2, 2], [40, 40], [(0, 2)], [0], 4, 2, 128, 1, "bf16"),
    ([0, 0, 3], [32, 32, 50], [(0, 2), (2, 3)], [2, 3], 4, 2, 128, 2, "fp32"),                  # a group without rows, one of one
    ([1] * 140, [50 + i % 30 for i in range(140)], [(2 * i, 2 * i + 2) for i in range(70)], [2] * 70, 2, 1, 64, 1, "bf16"),   # more groups than lanes
]


@pytest.mark.parametrize("i", range(len(GROUPS)))
def test_attend_shared(i):
    rows, lens, groups, shared, heads, kv_heads, dim, terms, kind = GROUPS[i]
    c = ref.Case(200 + i, rows, lens, kv_heads, dim, terms, groups, shared, pad=i % 2).fill_fast()
    got, want, tol = run_attend(c, heads, kind, "fp32")
    close(got, want, tol, "shared")
    c.rng = np.random.default_rng(5)
    got, want, tol = run_attend(c, heads, kind, "fp32", hint_shared=0, max_kv=0)    # nothing known about lengths
    close(got, want, tol, "shared, no bounds given")


def test_attend_bounds_too_small_change_nothing():
    """max_kv and max_shared only choose the split."""
    c = ref.Case(7, [2, 3], [700, 650], 2, 64, 1, [(0, 2)], [30]).fill_fast()
    got, want, tol = run_attend(c, 4, "bf16", "fp32", max_kv=20, hint_shared=16)
    close(got, want, tol, "attention")


def test_attend_bad_pages_and_lengths():
    """Entries outside the pools hold nothing; lengths beyond the table end with it."""
    c = ref.Case(8, [2, 1, 3], [90, 40, 60], 2, 64, 1, table_extra=0).fill_fast()
    c.table[0, 1], c.table[0, 3], c.table[1, :3] = -1, c.n_pages, [-5, 2 ** 31 - 1, -2 ** 31]
    got, want, tol = run_attend(c, 4, "bf16", "fp32")
    close(got, want, tol, "bad pages")
    assert (got[2] == 0).all(), "a row without any page gets zeros"
    c = ref.Case(9, [2], [96], 2, 64, 1, table_extra=0).fill_fast()
    c.kv_len[0] = 96 + 50                                        # 50 positions more than the table has
    c.lens = [96]
    k, v, table = cache_of(c)
    q = c.rng.standard_normal((2, 4, 64)).astype(np.float32)
    dq, dout = Dev(q), Dev(np.zeros_like(q))
    cache, rs, kl = ee.PagedCache(k, v, table), Dev(c.row_start), Dev(c.kv_len)
    n = ee.ee_attend_workspace(cache, rs, dq)
    ee.ee_attend(cache, rs, kl, dq, dout, scale=0.125, workspace=workspace(n))
    c.rows, c.row_start = [2], c.row_start
    K, V = c.keys(0)[0], c.values(0)
    for i in range(2):
        for h in range(4):
            e = np.exp(K[:, h // 2] @ q[i, h] * 0.125)
            assert np.abs(dout.numpy()[i, h] - e @ V[:, h // 2] / e.sum()).max() < 1e-4    # (all 96 positions for both rows)


@pytest.mark.parametrize("terms", [1, 2])
@pytest.mark.parametrize("dim", [64, 128])
def test_attend_nan_where_a_row_does_not_look(dim, terms):
    """NaN and infinities in later rows' keys and values leave the rows in front of them as they are."""
    rows, lens = [6, 1, 20], [21, 16, 40]
    c = ref.Case(11, rows, lens, 2, dim, terms).fill_fast()
    clean = ref.Case(11, rows, lens, 2, dim, terms).fill_fast()
    for s, p, bits in ((0, 18, 0x7F80), (0, 20, 0x7FC0), (2, 30, 0xFF80)):
        page, slot = c.table[s, p // 16], p % 16
        c.k_pool[page, :, slot] = 0x7FC0
        c.v_pool[page, :, :, 5:9, slot] = bits
    q_seed = 3
    c.rng, clean.rng = np.random.default_rng(q_seed), np.random.default_rng(q_seed)
    got, _, _ = run_attend(c, 4, "fp32", "fp32")
    _, want, tol = run_attend(clean, 4, "fp32", "fp32")
    blind = np.ones(27, bool)           # rows that see none of them
    blind[[3, 4, 5]] = False            # positions 18..20 of sequence 0 (its rows are 15..20)
    blind[7 + 10:] = False              # positions 30..39 of sequence 2 (rows 20..39)
    close(got[blind], want[blind], tol[blind], "rows in front")
    assert np.isnan(got[~blind]).any(axis=(1, 2)).all()


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_attend_infinite_scores(kind):
    """A row whose every score is -infinity has no softmax: NaN; a part of them is as nothing.  A query beyond bf16 is two terms, and
    0 times an infinity is NaN: there an infinite key that a row sees makes its result NaN."""
    c = ref.Case(12, [1], [600], 1, 64, 1).fill_fast()
    q = np.zeros((1, 1, 64), np.float32)
    q[0, 0, 0] = 1.0
    for upto, bad in ((592, False), (600, True)):
        for p in range(upto):
            c.k_pool[c.table[0, p // 16], 0, p % 16, 0, 0] = 0xFF80
        k, v, table = cache_of(c)
        dq, dout = Dev(encode(q, kind)), Dev(q)
        cache, rs, kl = ee.PagedCache(k, v, table), Dev(c.row_start), Dev(c.kv_len)
        n = ee.ee_attend_workspace(cache, rs, dq, max_kv=600)
        ee.ee_attend(cache, rs, kl, dq, dout, scale=0.125, max_kv=600, workspace=workspace(n))
        out = dout.numpy()
        if bad or kind == "fp32":
            assert np.isnan(out).all()
        else:
            K, V = c.keys(0)[0][upto:, 0], c.values(0)[upto:, 0]
            e = np.exp(K[:, 0] * 0.125)
            assert np.abs(out[0, 0] - e @ V / e.sum()).max() < 1e-4


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("terms", [1, 2])
@pytest.mark.parametrize("dim", [64, 128])
def test_attend_many_rows_nan_where_a_row_does_not_look(dim, terms, kind):
    c, clean = (ref.Case(14, [120, 70], [700, 75], 2, dim, terms).fill_fast() for _ in range(2))
    for s, p, bits in ((0, 640, 0x7F80), (0, 699, 0x7FC0), (1, 40, 0xFF80)):
        page, slot = c.table[s, p // 16], p % 16
        c.k_pool[page, :, slot] = 0x7FC0
        c.v_pool[page, :, :, 5:9, slot] = bits
    c.rng, clean.rng = np.random.default_rng(4), np.random.default_rng(4)
    got, _, _ = run_attend(c, 2, kind, "fp32")
    _, want, tol = run_attend(clean, 2, kind, "fp32")
    blind = np.concatenate([580 + np.arange(120) < 640, 5 + np.arange(70) < 40])
    close(got[blind], want[blind], tol[blind], "rows in front")
    assert np.isnan(got[~blind]).any(axis=(1, 2)).all()


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("terms", [1, 2])
@pytest.mark.parametrize("at", [0, 128, 256, 1023, 1024])
def test_attend_nan_score_alone_in_a_part(at, terms, kind):
    """A key of NaN makes its row NaN, also where a part of the positions, or a wave of it, has no other score above -infinity."""
    c = ref.Case(17, [1], [1025], 2, 64, terms).fill_fast()
    q = np.zeros((1, 2, 64), np.float32)
    q[0, :, 0] = 1.0
    for p in range(at // 128 * 128, 1025 if at == 1024 else at // 128 * 128 + 128):
        c.k_pool[c.table[0, p // 16], :, p % 16, :, 0] = 0xFF80 if kind == "bf16" and terms == 1 else c.k_pool[c.table[0, p // 16], :, p % 16, :, 0]
    c.k_pool[c.table[0, at // 16], :, at % 16] = 0x7FC0
    k, v, table = cache_of(c)
    dq, dout = Dev(encode(q, kind)), Dev(q)
    cache, rs, kl = ee.PagedCache(k, v, table), Dev(c.row_start), Dev(c.kv_len)
    n = ee.ee_attend_workspace(cache, rs, dq, max_kv=1025)
    ee.ee_attend(cache, rs, kl, dq, dout, scale=0.125, max_kv=1025, workspace=workspace(n))
    assert np.isnan(dout.numpy()).all()


def test_attend_many_rows_infinite_scores():
    """40 rows behind 560 positions: those that see the first 580 only have no softmax, the others have that of what is behind."""
    c = ref.Case(15, [40], [600], 1, 64, 1).fill_fast()
    q = np.zeros((40, 1, 64), np.float32)
    q[:, 0, 0] = 1.0
    for p in range(580):
        c.k_pool[c.table[0, p // 16], 0, p % 16, 0, 0] = 0xFF80
    k, v, table = cache_of(c)
    dq, dout = Dev(encode(q, "bf16")), Dev(q)
    cache, rs, kl = ee.PagedCache(k, v, table), Dev(c.row_start), Dev(c.kv_len)
    n = ee.ee_attend_workspace(cache, rs, dq, max_kv=600)
    ee.ee_attend(cache, rs, kl, dq, dout, scale=0.125, max_kv=600, workspace=workspace(n))
    out = dout.numpy()
    assert np.isnan(out[:20]).all()
    K, V = c.keys(0)[0][580:, 0], c.values(0)[580:, 0]
    for i in range(20, 40):
        e = np.exp(K[: i - 19, 0] * 0.125)
        assert np.abs(out[i, 0] - e @ V[: i - 19] / e.sum()).max() < 1e-4


def test_attend_large_scores_of_many_rows():
    c = ref.Case(16, [50], [200], 2, 64, 1).fill_fast(scale=30.0)
    got, want, tol = run_attend(c, 2, "bf16", "fp32", scale=3.0)
    assert np.isfinite(got).all()
    close(got, want, tol, "large scores")


def test_attend_large_scores():
    """Scores of thousands: the running maximum keeps exp in range."""
    c = ref.Case(13, [4], [200], 2, 64, 1).fill_fast(scale=30.0)
    got, want, tol = run_attend(c, 4, "bf16", "fp32", scale=3.0)
    assert np.isfinite(got).all()
    close(got, want, tol, "large scores")


# ---------------------------------------------------------------- ee_kv_append

def run_append(c, heads, kind, q_kind, norm, rope_len, pairs, in_place=False, fused=True, stream=0):
    Hk, dim = c.kv_heads, c.dim
    raw = 1.5 * c.rng.standard_normal((c.cap, heads + 2 * Hk, dim)).astype(np.float32)
    enc = encode(raw, kind)
    gains = [(0.5 + c.rng.random(dim)).astype(np.float32) if norm else None for _ in range(2)]
    rope = rope_table(rope_len, dim) if rope_len else None
    if fused:
        d = Dev(enc)
        w = (heads + 2 * Hk) * dim
        q, k, v = (d.view((c.cap, n, dim), (w, dim, 1), at * dim) for n, at in ((heads, 0), (Hk, heads), (Hk, heads + Hk)))
    else:
        parts = enc[:, :heads], enc[:, heads: heads + Hk], enc[:, heads + Hk:]
        keep = [Dev(np.ascontiguousarray(x.transpose(1, 0, 2))) for x in parts]     # heads outermost
        q, k, v = (x.view((c.cap, x.shape[0], dim), (dim, c.cap * dim, 1)) for x in keep)
    fill = encode(np.full((1,), 7.5, np.float32), q_kind)[0]
    out = Dev(np.full((c.cap, heads, dim), fill))
    pk, pv, table = cache_of(c)
    cache = ee.PagedCache(pk, pv, table)
    rs, kl = Dev(c.row_start), Dev(c.kv_len)
    g = [Dev(x) if x is not None else None for x in gains]
    ee.ee_kv_append(cache, rs, kl, q if heads else None, k, v, (q if in_place else out) if heads else None, q_gain=g[0], k_gain=g[1], eps=1e-5,
                    rope=Dev(rope) if rope is not None else None, rope_pairs=pairs, stream=stream)
    hip().hipDeviceSynchronize()
    x = decode(enc)
    want, tol, places = ref.append(c, x[: c.T, :heads], x[: c.T, heads: heads + Hk], x[: c.T, heads + Hk:], *gains, 1e-5, rope, pairs, q_kind)
    if heads:
        if in_place:
            now = d.numpy()
            assert (now[:, heads:] == enc[:, heads:]).all() and (now[c.T:] == enc[c.T:]).all()
            got = decode(now[: c.T, :heads])
        else:
            now = out.numpy()
            assert (now[c.T:] == fill).all(), "padding rows were written"
            got = decode(now[: c.T])
        close(got, want, tol, "q_out")
    nk, nv = pk.numpy(), pv.numpy()
    vk, vv = bf16_values(nk).astype(np.float64).sum(3), bf16_values(nv).astype(np.float64).sum(2)
    stored = 2.0 ** -8 if c.terms == 1 else 2.0 ** -16
    rest_k, rest_v = np.ones(nk.shape[:3], bool), np.ones((nk.shape[0], nk.shape[1], 16), bool)
    for (page, slot), (wk, tk, wv) in places.items():
        close(vk[page, :, slot], wk, tk, f"key at page {page} slot {slot}")
        close(vv[page, :, :, slot], wv, stored * np.abs(wv) + 2.0 ** -130, f"value at page {page} slot {slot}")
        rest_k[page, :, slot] = False
        rest_v[page, :, slot] = False
    assert (nk[rest_k] == c.k_pool[rest_k]).all(), "other places of the key pool changed"
    mask = np.broadcast_to(rest_v[:, :, None, None, :], nv.shape)
    assert (nv[mask] == c.v_pool[mask]).all(), "other places of the value pool changed"


APPEND = [
    # rows, lens, heads, kv_heads, dim, terms, kind, q kind, norm, rope_len, pairs
    ([1], [1], 4, 4, 64, 1, "bf16", "bf16", False, 32, False),
    ([1], [17], 8, 2, 128, 2, "fp32", "fp32", True, 32, True),
    ([5], [69], 4, 4, 64, 2, "fp32", "fp32", False, 128, False),
    ([16], [32], 5, 5, 128, 1, "fp16", "fp16", True, 64, False),
    ([17], [40], 6, 3, 64, 1, "bf16", "fp32", True, 64, True),
    ([1, 40, 0, 7], [100, 41, 9, 23], 9, 3, 128, 1, "bf16", "bf16", True, 128, False),
    ([33], [33], 10, 5, 64, 2, "fp16", "fp32", False, 0, False),
    ([3, 2], [20, 31], 0, 3, 128, 1, "fp32", "fp32", True, 64, False),            # keys and values only
    ([4, 3], [2, 3], 4, 2, 64, 1, "fp32", "fp32", True, 16, False),               # rows in front of position 0
    ([20], [45], 4, 2, 64, 1, "fp32", "fp32", False, 30, False),                  # rows behind the rope table
    ([1] * 70, list(range(1, 141, 2)), 3, 1, 64, 1, "bf16", "bf16", False, 256, False),
    ([200, 90], [215, 90], 6, 2, 128, 1, "fp32", "bf16", True, 256, True),
]


@pytest.mark.parametrize("fused", [True, False])
@pytest.mark.parametrize("i", range(len(APPEND)))
def test_append(i, fused):
    rows, lens, heads, kv_heads, dim, terms, kind, q_kind, norm, rope_len, pairs = APPEND[i]
    c = ref.Case(300 + i, rows, lens, kv_heads, dim, terms, pad=i % 3).fill()
    run_append(c, heads, kind, q_kind, norm, rope_len, pairs, fused=fused)


def test_append_in_place():
    c = ref.Case(320, [3, 30], [40, 31], 2, 128, 1, pad=2).fill()
    run_append(c, 6, "bf16", "bf16", True, 64, False, in_place=True)


def test_append_bad_pages():
    """Rows on entries outside the pools have no place; their queries are rotated all the same."""
    c = ref.Case(321, [20, 3], [40, 19], 2, 64, 1, table_extra=0).fill()
    c.table[0, 1], c.table[1, 1] = -3, c.n_pages + 4
    run_append(c, 4, "fp32", "fp32", True, 64, False)


@pytest.mark.parametrize("rows", [5, 70])
def test_pools_beyond_32_bits(rows):
    """Pools of 5.2 GB each, the pages in use behind 2^32 bytes and 2^31 elements."""
    n = 20000
    c = ref.Case(18, [rows, 2], [rows + 90, 40], 32, 128, 2, table_extra=0).fill_fast()
    there = c.table.copy()
    used = (there >= 0) & (there < c.n_pages)
    far = Far(np.ascontiguousarray(c.k_pool), n), Far(np.ascontiguousarray(c.v_pool), n)
    c.far = far + (Dev(np.where(used, there + n - c.n_pages, -1).astype(np.int32)),)
    got, want, tol = run_attend(c, 32, "fp32", "fp32")
    close(got, want, tol, "attention")
    k, v = c.rng.standard_normal((2, rows + 2, 32, 128)).astype(np.float32)
    rs, kl, dk, dv = Dev(c.row_start), Dev(c.kv_len), Dev(k), Dev(v)
    ee.ee_kv_append(ee.PagedCache(*c.far), rs, kl, None, dk, dv, None)
    kp, vp = c.k_pool.copy(), c.v_pool.copy()
    for s in range(2):
        for i in range(c.rows[s]):
            p = c.lens[s] - c.rows[s] + i
            page, slot, row = there[s, p // 16], p % 16, c.row_start[s] + i
            kp[page, :, slot] = ref.split(k[row], 2).transpose(1, 0, 2)
            vp[page, :, :, :, slot] = ref.split(v[row], 2).transpose(1, 0, 2)
    assert (far[0].pages() == kp).all() and (far[1].pages() == vp).all()


# ---------------------------------------------------------------- ee_accept_drafts

def run_accept(rows, logits, kind, drafts, probs, u, v, temperature, row_stride=None, stream=0, pad=0):
    rs = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    T, V = logits.shape
    enc = encode(logits, kind)
    wide = np.full((T + pad, row_stride or V), encode(np.full((1,), 1e4, np.float32), kind)[0])
    wide[:T, :V] = enc
    d = Dev(wide)
    dz = d.view((T + pad, V), (wide.shape[1], 1))
    fill = lambda a, x: Dev(np.concatenate([a, np.full(pad, x, a.dtype)]))  # noqa: E731
    dp = None
    if probs is not None:
        dp = Dev(np.concatenate([probs, np.full((pad, V), np.nan, np.float32)]))
    n = len(rows)
    acc, tok, drs = Dev(np.full(n + 2, -9, np.int32)), Dev(np.full(n + 2, -9, np.int32)), Dev(rs)
    size = ee.ee_accept_workspace(dz, drs)
    ws = workspace(size)
    ee.ee_accept_drafts(dz, drs, fill(drafts, 0), dp, None if u is None else fill(u, 0), None if v is None else fill(v, 0), Dev(temperature), acc, tok,
                        workspace=ws.view((size,), (1,)), stream=stream)
    got = acc.numpy(), tok.numpy()
    assert (ws.numpy()[size:] == GUARD).all()
    assert (got[0][n:] == -9).all() and (got[1][n:] == -9).all()
    want = ref.accept(rs, decode(enc).astype(np.float64), drafts, probs, u, v, temperature)
    return got[0][:n], got[1][:n], want


def drafted(rng, T, V, temperature=1.0, spread=0.5):
    z = 2 * rng.standard_normal((T, V))
    z[np.arange(T), rng.integers(V, size=T)] += np.log(V) + 3
    d = (z + spread * rng.standard_normal((T, V))) / temperature
    p = np.exp(d - d.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    x = np.array([rng.choice(V, p=r) for r in p], np.int32)
    return z.astype(np.float32), p.astype(np.float32), x, rng.random(T, dtype=np.float32), rng.random(T, dtype=np.float32)


@pytest.mark.parametrize("kind", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,V,stride", [([5], 1024, None), ([1], 7, None), ([2, 9, 1, 0, 16], 3001, None), ([5] * 8, 32000, 32003), ([3] * 70, 100, None), ([4, 2], 20000, None)])
def test_accept(rows, V, stride, kind):
    rng = np.random.default_rng(V + len(rows))
    z, p, x, u, v = drafted(rng, sum(rows), V)
    temp = (0.5 + rng.random(len(rows))).astype(np.float32)
    for pad in (0, 3):
        a, t, (wa, wt, margin) = run_accept(rows, z, kind, x, p, u, v, temp, row_stride=stride, pad=pad)
        assert margin > 1e-11
        assert (a == wa).all() and (t == wt).all()


def test_accept_greedy_and_mixed_temperatures():
    rng = np.random.default_rng(4)
    rows = [6, 6, 6, 6]
    z, p, x, u, v = drafted(rng, 24, 5000)
    z[3] = 1.0                                                       # ties: the lowest token
    z[9, [70, 4000]] = 50.0
    x[:] = z.argmax(1)
    x[4], x[14] = 17, -1
    temp = np.array([0.0, 0.0, 0.7, 0.0], np.float32)
    a, t, (wa, wt, _) = run_accept(rows, z, "fp32", x, p, u, v, temp)
    assert (a == wa).all() and (t == wt).all()
    a, t, (wa, wt, _) = run_accept(rows, z, "bf16", x, None, None, None, np.zeros(4, np.float32))
    assert (a == wa).all() and (t == wt).all()


def test_accept_certain_drafts():
    """No draft probabilities: p is 1 for the draft; what the row emits instead is never the draft."""
    rng = np.random.default_rng(5)
    rows = [4] * 12
    z, _, x, u, v = drafted(rng, 48, 700)
    a, t, (wa, wt, margin) = run_accept(rows, z, "fp32", x, None, u, v, np.ones(12, np.float32))
    assert margin > 1e-11 and (a == wa).all() and (t == wt).all() and (a < 3).any()


def test_accept_special_rows():
    rng = np.random.default_rng(6)
    V = 2500
    rows = [3] * 9
    z, p, x, u, v = drafted(rng, 27, V)
    temp = np.ones(9, np.float32)
    z[0, 5] = np.nan                                                 # no softmax
    z[3] = -np.inf
    z[6, 9] = np.inf
    z[9, 100:] = -np.inf                                             # masked tokens are ordinary
    x[9] = 2000
    q = np.exp(z[12].astype(np.float64) - z[12].max())
    p[12] = 1.0                                                      # p covers q: the row draws from q
    u[12] = 0.999999
    x[15] = V                                                        # no such token
    v[18:21] = 0.0                                                   # the first token with any weight
    v[21:24] = np.float32(1 - 2.0 ** -24)
    temp[8] = np.nan
    a, t, (wa, wt, _) = run_accept(rows, z, "fp32", x, p, u, v, temp)
    assert (a == wa).all() and (t == wt).all()
    assert t[0] == 0 and t[1] == 0 and t[2] == 0 and t[8] == 0 and (a[[0, 1, 2, 8]] == 0).all() and a[5] == 0
    assert q.sum() > 0
    temp[:] = [-1.0, np.inf, -np.inf, 1e-30, 1e30, 0.05, 20.0, 1.0, 1.0]
    z[:] = drafted(rng, 27, V)[0]
    a, t, (wa, wt, _) = run_accept(rows, z, "fp32", x, p, u, v, temp)
    assert (a == wa).all() and (t == wt).all() and (t[:3] == 0).all()


def test_accept_distribution():
    """Tokens are distributed as the target's softmax, whatever the drafts' (4000 rounds of one draft)."""
    rng = np.random.default_rng(7)
    n, V = 4000, 8
    z0, d0 = rng.standard_normal(V) * 1.5, rng.standard_normal(V)
    p = np.exp(d0) / np.exp(d0).sum()
    rows = [2] * n
    z = np.tile(z0.astype(np.float32), (2 * n, 1))
    x = rng.choice(V, size=2 * n, p=p).astype(np.int32)
    u, v = rng.random((2, 2 * n), dtype=np.float32)
    a, t, (wa, wt, _) = run_accept(rows, z, "fp32", x, np.tile(p.astype(np.float32), (2 * n, 1)), u, v, np.ones(n, np.float32))
    assert (a == wa).all() and (t == wt).all()
    first = np.where(a > 0, x[0::2], t)
    q = np.exp(z0) / np.exp(z0).sum()
    sigma = np.sqrt(q * (1 - q) / n)
    assert (np.abs(np.bincount(first, minlength=V) / n - q) < 5 * sigma).all()


# ---------------------------------------------------------------- together

def a_round(c, heads, seed, stream, arrays=None):
    """append -> attend -> accept as one round, the attention's output standing in for logits; returns the device arrays."""
    rng = np.random.default_rng(seed)
    dim, Hk = c.dim, c.kv_heads
    if arrays is None:
        raw = rng.standard_normal((c.T, heads + 2 * Hk, dim)).astype(np.float32)
        k, v, table = cache_of(c)
        d = Dev(raw)
        w = (heads + 2 * Hk) * dim
        n = c.n
        arrays = dict(raw=raw, d=d, q=d.view((c.T, heads, dim), (w, dim, 1)), k=d.view((c.T, Hk, dim), (w, dim, 1), heads * dim), v=d.view((c.T, Hk, dim), (w, dim, 1), (heads + Hk) * dim),
                      cache=ee.PagedCache(k, v, table), rs=Dev(c.row_start), kl=Dev(c.kv_len), q_out=Dev(np.zeros((c.T, heads, dim), np.float32)),
                      out=Dev(np.zeros((c.T, heads, dim), np.float32)), gain=Dev((0.5 + rng.random(dim)).astype(np.float32)), rope=Dev(rope_table(512, dim)),
                      gs=Dev(c.group_start), gp=Dev(c.group_pages), drafts=Dev(rng.integers(heads * dim, size=c.T).astype(np.int32)), u=Dev(rng.random(c.T, dtype=np.float32)),
                      v_=Dev(rng.random(c.T, dtype=np.float32)), temp=Dev(np.full(n, 0.2, np.float32)), acc=Dev(np.zeros(n, np.int32)), tok=Dev(np.zeros(n, np.int32)))
        arrays["z"] = arrays["out"].view((c.T, heads * dim), (heads * dim, 1))
        g = dict(group_start=arrays["gs"], group_pages=arrays["gp"], max_shared=16 * int(max(c.group_pages)))
        arrays["ws"] = Dev(np.zeros(ee.ee_attend_workspace(arrays["cache"], arrays["rs"], arrays["q_out"], max_kv=max(c.lens), **g) + 256, np.uint8))
        arrays["ws2"] = Dev(np.zeros(ee.ee_accept_workspace(arrays["z"], arrays["rs"]), np.uint8))
        hip().hipDeviceSynchronize()
    A = arrays
    ee.ee_kv_append(A["cache"], A["rs"], A["kl"], A["q"], A["k"], A["v"], A["q_out"], q_gain=A["gain"], k_gain=A["gain"], rope=A["rope"], stream=stream)
    ee.ee_attend(A["cache"], A["rs"], A["kl"], A["q_out"], A["out"], scale=dim ** -0.5, max_kv=max(c.lens), group_start=A["gs"], group_pages=A["gp"],
                 max_shared=16 * int(max(c.group_pages)), workspace=A["ws"], stream=stream)
    ee.ee_accept_drafts(A["z"], A["rs"], A["drafts"], None, A["u"], A["v_"], A["temp"], A["acc"], A["tok"], workspace=A["ws2"], stream=stream)
    return A


def together():
    return ref.Case(400, [3, 1, 5, 2], [150, 161, 133, 40], 2, 64, 2, [(0, 3)], [8]).fill_fast()


def test_round_of_all_three():
    c = together()
    A = a_round(c, 4, 1, 0)
    out, q_out = A["out"].numpy(), A["q_out"].numpy()
    # the cache as it now is, and the queries as they were handed over
    c.k_pool, c.v_pool = A["cache"].k_pool.numpy(), A["cache"].v_pool.numpy()
    gain = A["gain"].numpy()
    x = A["raw"].astype(np.float64)
    want, tol, places = ref.append(c, x[:, :4], x[:, 4:6], x[:, 6:], gain, gain, 1e-5, rope_table(512, 64), False, "fp32")
    close(q_out.astype(np.float64), want, tol, "q_out")
    assert len(places) == c.T
    want, tol = ref.attend(c, q_out.astype(np.float64), 64 ** -0.5, "fp32", "fp32")
    close(out.astype(np.float64), want, tol, "attention")
    wa, wt, margin = ref.accept(c.row_start, out.reshape(c.T, -1), A["drafts"].numpy(), None, A["u"].numpy(), A["v_"].numpy(), A["temp"].numpy())
    assert margin > 1e-11 and (A["acc"].numpy() == wa).all() and (A["tok"].numpy() == wt).all()


def test_round_captured_and_replayed():
    """Two graphs that share workspaces, replayed in turn with eager rounds between: every replay gives the eager bits."""
    h = hip()
    c = together()
    eager = a_round(c, 4, 1, 0)
    want = [eager[k].numpy().copy() for k in ("out", "acc", "tok")]
    s = ctypes.c_void_p()
    ok(h.hipStreamCreate(ctypes.byref(s)))
    A = a_round(together(), 4, 1, 0)
    B = dict(a_round(together(), 4, 1, 0), ws=A["ws"], ws2=A["ws2"])
    hip().hipDeviceSynchronize()
    execs = []
    for arrays in (A, B):
        graph, ex = ctypes.c_void_p(), ctypes.c_void_p()
        ok(h.hipStreamBeginCapture(s, 0))
        a_round(c, 4, 1, s.value, arrays)
        ok(h.hipStreamEndCapture(s, ctypes.byref(graph)))
        ok(h.hipGraphInstantiate(ctypes.byref(ex), graph, None, None, ctypes.c_size_t(0)))
        execs.append((graph, ex))
    for rep in range(4):
        for arrays, (_, ex) in zip((A, B), execs):
            for k in ("out", "acc", "tok", "q_out"):
                arrays[k].write(np.zeros(arrays[k].shape, arrays[k]._np))
            ok(h.hipGraphLaunch(ex, s))
            ok(h.hipStreamSynchronize(s))
            for k, w in zip(("out", "acc", "tok"), want):
                assert (arrays[k].numpy() == w).all(), f"replay {rep}: {k}"
        again = a_round(c, 4, 1, 0, eager)
        assert (again["out"].numpy() == want[0]).all()
    for graph, ex in execs:
        ok(h.hipGraphExecDestroy(ex))
        ok(h.hipGraphDestroy(graph))
    ok(h.hipStreamDestroy(s))


def test_results_do_not_depend_on_timing():
    c = ref.Case(401, [2] * 9, [900 + 40 * i for i in range(9)], 2, 128, 1, [(0, 9)], [40]).fill_fast()
    c.rng = np.random.default_rng(1)
    a = run_attend(c, 8, "bf16", "fp32")[0]
    for _ in range(5):
        c.rng = np.random.default_rng(1)
        assert (run_attend(c, 8, "bf16", "fp32")[0] == a).all()
