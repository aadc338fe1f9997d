"""ee_attend's precision by types: how many bf16 terms queries and softmax weights are in.

Every key has one or two elements, so that a score is one or two products and the matrix products' sums round it hardly at all; a value of
+-1 or close to it for every position makes results in which weights cancel.  What is left are the roundings that the header names.

Tolerance, relative to sum w |v|, in steps of U = 2^-24 (half a step of fp32 is U; a sum inside a matrix product is counted as 2 U, whatever the order and manner of its
rounding).  A score s (times scale) is off by at most, relative to the largest |s| of the row: 4 U for the two sums of a key with three terms of a query, with two-term keys 8 U for four
sums and U for the product of the smallest terms, which is left out (2^-8 times 2^-16); U where it is multiplied by log2(e), which is itself off by less than U / 2, and 2 U where it is taken relative
to a maximum that is moved once.  An error d of the scores changes a weight by a factor within exp(2 d).  exp2 is off by 2^-23.  The weights' terms: 2^-16 in two (half a step of half a
step), U in three; two-term values leave out U once more.  The sums of n positions: 2 U for each of three products, U for the sum of weights, and 4 U for the quotient.  Then the
result's half step."""
import numpy as np
import pytest

import paper_2505_21594_amd as ee
from tests import operators_ref as ref
from tests.device import Dev, HALF_STEP, bf16_bits, bf16_values, decode, encode

U = 2.0 ** -24


def tolerance(s, w, V, out, terms, out_kind):
    score = (3.5 + (9 if terms == 2 else 4)) * U * np.abs(s).max()
    weight = 2.0 ** -16 if out_kind != "fp32" and terms == 1 else U * (2 if terms == 2 else 1)
    rel = np.expm1(2 * score) + weight + 2.0 ** -23 + (7 * len(s) + 4) * U
    return rel * (w @ np.abs(V)) + HALF_STEP[out_kind] * np.abs(out) + (2.0 ** -25 if out_kind == "fp16" else 0)


def softmax(s):
    e = np.exp(s - s.max())
    return e / e.sum()


def in_terms(x, n):
    """x as the sum of n bf16 terms, each rounded to nearest."""
    left, out = np.asarray(x, np.float32), np.zeros(np.shape(x))
    for _ in range(n):
        t = bf16_values(bf16_bits(left))
        out += t
        left = (left - t).astype(np.float32)
    return out


def make(seed, positions, heads, dim, terms, kind, spread, seqs=6):
    """Sequences of one row.  Position j's key is `unit` at one of two dims (j odd or even), plus smaller bits where the cache has two terms; queries have two
    values about 1.5 of all bits that their type has."""
    rng = np.random.default_rng(seed)
    c = ref.Case(seed, [1] * seqs, [positions] * seqs, 1, dim, terms)
    unit = spread * (1 + np.where(rng.random((seqs, positions)) < 0.5, 0, rng.integers(-16, 17, (seqs, positions)) / 128.0))
    K = np.zeros((seqs, positions, dim), np.float32)
    for s in range(seqs):
        for j in range(positions):
            K[s, j, j % 2] = unit[s, j] * (1 + (rng.integers(-60, 61) * 2.0 ** -15 if terms == 2 else 0))
    V = np.where(rng.random((seqs, positions, dim)) < 0.5, 1.0, -1.0) * (1 + (rng.integers(-60, 61, (seqs, positions, dim)) * 2.0 ** -15 if terms == 2 else 0))
    for s in range(seqs):
        for p in range(positions):
            page, slot = c.table[s, p // 16], p % 16
            c.k_pool[page, 0, slot] = ref.split(K[s, p], terms)
            c.v_pool[page, 0, :, :, slot] = ref.split(V[s, p].astype(np.float32), terms)
    q = np.zeros((seqs, heads, dim), np.float32)
    q[:, :, :2] = 1.5 + 0.004 * rng.random((seqs, heads, 2), dtype=np.float32) / spread + rng.random((seqs, heads, 2), dtype=np.float32) * 2.0 ** -9
    enc = encode(q, kind)
    return c, enc


def expected(c, q, scale, out_kind, weight=lambda w: w):
    """(results, tolerance); weight: how the unnormalised weights enter the product with the values (not their sum)."""
    S, H, hd = q.shape
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    for s in range(S):
        K, V = c.keys(s)[0][:, 0], c.values(s)[:, 0]
        for h in range(H):
            z = K @ q[s, h] * scale
            e = np.exp(z - z.max())
            out[s, h] = weight(e) @ V / e.sum()
            tol[s, h] = tolerance(z, e / e.sum(), V, out[s, h], c.terms, out_kind)
    return out, tol


# heads on one key head: 1 and 20 lines a sequence go by tiles of 16 and 32, 40 and 72 by 128 (72: with two-term caches too)
LINES = [1, 20, 40, 72]
KINDS = [("bf16", "bf16"), ("bf16", "fp16"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp16", "fp32"), ("fp32", "bf16"), ("fp32", "fp32")]


@pytest.mark.gpu
@pytest.mark.parametrize("kind,out_kind", KINDS)
@pytest.mark.parametrize("heads", LINES)
@pytest.mark.parametrize("positions,spread", [(2, 64.0), (2, 0.25), (26, 1.0)])
@pytest.mark.parametrize("dim,terms", [(64, 1), (128, 1), (64, 2), (128, 2)])
def test_terms(dim, terms, positions, spread, heads, kind, out_kind):
    c, enc = make(positions * 100 + heads + dim + terms, positions, heads, dim, terms, kind, spread)
    cache, rs, kl = ee.PagedCache(Dev(c.k_pool), Dev(c.v_pool), Dev(c.table)), Dev(c.row_start), Dev(c.kv_len)
    dq, out = Dev(enc), Dev(encode(np.full(enc.shape, 7.5, np.float32), out_kind))
    n = ee.ee_attend_workspace(cache, rs, dq, max_kv=positions)
    ee.ee_attend(cache, rs, kl, dq, out, scale=1.0, max_kv=positions, workspace=Dev(np.full(max(n, 1), 0x5A, np.uint8)))
    want, tol = expected(c, decode(enc), 1.0, out_kind)
    bad = ~(np.abs(decode(out.numpy()) - want) <= tol)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, at most {(np.abs(decode(out.numpy()) - want) / tol).max():.1f} tolerances"


@pytest.mark.gpu
def test_a_row_does_not_lose_bits_to_its_neighbours():
    """A single token beside a prompt: its result has the same tolerance as alone."""
    dim, positions = 64, 26
    c, enc = make(7, positions, 1, dim, 1, "bf16", 1.0, seqs=2)
    big = ref.Case(8, [400, 1, 1], [400, positions, positions], 1, dim, 1).fill_fast()
    for s in range(2):                                           # the two sequences behind a prompt of 400 rows
        big.k_pool[big.table[1 + s, :2]] = c.k_pool[c.table[s, :2]]
        big.v_pool[big.table[1 + s, :2]] = c.v_pool[c.table[s, :2]]
    rows = np.concatenate([encode(big.rng.standard_normal((400, 1, dim)).astype(np.float32), "bf16"), enc])
    cache, rs, kl = ee.PagedCache(Dev(big.k_pool), Dev(big.v_pool), Dev(big.table)), Dev(big.row_start), Dev(big.kv_len)
    dq, out = Dev(rows), Dev(encode(np.zeros(rows.shape, np.float32), "bf16"))
    n = ee.ee_attend_workspace(cache, rs, dq, max_kv=400)
    ee.ee_attend(cache, rs, kl, dq, out, scale=1.0, max_kv=400, workspace=Dev(np.full(max(n, 1), 0x5A, np.uint8)))
    want, tol = expected(c, decode(enc), 1.0, "bf16")
    assert (np.abs(decode(out.numpy()[400:]) - want) <= tol).all()


@pytest.mark.parametrize("heads", [20, 40])
def test_fewer_terms_fall_outside(heads):
    """Mistakes planted in the plain form: the tolerances find a query or weights of one term less."""
    for dim, terms in ((64, 1), (64, 2)):
        c, enc = make(200 + heads + dim + terms, 2, heads, dim, terms, "fp32", 64.0)
        want, tol = expected(c, decode(enc), 1.0, "fp32")
        assert (np.abs(expected(c, in_terms(enc, 3), 1.0, "fp32")[0] - want) <= tol).all()
        assert (np.abs(expected(c, in_terms(enc, 2), 1.0, "fp32")[0] - want) > tol).any(), "queries in two terms"
        c, enc = make(200 + heads + dim + terms, 2, heads, dim, terms, "fp32", 0.25)
        want, tol = expected(c, decode(enc), 1.0, "fp32")
        assert (np.abs(expected(c, decode(enc), 1.0, "fp32", lambda w: in_terms(w, 3))[0] - want) <= tol).all()
        assert (np.abs(expected(c, decode(enc), 1.0, "fp32", lambda w: in_terms(w, 2))[0] - want) > tol).any(), "weights in two terms"
    for kind in ("bf16", "fp16"):
        c, enc = make(2600 + heads + 64 + 1, 26, heads, 64, 1, kind, 1.0)
        want, tol = expected(c, decode(enc), 1.0, kind)
        assert (np.abs(expected(c, decode(enc), 1.0, kind, lambda w: in_terms(w, 2))[0] - want) <= tol).all()
        assert (np.abs(expected(c, decode(enc), 1.0, kind, lambda w: in_terms(w, 1))[0] - want) > tol).any(), "weights in one term"
