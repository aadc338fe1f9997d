"""Plain 64-bit forms of the operators on device memory, sequence by sequence, and inputs for them (numpy, no GPU)."""
import numpy as np

from tests.device import HALF_STEP, bf16_bits, bf16_values

PAGE = 16
NAN_BITS = 0x7FC0


def split(x, terms):
    """float32 -> [terms][...] bf16 bits."""
    hi = bf16_bits(x)
    if terms == 1:
        return hi[None]
    return np.stack([hi, bf16_bits(np.asarray(x, np.float32) - bf16_values(hi))])


class Case:
    """A batch over paged caches: page tables in no order, everything nobody may read poisoned with NaN."""

    def __init__(self, seed, rows, lens, kv_heads, dim, terms, groups=(), shared=(), spare_pages=3, pad=0, table_extra=2):
        self.rng = rng = np.random.default_rng(seed)
        self.rows, self.lens, self.kv_heads, self.dim, self.terms = list(rows), list(lens), kv_heads, dim, terms
        self.row_start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.T, self.n = int(self.row_start[-1]), len(rows)
        self.cap = self.T + pad
        pages = [-(-max(x, 0) // PAGE) for x in lens]
        stride = max(pages + [1]) + table_extra
        ids = iter(range(10 ** 6))
        table = np.full((self.n, stride), -1, np.int64)
        common = {}
        for g, (lo, hi) in enumerate(groups):
            for s in range(lo, hi):
                for i in range(shared[g]):
                    if (g, i) not in common:
                        common[g, i] = next(ids)
                    table[s, i] = common[g, i]
        for s in range(self.n):
            for i in range(pages[s]):
                if table[s, i] < 0:
                    table[s, i] = next(ids)
        used = next(ids)
        self.n_pages = used + spare_pages
        order = rng.permutation(self.n_pages)
        self.table = np.where(table >= 0, order[np.maximum(table, 0)], rng.choice([-1, -7, self.n_pages, 2 ** 31 - 1], table.shape)).astype(np.int32)
        self.k_pool = np.full((self.n_pages, kv_heads, PAGE, terms, dim), NAN_BITS, np.uint16)
        self.v_pool = np.full((self.n_pages, kv_heads, terms, dim, PAGE), NAN_BITS, np.uint16)
        self.kv_len = np.array(lens, np.int32)
        self.group_start = np.array([g[0] for g in groups] + [groups[-1][1]], np.int32) if groups else None
        self.group_pages = np.array(shared, np.int32) if groups else None

    def fill(self, scale=1.0):
        """Random keys and values at every position that a sequence has."""
        for s in range(self.n):
            for p in range(max(self.lens[s], 0)):
                page, slot = self.table[s, p // PAGE], p % PAGE
                if not (0 <= page < self.n_pages):
                    continue
                k, v = self.rng.standard_normal((2, self.kv_heads, self.dim)).astype(np.float32) * np.float32(scale)
                self.k_pool[page, :, slot] = split(k, self.terms).transpose(1, 0, 2)
                self.v_pool[page, :, :, :, slot] = split(v, self.terms).transpose(1, 0, 2)
        return self

    def fill_fast(self, scale=1.0):
        """The same for large caches: whole pages at once, the unused places of last pages poisoned again."""
        used = sorted({int(x) for s in range(self.n) for x in self.table[s, : -(-max(self.lens[s], 0) // PAGE)] if 0 <= x < self.n_pages})
        k, v = self.rng.standard_normal((2, len(used), self.kv_heads, PAGE, self.dim), dtype=np.float32) * np.float32(scale)
        self.k_pool[used] = np.moveaxis(split(k, self.terms), 0, 3)
        self.v_pool[used] = np.moveaxis(split(v, self.terms), 0, 2).swapaxes(3, 4)
        for s in range(self.n):
            if self.lens[s] % PAGE:
                page = self.table[s, self.lens[s] // PAGE]
                self.k_pool[page, :, self.lens[s] % PAGE:] = NAN_BITS
                self.v_pool[page, :, :, :, self.lens[s] % PAGE:] = NAN_BITS
        return self

    def keys(self, s, k_pool=None):
        """[positions][kv_heads][dim] in 64 bits, and which positions have a place."""
        n = max(self.lens[s], 0)
        pool = self.k_pool if k_pool is None else k_pool
        out, ok = np.zeros((n, self.kv_heads, self.dim)), np.zeros(n, bool)
        for i in range(-(-n // PAGE)):
            page, m = self.table[s, i], min(PAGE, n - i * PAGE)
            if 0 <= page < self.n_pages:
                out[i * PAGE: i * PAGE + m] = bf16_values(pool[page]).astype(np.float64).sum(2)[:, :m].transpose(1, 0, 2)
                ok[i * PAGE: i * PAGE + m] = True
        return out, ok

    def values(self, s, v_pool=None):
        n = max(self.lens[s], 0)
        pool = self.v_pool if v_pool is None else v_pool
        out = np.zeros((n, self.kv_heads, self.dim))
        for i in range(-(-n // PAGE)):
            page, m = self.table[s, i], min(PAGE, n - i * PAGE)
            if 0 <= page < self.n_pages:
                out[i * PAGE: i * PAGE + m] = bf16_values(pool[page]).astype(np.float64).sum(1)[:, :, :m].transpose(2, 0, 1)
        return out


def attend(case, q, scale, kind, out_kind):
    """(expected [T][heads][dim], tolerance of the same shape).

    Tolerance.  A score is a sum of dim products with an error of dim 2^-24 of sum |q k| (fp32 sums); a q beyond bf16 is two bf16 terms (off by
    2^-16: half a step of half a step), and with two-term keys the product of two lo terms is left out (2^-16).  An error d of the scores
    changes a softmax weight by a factor within exp(2 d); exp2 and the running rescale add 2^-21 per step of the running maximum, n 2^-24 for sums of
    n terms; the weights are two bf16 terms (2^-16), with two-term values another 2^-16.  All of it relative to sum w |v|; and the type's half step."""
    H, hd = q.shape[1], q.shape[2]
    G = H // case.kv_heads
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    for s in range(case.n):
        r0, n, L = case.row_start[s], case.rows[s], case.lens[s]
        if not n:
            continue
        K, ok = case.keys(s)
        V = case.values(s)
        for i in range(n):
            seen = np.zeros(len(K), bool)
            seen[: max(L - n + i + 1, 0)] = True
            seen &= ok
            if not seen.any():
                continue
            for h in range(H):
                Ks, Vs, x = K[seen, h // G], V[seen, h // G], q[r0 + i, h].astype(np.float64)
                z = Ks @ x * scale
                e = np.exp(z - z.max())
                w = e / e.sum()
                out[r0 + i, h] = w @ Vs
                rel = hd * 2.0 ** -24 + (0 if kind == "bf16" else 2.0 ** -16) + (2.0 ** -16 if case.terms == 2 else 0)
                d = rel * scale * (np.abs(Ks) @ np.abs(x)).max()
                part = np.expm1(2 * d) + 2.0 ** -16 * case.terms + (len(z) / 32 + 8) * 2.0 ** -21 + len(z) * 2.0 ** -24
                tol[r0 + i, h] = part * (w @ np.abs(Vs)) + HALF_STEP[out_kind] * np.abs(out[r0 + i, h]) + (2.0 ** -25 if out_kind == "fp16" else 0)
    return out, tol


def append(case, q, k, v, q_gain, k_gain, eps, rope, pairs, q_kind):
    """(q_out, its tolerance, {(page, slot): (k, k tolerance, v)}).  fp32: a norm's sum, root and two products are off by less than 24 steps of
    2^-24, a rotation's products and sum by 3, each relative to the magnitudes that enter; then one rounding."""
    dim, u = case.dim, 2.0 ** -24

    def normed(x, gain, cs):
        x = x.astype(np.float64)
        if gain is not None:
            x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * gain.astype(np.float64)
        slack = (24 if gain is not None else 0) * u
        if cs is None:
            return x, slack * np.abs(x)
        c, s = cs[:, 0].astype(np.float64), cs[:, 1].astype(np.float64)
        a, b = (x[..., 0::2], x[..., 1::2]) if pairs else (x[..., : dim // 2], x[..., dim // 2:])
        y, t = np.empty_like(x), np.empty_like(x)
        one, two, mag = a * c - b * s, b * c + a * s, (slack + 3 * u)
        ma, mb = mag * (np.abs(a * c) + np.abs(b * s)), mag * (np.abs(b * c) + np.abs(a * s))
        if pairs:
            y[..., 0::2], y[..., 1::2], t[..., 0::2], t[..., 1::2] = one, two, ma, mb
        else:
            y, t = np.concatenate([one, two], -1), np.concatenate([ma, mb], -1)
        return y, t

    q_out, q_tol, places = np.zeros(q.shape), np.zeros(q.shape), {}
    stored = 2.0 ** -8 if case.terms == 1 else 2.0 ** -16
    for s in range(case.n):
        r0, n, L = case.row_start[s], case.rows[s], max(case.lens[s], 0)
        for i in range(n):
            p = L - n + i
            if p < 0 or p >= case.table.shape[1] * PAGE or (rope is not None and p >= len(rope)):
                continue
            cs = rope[p] if rope is not None else None
            y, t = normed(q[r0 + i], q_gain, cs)
            q_out[r0 + i], q_tol[r0 + i] = y, t + HALF_STEP[q_kind] * np.abs(y) + (2.0 ** -25 if q_kind == "fp16" else 0)
            page = case.table[s, p // PAGE]
            if 0 <= page < case.n_pages:
                y, t = normed(k[r0 + i], k_gain, cs)
                places[(int(page), p % PAGE)] = (y, t + stored * (np.abs(y) + t) + 2.0 ** -130, v[r0 + i].astype(np.float64))
    return q_out, q_tol, places


def accept(row_start, logits, drafts, probs, u, v, temperature):
    """(accept_len, next_token) of every sequence, and how far the nearest decision is from its border (relative)."""
    lens, toks, margin = [], [], np.inf
    for s in range(len(row_start) - 1):
        r0, n = row_start[s], row_start[s + 1] - row_start[s]
        if n <= 0:
            lens.append(0)
            toks.append(-1)
            continue
        T = float(temperature[s])
        bad_T = not (T >= 0 and np.isfinite(T))

        def soft(r):
            z = logits[r].astype(np.float64)
            with np.errstate(all="ignore"):
                e = np.exp((z - np.nanmax(z) if not np.isnan(z).all() else z) / T)
                return e / e.sum()

        def best(r):
            z = np.where(np.isnan(logits[r]), -np.inf, logits[r].astype(np.float64))
            return 0 if np.isnan(logits[r]).all() else int(np.argmax(z))

        def p_row(r):
            if probs is not None:
                return probs[r].astype(np.float64)
            p = np.zeros(logits.shape[1])
            if 0 <= drafts[r] < len(p):
                p[drafts[r]] = 1.0
            return p

        i = 0
        while i < n - 1:
            r, x = r0 + i, int(drafts[r0 + i])
            if bad_T or not 0 <= x < logits.shape[1]:
                break
            if T == 0:
                if x != best(r):
                    break
            else:
                a, b = float(u[r]) * p_row(r)[x], soft(r)[x]
                if np.isfinite(b) and max(a, b) > 0:
                    margin = min(margin, abs(a - b) / max(a, b))
                if not a < b:
                    break
            i += 1
        r = r0 + i
        lens.append(i)
        if bad_T:
            toks.append(0)
            continue
        if T == 0:
            toks.append(best(r))
            continue
        q = soft(r)
        if not np.isfinite(q).all():
            toks.append(0)
            continue
        w = q
        if i < n - 1:
            with np.errstate(invalid="ignore"):
                w = np.fmax(q - p_row(r), 0.0)
            if not w.sum() > 0:
                w = q
        c = np.cumsum(w)
        target = float(v[r]) * c[-1]
        k = int(np.searchsorted(c, target, side="right"))
        k = min(k, int(np.flatnonzero(w > 0)[-1]))
        edges = np.abs(c[max(k - 1, 0): k + 1] - target) / c[-1]
        margin = min(margin, edges.min() if target > 0 else np.inf)
        toks.append(k)
    return np.array(lens, np.int32), np.array(toks, np.int32), margin
