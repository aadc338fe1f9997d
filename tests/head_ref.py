"""Plain 64-bit forms of the operators around the LM head, with the tolerances of their results (numpy, no GPU).

Tolerances.  U = 2^-24 is half a step of fp32.  A sum of n fp32 numbers taken one after the other is off by at most n U times the sum of their magnitudes.
exp2 of an fp32 argument a: the instruction is off by 2 U of its result, the argument by 3 U |a| (difference, factor, product), which moves the result by 0.7 * 3 U |a| of it.  In the sum S
of the exponentials of a row, relative to its largest, sum p_i |a_i| is at most the entropy in bits, 24 for every vocabulary that is allowed, so that S is off by
at most (2 + 51 + n) U of it, n <= 128 terms of a thread, and a few U for the threads' common scale: SUM = 190 U covers all of it.  What is formed from S is in 64 bits."""
import numpy as np

U = 2.0 ** -24
SUM = 190 * U


def score(z, tokens, top, T, half=U):
    """z: float64 logits as the call reads them.  {name: (values, tolerance)}; tokens of the lists exactly."""
    T = float(np.float32(T))                                     # (what the call receives)
    rows, V = z.shape
    out = {k: (np.zeros(rows), np.zeros(rows)) for k in ("logprob", "entropy")}
    ids, lps, tols = np.full((rows, top), -1, np.int64), np.full((rows, top), -np.inf), np.zeros((rows, top))
    for r in range(rows):
        x = z[r]
        if np.isnan(x).any() or (x == np.inf).any() or not np.isfinite(x).any():
            out["logprob"][0][r] = out["entropy"][0][r] = np.nan
            lps[r] = np.nan
            continue
        m = x.max()
        e = np.exp((x - m) / T)
        S = e.sum()
        lse = np.log(S)
        p = e / S
        y = np.where(p > 0, (x - m) / T, 0.0)
        t = tokens[r] if tokens is not None else -1
        lp = (x[t] - m) / T - lse if 0 <= t < V else -np.inf
        out["logprob"][0][r] = lp
        out["logprob"][1][r] = SUM + U * abs(lp) if np.isfinite(lp) else 0
        mean = (p * y).sum()
        out["entropy"][0][r] = lse - mean
        # D = sum y e is off as S is, each term a little more for its own factor; D / S has both
        out["entropy"][1][r] = SUM * (1 + 2 * abs(mean) + 24) + U * abs(lse - mean)
        order = np.lexsort((np.arange(V), -(x + 0.0)))[:top]
        order = order[np.isfinite(x[order])]
        ids[r, : len(order)] = order
        lps[r, : len(order)] = (x[order] - m) / T - lse
        tols[r] = SUM + U * np.where(np.isfinite(lps[r]), np.abs(lps[r]), 0)
    return dict(out, top_ids=ids, top_logprobs=(lps, tols))


def distill(z, ids, logprobs, T, rest, weight=None, half=U, subnormal=0.0):
    """(loss, tolerance), (gradient, tolerance); `half`: half a step of the gradient's type, `subnormal`: of its smallest numbers."""
    T = float(np.float32(T))                                     # (what the call receives)
    rows, V = z.shape
    loss, loss_tol, grad, grad_tol = np.zeros(rows), np.zeros(rows), np.zeros((rows, V)), np.zeros((rows, V))
    for r in range(rows):
        w = (1.0 if weight is None else float(weight[r]))
        x = z[r]
        if np.isnan(x).any() or (x == np.inf).any() or not np.isfinite(x).any():
            loss[r] = np.nan
            grad[r] = np.nan if w else 0.0
            continue
        with np.errstate(divide="ignore"):
            m = x.max()
            e = np.exp((x - m) / T)
            q = e / e.sum()
            log_q = (x - m) / T - np.log(e.sum())
            p = np.zeros(V)
            merged = {}                                          # (a token that is named twice has the sum of both probabilities)
            for i, l in zip(ids[r], logprobs[r].astype(np.float64)):
                if 0 <= i < V and l != -np.inf:
                    merged[int(i)] = np.logaddexp(merged.get(int(i), -np.inf), l)
            entries = list(merged.items())
            for i, l in entries:
                p[i] += np.exp(l)
            named = np.zeros(V, bool)
            named[[i for i, _ in entries]] = True
            share = p.sum()
            if rest:
                pi = max(1 - share, 0.0)
                rho = q[~named].sum()
                loss[r] = sum(np.exp(l) * (l - log_q[i]) for i, l in entries)
                g = q - p
                others = np.zeros(V)
                if pi > 0 and not named.all():
                    # (the logarithm apart from q, which may be below every number)
                    at = np.where(named, -np.inf, x)
                    log_rho = -np.inf
                    if np.isfinite(at).any():
                        log_rho = (at.max() - m) / T + np.log(np.exp((at - at.max()) / T).sum()) - np.log(e.sum())
                    loss[r] += pi * (np.log(pi) - log_rho)
                    others = pi * np.exp(np.where(named, -np.inf, log_q - log_rho)) if np.isfinite(log_rho) else others
                g[~named] = (q - others)[~named]
                parts = np.where(named, q + p, q + others)
            else:
                l0 = np.log(share) if share > 0 else 0.0
                loss[r] = sum(np.exp(l) / share * (l - l0 - log_q[i]) for i, l in entries) if share > 0 else 0.0
                g = q - p / share if share > 0 else np.zeros(V)
                parts = q + p / share if share > 0 else np.zeros(V)
        a = np.where(np.isfinite(x), np.abs(x - m) / T * 1.4427, 0.0)
        # log2(e) / T in fp32 is off by U of it: the loss of a temperature that is, by U times d loss / d log T = sum p y - sum q y (the unnamed tokens' share pi spread as q is)
        y = np.where(q > 0, (x - m) / T, 0.0)
        at_p = 0.0
        if entries and np.isfinite(loss[r]):
            at_p = sum(np.exp(l) * (x[i] - m) / T for i, l in entries if np.isfinite(x[i])) / (1.0 if rest else max(share, 1e-300))
            if rest and pi > 0 and not named.all():
                weight_of = np.exp((at - at.max()) / T)
                at_p += pi * (weight_of * np.where(weight_of > 0, (x - m) / T, 0.0)).sum() / weight_of.sum()
        # An unnamed token's exponential is off by a factor 1 + e_i, |e_i| <= (2 + 2.1 |a| + 138) U: a its exponent from the largest unnamed one, the thread's sum in the rest.  It
        # is in S, of which the loss has P log S (P: all of p), and in rho, of which it has - pi log rho: sum q_i (P - pi / rho) e_i, and squares.  All else is in 64 bits.
        P, moved = (share + max(1 - share, 0.0) if rest else 1.0), 0.0
        if entries and not named.all() and np.isfinite(x[~named]).any():
            u = x[~named]
            a_u = np.where(np.isfinite(u), (u.max() - u) / T * 1.4427, 0.0)
            w_u = np.where(np.isfinite(u), np.exp((u - u.max()) / T), 0.0)
            moved = (np.abs(P * q[~named] - (P - share if rest else 0.0) * w_u / w_u.sum()) * (140 + 2.1 * a_u)).sum() * U
        loss_tol[r] = moved + P * SUM ** 2 + U * abs(loss[r]) + U * abs(at_p - P * (q * y).sum()) if np.isfinite(loss[r]) else 0
        grad[r] = g * w / T
        # a factor of the row that is off as two sums are, and the element's own exponential
        grad_tol[r] = np.abs(w / T) * parts * (2 * SUM + (6 + 2.1 * a) * U) + half * np.abs(grad[r]) + subnormal + 1e-37
        if w == 0:
            grad[r] = 0
    return (loss, loss_tol), (grad, grad_tol)


def norm(x, gain, bias, eps, center, half=U):
    """(y, tolerance).  A thread adds up to 32 elements, lanes and waves 10 sums: 42 U for a sum of squares, of which the root takes half; mu as much of the magnitudes' mean."""
    g = np.ones(x.shape[1]) if gain is None else gain.astype(np.float64)
    b = np.zeros(x.shape[1]) if bias is None else bias.astype(np.float64)
    mu = x.mean(1, keepdims=True) if center else 0.0
    d = x - mu
    r = 1 / np.sqrt((d * d).mean(1, keepdims=True) + eps)
    y = d * r * g + b
    off = 44 * U * np.abs(x).mean(1, keepdims=True) * r if center else 0.0       # of x^, by the mean's error
    tol = half * np.abs(y) + np.abs(g) * (np.abs(d) * r * 32 * U + off * (1 + np.abs(d) * r)) + 2 * U * np.abs(b)
    return y, tol


def norm_grad(x, dy, gain, eps, center, half=U, groups=512):
    """(dx, tolerance), (d_gain, tolerance), (d_bias, tolerance)."""
    rows, dim = x.shape
    g = np.ones(dim) if gain is None else gain.astype(np.float64)
    mu = x.mean(1, keepdims=True) if center else 0.0
    d = x - mu
    r = 1 / np.sqrt((d * d).mean(1, keepdims=True) + eps)
    unit, u = d * r, dy * g
    along = (u * unit).mean(1, keepdims=True)
    mean = u.mean(1, keepdims=True) if center else 0.0
    dx = r * (u - mean - unit * along)
    off = 44 * U * np.abs(x).mean(1, keepdims=True) * r if center else 0.0
    sizes = np.abs(u).mean(1, keepdims=True), np.abs(u * unit).mean(1, keepdims=True)
    off_unit = np.abs(unit) * 32 * U + off * (1 + np.abs(unit))                     # how far a unit may be off
    tol = half * np.abs(dx) + r * ((np.abs(u) + sizes[0]) * 80 * U + np.abs(unit) * (sizes[1] * 80 * U + sizes[0] * off * 2) + off_unit * np.abs(along)) + r * 4 * U * np.abs(u)
    n = (rows / groups + groups / 16 + 40) * U                                       # rows of a workgroup, of the second launch's thread, the rest
    d_gain, d_bias = (dy * unit).sum(0), dy.sum(0)
    return (dx, tol), (d_gain, n * np.abs(dy * unit).sum(0) + (np.abs(dy) * off_unit).sum(0)), (d_bias, n * np.abs(dy).sum(0))


def phi(z):
    from math import erf
    return 0.5 * (1 + np.vectorize(erf)(z * 0.5 ** 0.5)) if z.size else z


def act(z, kind):
    if kind == 1:
        return z / (1 + np.exp(-z))
    return z if kind == 0 else z * phi(z)


def slope(z, kind):
    if kind == 1:
        s = 1 / (1 + np.exp(-z))
        return s * (1 + z * (1 - s))
    return np.ones_like(z) if kind == 0 else phi(z) + z * np.exp(-z * z / 2) / np.sqrt(2 * np.pi)


# the fp32 activations: 8 U of their value where they are formed, and 1.13 times what z is off by
ACT = 16 * U


def linear(x, w, bias, residual, kind, half, half_pre):
    """(y, tolerance), (pre, tolerance)."""
    K = x.shape[1]
    z = x @ w.T
    size = np.abs(x) @ np.abs(w).T
    if bias is not None:
        z = z + bias
    tol_z = (K + 2) * U * size + 2 * U * np.abs(z)
    y = act(z, kind)
    tol = (1.13 if kind else 1.0) * tol_z + (ACT * (np.abs(z) + np.abs(y)) if kind else 0)
    if residual is not None:
        y = y + residual
        tol = tol + 2 * U * np.abs(y)
    return (y, tol + half * np.abs(y) * (1 + 2.0 ** -8)), (z, tol_z + half_pre * np.abs(z) * (1 + 2.0 ** -8))


def linear_grad(x, w, dy, pre, kind, half_dx, half_dw, step_dx, step_dw):
    """(dx, tolerance), (dw, tolerance), (db, tolerance); step_*: how far dz is rounded for that result (0: not)."""
    rows = x.shape[0]
    dz = dy * (slope(pre, kind) if kind else 1.0)
    tol_dz = ACT * np.abs(dy) * (1 + np.abs(pre)) if kind else 0 * dy
    size_x, size_w = np.abs(dz) @ np.abs(w), np.abs(dz).T @ np.abs(x)
    dx, dw = dz @ w, dz.T @ x
    n = 3 if kind else 1                                                              # terms that a result may be summed in
    tol_x = (n * w.shape[0] * U + step_dx) * size_x + tol_dz @ np.abs(w) + half_dx * np.abs(dx) * (1 + 2.0 ** -8)
    tol_w = (n * rows * U + step_dw) * size_w + tol_dz.T @ np.abs(x) + half_dw * np.abs(dw) * (1 + 2.0 ** -8)
    return (dx, tol_x), (dw, tol_w), (dz.sum(0), rows * U * np.abs(dz).sum(0) + tol_dz.sum(0))
