"""Plain 64-bit definitions of the calls around a student (pb_embed_tokens, pb_embed_tokens_backward, pb_grad_norm, pb_grad_clip,
pb_verify_draft), and how far an evaluation may be off them."""
import numpy as np

U = 2.0 ** -24
BELOW_1 = np.float32(1 - 2.0 ** -24)
FEW = 32        # places of a token's positions that are summed one after the other, before those sums are


def probabilities(x, T):
    """(p, log p, marked) of a row of float64 values."""
    if np.isnan(x).any() or (x == np.inf).any():
        return np.full(x.shape, np.nan), np.full(x.shape, np.nan), True
    m = x.max()
    if m == -np.inf:
        return np.zeros(x.shape), np.full(x.shape, -np.inf), False
    with np.errstate(over="ignore", under="ignore"):
        z = (x - m) / T
        e = np.exp(z)
    ones, rest = (e == 1.0).sum(), e[e < 1.0].sum()  # (apart: a sum of 150000 of them with the 1 among them loses 2^-53 at each of its steps)
    return e / (ones + rest), z - (np.log(ones) + np.log1p(rest / ones)), False


def number(u):
    """A random number as the call takes it: the nearest in [0, 1) that fp32 holds, NaN as 0."""
    return 0.0 if np.isnan(u) else float(np.clip(np.float32(u), np.float32(0), BELOW_1))


def drawn(r, w):
    """The first token whose sum up to it passes w times the whole; -1 where there is no mass.  In units of the largest one, so that the sums of
    equal weights, 1 each, are exact: 75000 of 150000 tokens are not more than 0.5 of them, but 75000 times p, p = 1 / 150000 rounded and the
    sums rounded 75000 times, may come out as more."""
    if not r.max() > 0:
        return -1
    upto = np.cumsum(r / r.max())
    has = (upto > w * upto[-1]) & (r > 0)
    return int(np.argmax(has)) if has.any() else int(np.flatnonzero(r > 0)[-1])


def verify(x, y, T, Ty, tokens, numbers):
    """One sequence: x [n + 1, V], y [n, V] or None, tokens [n], numbers [n + 1]: (tokens [n + 1], accepted, log-probs [n + 1])."""
    n, V = len(tokens), x.shape[1]
    out, logp = np.full(n + 1, -1), np.full(n + 1, np.nan)
    outside = [i for i in range(n) if not 0 <= tokens[i] < V]
    count = outside[0] if outside else n
    for k in range(count + 1):
        p, lp, bad = probabilities(x[k], T)
        if k < count:
            t = tokens[k]
            q, bad_y = np.zeros(V), False
            if y is None:
                q[t] = 1.0
            else:
                q, _, bad_y = probabilities(y[k], Ty)
            if not (bad or bad_y) and number(numbers[k]) * q[t] < p[t]:
                out[k], logp[k] = t, lp[t]
                continue
            if bad or bad_y:
                return out, k, logp
            rest = np.maximum(p - q, 0.0)
            if rest.sum() > 2.0 ** -40:
                p = rest
        elif bad:
            return out, k, logp
        out[k] = drawn(p, number(numbers[n]))
        if out[k] >= 0:
            logp[k] = lp[out[k]]
        return out, k, logp


def table_gradient(g, tokens, V, scale):
    """(gradient, bound on an fp32 evaluation's error, occurrences): g [n, dim] float64."""
    inside = (tokens >= 0) & (tokens < V)
    total, size, count = np.zeros((V, g.shape[1])), np.zeros((V, g.shape[1])), np.bincount(tokens[inside], minlength=V)
    np.add.at(total, tokens[inside], g[inside])
    np.add.at(size, tokens[inside], np.abs(g[inside]))
    # (a sum of at most FEW terms one after the other, then of a piece each FEW places; or, few tokens on a small table, a quarter of the
    # terms at most one after the other, then of up to 256 such shares; the product with the scale)
    chain = np.maximum(np.minimum(count, FEW) + count // FEW, np.minimum(count, count // 4 + 8) + 256 * (len(tokens) <= 16384)) + 3
    return total * scale, size * abs(scale) * U * chain[:, None], count


def norm(tensors):
    return float(np.sqrt(sum(float((t * t).sum()) for t in tensors)))
