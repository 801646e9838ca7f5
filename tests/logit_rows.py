"""Plain 64-bit definitions of the calls on rows of logits, row by row, and how far an fp32 evaluation may be off them.

A rounding to fp32 is off by at most U relative to the value.  A sum of n non-negative terms, added up in any order, is off
by at most the longest chain of additions times U; the kernels give every wave's lane at most V / 64 (rows up to 2048 tokens)
or V / 256 tokens and join the lanes in a tree, so `chain` bounds it."""
import numpy as np

U = 2.0 ** -24
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -25, "bf16": 2.0 ** -126}   # half a step of subnormals, or flushed ones
LARGEST = {"f32": 3.4e38, "f16": 65504.0, "bf16": 3.38e38}


def chain(V):
    return 24 + (V // 64 if V <= 2048 else V // 256)


def row_log_probs(x, T):
    """(log-probs, marked): x a row of float64 values."""
    if np.isnan(x).any() or (x == np.inf).any():
        return np.full(x.shape, np.nan), True
    m = x.max()
    if m == -np.inf:
        return np.full(x.shape, -np.inf), False
    d = (x - m) / T
    return d - np.log(np.exp(d).sum()), False


def entropy(lp):
    p = np.exp(lp)
    return float(-(p[p > 0] * lp[p > 0]).sum())


def lp_error(x, lp, T):
    """Bound on the error of every log-prob: the rounded difference, quotient (a product with a rounded 1/T) and exponential
    argument, 4 U |d|; the sum's chain and its terms' own errors, weighted by their share; the logarithm and the last
    difference."""
    m = x.max()
    if not np.isfinite(m):
        return np.zeros(x.shape)
    d = np.where(x == -np.inf, 0.0, (x - m) / T)
    p = np.exp(lp)
    mean = float((p * np.abs(d)).sum())
    logs = -float(lp.max())
    return U * (chain(len(x)) + 8 + 6 * mean + 6 * np.abs(d) + 4 * logs)


def logprobs(x, T, tokens, n_top):
    """One row: dict of logp, entropy, top tokens, their log-probs, stats and the bounds on their errors."""
    V = len(x)
    lp, marked = row_log_probs(x, T)
    err = lp_error(x, lp, T) if not marked else np.zeros(V)
    inside = (tokens >= 0) & (tokens < V)
    at = np.where(inside, tokens, 0)
    order = np.lexsort((np.arange(V), -x)) if not marked else np.full(V, -1)
    top = order[:n_top]
    H = np.nan if marked else entropy(lp)
    m = np.nan if marked else x.max()
    logs = np.nan if marked else 0.0 if m == -np.inf else -lp.max()
    herr = 0.0
    if not marked and m != -np.inf:
        d = np.where(x == -np.inf, 0.0, (x - m) / T)
        p = np.exp(lp)
        mean, square = float((p * np.abs(d)).sum()), float((p * d * d).sum())
        herr = U * ((2 * chain(V) + 16) * (1 + mean) + 6 * (square + mean * mean) + 6 * logs)
    return dict(logp=np.where(inside, lp[at], np.nan), entropy=H, top=top, top_logp=np.full(n_top, np.nan) if marked else lp[top],
                stats=np.array([m, logs, H]),
                e_logp=np.where(inside, err[at], 0.0), e_entropy=herr, e_top=np.zeros(n_top) if marked else err[top],
                e_logs=0.0 if marked else float(err[np.argmax(x)]))


def logprobs_grad(x, T, tokens, g, h):
    """Gradient of sum g log p(t) + h H of one row and the bound on its error (before the last rounding)."""
    V = len(x)
    inside = (tokens >= 0) & (tokens < V)
    lp, marked = row_log_probs(x, T)
    if h == 0 and not (g[inside] != 0).any():
        return np.zeros(V), np.zeros(V)
    if marked:
        return np.full(V, np.nan), np.zeros(V)
    if x.max() == -np.inf:
        return np.zeros(V), np.zeros(V)
    p, H, G = np.exp(lp), entropy(lp), g[inside].sum()
    onto = np.zeros(V)
    np.add.at(onto, tokens[inside], g[inside])
    flat = np.where(p > 0, lp, 0.0)
    grad = (onto - p * (G + h * np.where(p > 0, lp + H, 0.0))) / T
    size = np.abs(g[inside]).sum()
    herr = logprobs(x, T, np.zeros(0, int), 0)["e_entropy"]
    e = lp_error(x, lp, T)
    err = (p * (size + abs(h) * (np.abs(flat) + H)) * (e + (len(g) + 12) * U) + p * abs(h) * (e + herr) +
           np.abs(onto) * 4 * U + (onto != 0) * size * len(g) * U) / T
    return grad, err


def distill(x, T, tokens, l, tail, w):
    """(loss, gradient, bounds on their errors) of one row."""
    V, K = len(x), len(tokens)
    inside = (tokens >= 0) & (tokens < V)
    zero = np.zeros(V)
    if not inside.any() or (not tail and not (l[inside] > -np.inf).any()):
        return 0.0, zero, 0.0, zero
    l = np.where(inside, l, -np.inf)
    if tail:
        q = np.exp(l)
        rest = 1.0 - q.sum()
        rest = 0.0 if rest < 2.0 ** -20 else rest
    else:
        l = l - l.max()
        l = l - np.log(np.exp(l).sum())
        q, rest = np.exp(l), 0.0
    lp, marked = row_log_probs(x, T)
    if marked:
        return np.nan, (zero if w == 0 else np.full(V, np.nan)), 0.0, zero
    p, e = np.exp(lp), lp_error(x, lp, T)
    on = np.zeros(V, bool)
    on[tokens[inside]] = True
    target = np.zeros(V)
    np.add.at(target, tokens[inside], q[inside])
    mass = q.sum() + rest
    p_rest = p[~on].sum()
    loss, el = 0.0, 0.0
    for k in range(K):
        if inside[k] and q[k] > 0:
            loss += q[k] * (l[k] - lp[tokens[k]])
            if np.isfinite(lp[tokens[k]]):
                el += q[k] * (e[tokens[k]] + U * (6 * abs(l[k]) + 4 * abs(l[k] - lp[tokens[k]]) + 8)) + U * K * abs(q[k] * (l[k] - lp[tokens[k]]))
    e_rest = float(e.max()) + (chain(V) + 12) * U   # (relative)
    if rest > 0:
        loss += rest * (np.log(rest) - np.log(p_rest)) if p_rest > 0 else np.inf
        if p_rest > 0:
            el += rest * (e_rest + U * (8 + K + 6 * abs(np.log(rest) - np.log(p_rest))))
    if x.max() == -np.inf or w == 0:
        return loss, zero, el, zero
    ratio = rest / p_rest if rest > 0 and p_rest > 0 else 0.0
    grad = (p * mass - target - np.where(on, 0.0, p * ratio)) * w / T
    eg = (p * mass * (e + (K + 12) * U) + target * (K + 20) * U + target * U * 6 * np.abs(np.where(np.isfinite(l), l, 0.0)).max() +
          np.where(on, 0.0, p * ratio) * (e + e_rest + 16 * U)) * abs(w) / T
    return loss, grad, el, eg


def rounded(err, want, kind):
    """The bound on an output held in `kind`: what its value may be off by, and the last rounding."""
    return err * (1 + HALF_STEP[kind]) + HALF_STEP[kind] * (np.abs(want) + err) + TINY[kind]


def check(got, want, bound, where):
    """`got` (any float type, as float64) within `bound` of `want`; infinities and NaN in the same places.  A value past the
    largest fp32 number (2^128 - 2^104) by half a step or more rounds to an infinity: the lowest fp32 value as a logit,
    at temperature 0.7, has the log-prob -4.9e38, which fp32 does not hold."""
    got, want, bound = (np.asarray(a, np.float64) for a in (got, want, bound))
    want = np.where(np.abs(want) >= 2.0 ** 128 - 2.0 ** 103, np.copysign(np.inf, want), want)
    assert got.shape == want.shape, where
    assert np.array_equal(np.isnan(got), np.isnan(want)), where
    fin = np.isfinite(want)
    odd = ~fin & ~np.isnan(want)
    assert np.array_equal(got[odd], want[odd]), where
    bound = np.broadcast_to(bound, want.shape)
    off = np.abs(got[fin] - want[fin])
    assert (off <= bound[fin]).all(), (where, float((off / np.maximum(bound[fin], 1e-300)).max()))
