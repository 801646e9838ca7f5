"""Rows of logits of which one part says nothing beside another, and gradients and losses that are small beside the numbers they
are the difference of, on the GPU against the 64-bit definitions in logit_rows.py."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import logit_rows as R  # noqa: E402
from gpu_helpers import DEV, dev  # noqa: E402
from test_gpu_logits import JUNK, KIND, check_logprobs, host, place, run_backward, run_distill, run_logprobs, tokens_of  # noqa: E402


def masked_rows(rng, rows, V, kind):
    """Rows of which whole stretches are masked by finite values, in turn: all but the first token, the last, three of them, a
    run of an eighth, the last few, and ordinary rows with one logit so large that nothing else counts."""
    low = [-R.LARGEST[kind], -6e4 if kind == "f16" else -1e37, -2e4 if kind == "f16" else -6e35]
    x = rng.normal(0, 2.5, (rows, V))
    for r in range(rows):
        keep = np.zeros(V, bool)
        sort = r % 6
        if sort == 0:
            keep[0] = True
        elif sort == 1:
            keep[V - 1] = True
        elif sort == 2:
            keep[rng.integers(0, V, 3)] = True
        elif sort == 3:
            keep[V // 4:V // 4 + V // 8] = True
        elif sort == 4:
            keep[-17:] = True
        else:
            keep[:] = True
            x[r, rng.integers(0, V)] = R.LARGEST[kind] if r // 6 % 2 == 0 else 3e4 if kind == "f16" else 1e36
        x[r, ~keep] = low[r // 6 % 3]
    return x


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("rows,V", [(18, 600), (18, 2100), (18, 9000), (300, 9000), (1030, 9000), (18, 40000), (18, 80000), (18, 131072)])
def test_finite_masks_of_whole_stretches(rows, V, kind):
    """A wave, or a part of a split row, that holds nothing but a mask of a lowest value beside one that holds ordinary logits:
    the entropy counts what is left, and so do the statistics and the gradients that are formed from them."""
    rng = np.random.default_rng(rows + V)
    some = 18
    x = masked_rows(rng, some, V, kind)
    for T in (1.0, 0.7):
        buf, view, values = place(np.tile(x, (rows // some + 1, 1))[:rows], kind)
        tokens = tokens_of(rng, values[:some], 3)
        tokens[:, 2] = values[:some].argmax(axis=1)
        all_tokens = np.tile(tokens, (rows // some + 1, 1))[:rows]
        d_tokens = dev(all_tokens.astype(np.int32))
        for top in (0, 5):
            o = run_logprobs(view, kind, V, V, T, d_tokens, top)
            check_logprobs({k: None if v is None else v[:some] for k, v in o.items() if k != "ws"}, values[:some], T, tokens, top,
                           (rows, V, kind, T, top))
            assert not bool(torch.isnan(o["entropy"]).any()) and not bool(torch.isnan(o["stats"]).any())
        g, h = rng.normal(0, 1, (rows, 3)).astype(np.float32), rng.normal(0, 1, rows).astype(np.float32)
        for d_h in (None, dev(h)):
            grad = torch.full((rows, V), JUNK, dtype=KIND[kind][1], device=DEV)
            run_backward(view, kind, V, V, T, o["stats"], d_tokens, dev(g), d_h, grad, V)
            got = host(grad[:some])
            for r in range(some):
                want, err = R.logprobs_grad(values[r], T, tokens[r], g[r].astype(np.float64), 0.0 if d_h is None else float(h[r]))
                R.check(got[r], want, R.rounded(err, want, kind), (rows, V, kind, T, r))


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("V", [5, 600, 1025, 9000, 40000])
def test_gradient_without_an_entropy_term_does_not_look_at_the_entropy(V, kind):
    """Where h is 0 or not given, whatever the statistics hold for H: the same bits.  A marked row keeps its mark."""
    rng = np.random.default_rng(V)
    x = rng.normal(0, 2.5, (8, V))
    x[2, :V // 2] = -np.inf
    x[3, V // 2] = np.nan
    x[4] = -np.inf
    buf, view, values = place(x, kind)
    tokens = dev(rng.integers(0, V, (8, 2)).astype(np.int32))
    g = dev(rng.normal(0, 1, (8, 2)).astype(np.float32))
    stats = run_logprobs(view, kind, V, V, 1.0)["stats"]
    zero = torch.zeros(8, device=DEV)
    some = zero.clone()
    some[0] = 0.5        # (a row that does look)
    want = {}
    for H in (None, float("nan"), float("inf"), -1e38):
        s = stats.clone()
        if H is not None:
            s[1:, 2] = H
        for name, h in (("none", None), ("zero", zero), ("some", some)):
            grad = torch.full((8, V), JUNK, dtype=KIND[kind][1], device=DEV)
            run_backward(view, kind, V, V, 1.0, s, tokens, g, h, grad, V)
            got = host(grad)
            assert np.isnan(got[3]).all() and np.isfinite(np.delete(got, 3, axis=0)).all(), (V, kind, H, name)
            assert np.array_equal(got, want.setdefault(name, got), equal_nan=True), (V, kind, H, name)
    assert np.array_equal(want["none"], want["zero"], equal_nan=True)


def listed_gradient(x, T, tokens, g):
    """(gradient, bound on its error before the last rounding) of sum g log p(t): on a token t that takes `onto`, the sum of its
    own g, and leaves `rest`, that of the others, ((1 - p) onto - p rest) / T.  Neither term is a difference of larger ones, so the
    error is p's, of either term its own: of 1 - p the log-prob's times p and a few roundings of itself, of onto and rest one
    rounding a term of the sum; 10 U for the products and exponentials."""
    V = len(x)
    inside = (tokens >= 0) & (tokens < V)
    lp, marked = R.row_log_probs(x, T)
    if marked or not (g[inside] != 0).any() or x.max() == -np.inf:
        return np.full(V, np.nan if marked and (g[inside] != 0).any() else 0.0), np.zeros(V)
    p, e, M = np.exp(lp), R.lp_error(x, lp, T), len(g)
    not_p = np.where(lp > -0.5, -np.expm1(lp), 1 - p)
    onto, size = np.zeros(V), np.zeros(V)
    np.add.at(onto, tokens[inside], g[inside])
    np.add.at(size, tokens[inside], np.abs(g[inside]))
    rest, others = g[inside].sum() - onto, np.abs(g[inside]).sum() - size
    for t in set(tokens[inside]):      # (without the rounding of that difference)
        rest[t], others[t] = g[inside & (tokens != t)].sum(), np.abs(g[inside & (tokens != t)]).sum()
    grad = (not_p * onto - p * rest) / T
    return grad, (size * (not_p * (M + 10) * R.U + p * (e + 4 * R.U)) + p * others * (e + (M + 10) * R.U)) / T


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("V", [2, 7, 129, 1025, 9000, 40000])
def test_gradients_on_listed_tokens_of_little_weight(V, kind):
    """Tokens whose own g is 0, or small, beside others of weight: what they get is -p times the others' sum, however small p is;
    the same where the row is sure of a token, listed or not."""
    rng = np.random.default_rng(V)
    for M in (2, 3, 17, 64):
        rows = 12
        x = rng.normal(0, 4, (rows, V))
        x[rows // 2:, rng.integers(0, V)] += 25.0
        buf, view, values = place(x, kind)
        tokens = tokens_of(rng, values, M)
        tokens[::2, 0] = values[::2].argmax(axis=1)
        g = rng.choice([0.0, 0.0, 1e-6, -1e-9, 1.0, -1.0, 100.0], (rows, M)).astype(np.float32)
        g[0], g[0, 0] = 0.0, 1.0
        g[1], g[1, 1] = 0.0, -1.0
        for T in (1.0, 0.7):
            grad = torch.full((rows, V), JUNK, dtype=KIND[kind][1], device=DEV)
            stats = run_logprobs(view, kind, V, V, T)["stats"]
            run_backward(view, kind, V, V, T, stats, dev(tokens.astype(np.int32)), dev(g), None, grad, V)
            got = host(grad)
            for r in range(rows):
                want, err = listed_gradient(values[r], T, tokens[r], g[r].astype(np.float64))
                R.check(got[r], want, R.rounded(err, want, kind), (V, kind, M, T, r))


@pytest.mark.parametrize("rows,V", [(6, 40), (6, 9000), (6, 70000), (6, 131072)])
def test_entries_that_are_no_numbers_where_nothing_is_left(rows, V):
    """An entry of +inf or NaN where the student leaves nothing to the tokens that are not listed (p' = 0): loss and gradient are
    NaN, in split rows too.  Without it the loss is +inf where the list leaves something and a number where it does not."""
    x = torch.full((rows, V), -float("inf"), device=DEV)
    x[:, :5] = torch.arange(5, device=DEV) / 4.0
    t = torch.arange(5, dtype=torch.int32, device=DEV).repeat(rows, 1)
    l = torch.full((rows, 5), -2.0, device=DEV)
    l[1, 2], l[2, 0], l[3, 4] = float("inf"), float("nan"), float("inf")
    l[4] = float(np.log(0.2))
    for tail in (False, True):
        loss, grad = torch.full((rows,), JUNK, device=DEV), torch.full((rows, V), JUNK, device=DEV)
        run_distill(x, "f32", V, V, 1.0, t, l, tail, None, loss, grad, V)
        only = torch.full((rows,), JUNK, device=DEV)
        run_distill(x, "f32", V, V, 1.0, t, l, tail, None, only, None, 0)
        got = host(loss)
        assert np.isnan(got[1:4]).all() and np.isnan(host(only)[1:4]).all() and np.isnan(host(grad)[1:4]).all(), (V, tail)
        assert np.isfinite(got[4]) and np.isfinite(host(grad)[[0, 4, 5]]).all()
        assert (got[[0, 5]] == np.inf).all() if tail else np.isfinite(got[[0, 5]]).all()


# (type, temperature, a): at -a, or just beside it, lies the line past which rows are summed from the differences to their maximum
FAR = [("f32", 1.0, 726817.5), ("f32", 1.4426950408889634, 1048576.0), ("bf16", 1.4426950408889634, 1048576.0),
       ("f16", 4096 / 1048576 * 1.4426950408889634, 4096.0), ("bf16", 1.4426950408889634 / 8192, 128.0)]


@pytest.mark.parametrize("kind,T,a", FAR)
@pytest.mark.parametrize("V", [1, 5, 40, 1025, 9000, 131072])
def test_rows_on_the_line_of_far_logits(V, kind, T, a):
    """Rows whose maximum is -2^20 T ln 2 exactly, as far from 0 as a row is summed in one pass, or the next number on either side:
    equal throughout, half of them, one token ahead of others that are as far."""
    T = float(np.float32(T))
    step = {"f32": 2.0 ** -23, "f16": 2.0 ** -10, "bf16": 2.0 ** -7}[kind]
    rng = np.random.default_rng(V)
    x = np.full((9, V), -np.inf)
    for r in range(9):
        m = -a * [1.0, 1.0 + step, 1.0 - step / 2][r // 3]
        if r % 3 == 0:
            x[r] = m
        elif r % 3 == 1:
            x[r] = np.where(rng.random(V) < 0.5, m, m - a * step * rng.integers(1, 4, V))
            x[r, rng.integers(0, V)] = m
        else:
            x[r] = np.where(rng.random(V) < 0.5, -np.inf, m - 3 * a * step)
            x[r, rng.integers(0, V)] = m
    buf, view, values = place(x, kind)
    tokens = tokens_of(rng, values, 2)
    o = run_logprobs(view, kind, V, V, T, dev(tokens.astype(np.int32)), min(V, 3))
    check_logprobs(o, values, T, tokens, min(V, 3), (V, kind, T))
    t = np.stack([rng.permutation(V)[:min(V, 3)] for _ in range(9)])
    l = np.log(rng.dirichlet(np.ones(min(V, 3) + 1), 9)[:, :-1]).astype(np.float32)
    for tail in (False, True):
        loss, grad = torch.full((9,), JUNK, device=DEV), torch.full((9, V), JUNK, dtype=KIND[kind][1], device=DEV)
        run_distill(view, kind, V, V, T, dev(t.astype(np.int32)), dev(l), tail, None, loss, grad, V)
        got, got_loss = host(grad), host(loss)
        for r in range(9):
            want, gr, e, eg = R.distill(values[r], T, t[r], l[r].astype(np.float64), tail, 1.0)
            R.check(got_loss[r], want, e * (1 + 2 ** -20) + R.U * abs(want) + 1e-37, (V, kind, T, tail, r, "loss"))
            R.check(got[r], gr, R.rounded(eg, gr, kind), (V, kind, T, tail, r, "grad"))


def near_certain(rng, V, kind):
    """Six rows with all but 1e-3 .. 1e-8 of their mass on one token; (rows, their values, the tokens, the others' terms seen from
    the token's, their sums, the bounds on those, relative)."""
    x = np.where(rng.random((6, V)) < 30.0 / V, rng.uniform(-21, -10, (6, V)), -np.inf)
    at = np.array([0, V - 1, *rng.integers(0, V, 4)])
    x[np.arange(6), at] = np.array([0.0, 3.0, -2.0, 0.0, 5.5, 0.0])
    buf, view, values = place(x, kind)
    d = values - values.max(axis=1, keepdims=True)
    e = np.where(np.arange(V) == at[:, None], 0.0, np.exp(d))
    far = np.abs(np.where(np.isfinite(d), d, 0.0)).max(axis=1)
    return view, values, at, e, e.sum(axis=1), R.U * (R.chain(V) + 20 + 8 * far)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V", [5, 40, 1025, 9000, 70001, 131072])
def test_small_gradient_of_a_list_that_leaves_next_to_nothing(V, kind):
    """One entry of q = 1 - 5e-7, whose rest counts as 0, and a student that is as sure of it: the gradient q p - q on it, -q R / (1 + R),
    is as near relative to itself as R is.  (The loss is q (l + log(1 + R)).)"""
    rng = np.random.default_rng(V)
    view, values, at, e, R_, off = near_certain(rng, V, kind)
    l = np.array([-5e-7, -1e-7, -9e-7, -3e-8, 2e-7, -6e-7], np.float32)
    loss, grad = torch.full((6,), JUNK, device=DEV), torch.full((6, V), JUNK, dtype=KIND[kind][1], device=DEV)
    run_distill(view, kind, V, V, 1.0, dev(at[:, None].astype(np.int32)), dev(l[:, None]), True, None, loss, grad, V)
    for r in range(6):
        q = np.exp(np.float64(l[r]))
        small = np.log1p(R_[r])
        R.check(host(loss)[r], q * (l[r] + small), q * small * off[r] + R.U * abs(q * (l[r] + small)) + 1e-13, (V, kind, r, "loss"))
        want = q * e[r] / (1 + R_[r])
        want[at[r]] = -q * R_[r] / (1 + R_[r])
        R.check(host(grad)[r], want, np.abs(want) * (off[r] + R.HALF_STEP[kind]) + 1e-14 + R.TINY[kind], (V, kind, r, "grad"))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 1025, 9000, 70001, 131072])
def test_small_losses_of_a_student_sure_of_a_token_not_listed(V, kind):
    """Teacher and student leave all but 1e-8 or so to the tokens that are not listed, the student to one of them: log p' =
    -log(1 + L / (1 + S)) with L and S the sums of the listed and of the other tokens beside that one, and the gradient's share
    q' / p' - 1, are as near as L is, not as 1 is."""
    rng = np.random.default_rng(V)
    view, values, at, e, R_, off = near_certain(rng, V, kind)
    t, l = np.zeros((6, 2), int), np.zeros((6, 2), np.float32)
    for r in range(6):
        some = np.flatnonzero(e[r] > 0)
        t[r] = rng.choice(some, 2, replace=False)
        l[r] = np.log(e[r][t[r]]) + rng.normal(0, 1, 2)
    loss, grad = torch.full((6,), JUNK, device=DEV), torch.full((6, V), JUNK, dtype=KIND[kind][1], device=DEV)
    run_distill(view, kind, V, V, 1.0, dev(t.astype(np.int32)), dev(l), True, None, loss, grad, V)
    for r in range(6):
        where = (V, kind, r)
        q = np.exp(l[r].astype(np.float64))
        terms = np.where(np.arange(V) == at[r], 1.0, e[r])
        L, S = e[r][t[r]].sum(), R_[r] - e[r][t[r]].sum()
        rest, log_rest = 1 - q.sum(), np.log1p(-q.sum())
        lp = np.log(e[r][t[r]]) - np.log1p(R_[r])
        if rest < 0.5:
            continue
        log_p = -np.log1p(L / (1 + S))
        want = (q * (l[r] - lp)).sum() + rest * (log_rest - log_p)
        bound = (q * off[r]).sum() + L * off[r] + R.U * abs(want) + 1e-13
        R.check(host(loss)[r], want, bound, where + ("loss",))
        share = q.sum() - rest * np.expm1(-log_p)      # 1 - q' / p', q' = 1 - sum q, 1 / p' = 1 + L / (1 + S)
        p = terms / (1 + R_[r])
        g = p * share
        g[t[r]] = p[t[r]] - q
        err = p * (abs(share) * off[r] + L * off[r] + 1e-13)
        err[t[r]] = (p[t[r]] + q) * off[r]
        R.check(host(grad)[r], g, R.rounded(err, g, kind), where + ("grad",))


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("V", [1, 2, 7, 40, 1025, 9000, 40000, 70000, 131072])
def test_rows_without_a_number(V, kind):
    """Rows of nothing but NaN, or of NaN and -inf, are marked throughout, their gradients too: they are no rows of nothing but -inf.
    A row of weight 0 has gradient 0 all the same."""
    rng = np.random.default_rng(V)
    x = np.full((6, V), np.nan)
    x[1, rng.random(V) < 0.5] = -np.inf
    x[2] = -np.inf
    x[3] = -np.inf
    x[3, rng.integers(0, V)] = np.nan
    x[4] = rng.normal(0, 1, V)
    buf, view, values = place(x, kind)
    marked = np.isnan(values).any(axis=1)
    tokens = rng.integers(0, V, (6, 2))
    d_tokens = dev(tokens.astype(np.int32))
    o = run_logprobs(view, kind, V, V, 1.0, d_tokens, min(V, 3))
    check_logprobs(o, values, 1.0, tokens, min(V, 3), (V, kind))
    grad = torch.full((6, V), JUNK, dtype=KIND[kind][1], device=DEV)
    run_backward(view, kind, V, V, 1.0, o["stats"], d_tokens, torch.ones((6, 2), device=DEV), None, grad, V)
    assert np.array_equal(np.isnan(host(grad)), np.tile(marked[:, None], (1, V))) and not host(grad)[2].any()
    l = torch.full((6, 2), -1.0, device=DEV)
    w = np.array([1.0, -2.0, 1.0, 0.5, 1.0, 0.0], np.float32)
    for tail in (False, True):
        loss = torch.full((6,), JUNK, device=DEV)
        run_distill(view, kind, V, V, 1.0, d_tokens, l, tail, dev(w), loss, grad, V)
        got = host(grad)
        assert np.array_equal(np.isnan(host(loss)), marked), (V, kind, tail)
        assert np.array_equal(np.isnan(got), np.tile((marked & (w != 0))[:, None], (1, V))), (V, kind, tail)
        assert not got[2].any() and not got[5].any(), (V, kind, tail)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V", [2, 40, 1025, 9000, 131072])
def test_log_probs_whose_difference_passes_the_range(V, kind):
    """The type's largest and lowest value in one row: x - max is -6.8e38, which fp32 does not hold, (x - max) / T is a number for T
    from 2 on, and so are the log-probs."""
    rng = np.random.default_rng(V)
    x = rng.normal(0, 2, (4, V))
    x[:, 0] = -R.LARGEST[kind]
    x[0, V - 1], x[1, V - 1], x[2, V // 2] = R.LARGEST[kind], 2e38, 1e38
    x[3] = np.where(rng.random(V) < 0.5, R.LARGEST[kind], -R.LARGEST[kind])
    tokens = np.stack([np.zeros(4, int), np.full(4, V - 1), rng.integers(0, V, 4)], axis=1)
    for T in (1.0, 2.5, 100.0, 1e4):
        T = float(np.float32(T))
        buf, view, values = place(x, kind)
        o = run_logprobs(view, kind, V, V, T, dev(tokens.astype(np.int32)), min(V, 64))
        check_logprobs(o, values, T, tokens, min(V, 64), (V, kind, T))
        for r in range(4):
            assert np.isfinite(host(o["logp"][r])).all() or T == 1.0


@pytest.mark.parametrize("T", [1.0, 1.4426950408889634, 0.03, 1e-4, 500.0])
@pytest.mark.parametrize("V", [3, 40, 300, 1025, 9000, 131072])
def test_rows_across_the_line_of_far_logits(V, T):
    """Rows with ordinary logits on either side of -2^20 T ln 2: a lane that has none above it counts beside lanes that have."""
    T = float(np.float32(T))
    rng = np.random.default_rng(V)
    a = 1048576 * T / 1.4426950408889634
    x = -a + T * rng.uniform(-6, 6, (8, V))
    x[2:4] = -a + T * rng.uniform(-6, 0, (2, V))
    x[4:6] = -a + T * np.where(rng.random((2, V)) < 0.9, rng.uniform(-30, -1, (2, V)), rng.uniform(0, 3, (2, V)))
    x[6] = -a - T * 4.0
    x[6, V // 2] = -a + T
    x[7] = -2 * a + T * rng.uniform(-6, 6, V)
    buf, view, values = place(x, "f32")
    tokens = tokens_of(rng, values, 3)
    o = run_logprobs(view, "f32", V, V, T, dev(tokens.astype(np.int32)), min(V, 9))
    check_logprobs(o, values, T, tokens, min(V, 9), (V, T))
    t = np.stack([rng.permutation(V)[:3] for _ in range(8)])
    l = np.log(rng.dirichlet(np.ones(4), 8)[:, :-1]).astype(np.float32)
    for tail in (False, True):
        loss, grad = torch.full((8,), JUNK, device=DEV), torch.full((8, V), JUNK, device=DEV)
        run_distill(view, "f32", V, V, T, dev(t.astype(np.int32)), dev(l), tail, None, loss, grad, V)
        got, got_loss = host(grad), host(loss)
        for r in range(8):
            want, gr, e, eg = R.distill(values[r], T, t[r], l[r].astype(np.float64), tail, 1.0)
            R.check(got_loss[r], want, e * (1 + 2 ** -20) + R.U * abs(want) + 1e-37, (V, T, tail, r, "loss"))
            R.check(got[r], gr, R.rounded(eg, gr, "f32"), (V, T, tail, r, "grad"))
