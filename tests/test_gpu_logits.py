"""Log-probs, entropy, alternatives, their gradient and the distillation loss on the GPU against the 64-bit definitions in
logit_rows.py: rows of every length, type, stride and alignment, masked, empty, marked and padded rows, ties, rows whose
largest values crowd together, few long rows and many short ones, gradients in the logits' place, graphs, streams."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import logit_rows as R  # noqa: E402
import paper_2508_07014_amd as pb  # noqa: E402
from gpu_helpers import DEV, dev, stream_ptr  # noqa: E402

KIND = {"f32": (pb.PB_F32, torch.float32), "f16": (pb.PB_F16, torch.float16), "bf16": (pb.PB_BF16, torch.bfloat16)}
JUNK = -77.0


def place(x, kind, stride=None, shift=0):
    """Rows on the device, `shift` elements behind an aligned address, with junk between and behind them; the buffer and the
    float64 values they have in their type."""
    rows, V = x.shape
    stride = stride or V
    buf = torch.full((shift + rows * stride + 8,), JUNK, dtype=KIND[kind][1], device=DEV)
    view = torch.as_strided(buf, (rows, V), (stride, 1), shift)
    view.copy_(torch.from_numpy(x.astype(np.float32)).to(DEV))
    return buf, view, view.double().cpu().numpy()


def workspace(size):
    return torch.full((max(16, size),), 0x5a, dtype=torch.uint8, device=DEV) if size else None


def run_logprobs(view, kind, stride, V, T, tokens=None, top=0, entropy=True, stats=True, stream=None):
    rows = view.shape[0]
    M = 0 if tokens is None else tokens.shape[1]
    o = dict(logp=torch.full((rows, M), JUNK, device=DEV) if M else None, entropy=torch.full((rows,), JUNK, device=DEV) if entropy else None,
             top=torch.full((rows, top), -7, dtype=torch.int32, device=DEV) if top else None,
             top_logp=torch.full((rows, top), JUNK, device=DEV) if top else None,
             stats=torch.full((rows, 3), JUNK, device=DEV) if stats else None)
    size = pb.pb_token_logprobs_workspace_bytes(KIND[kind][0], rows, V, top)
    ws = workspace(size)
    pb.pb_token_logprobs(view, KIND[kind][0], stride, rows, V, T, tokens, M, top, o["logp"], o["entropy"], o["top"], o["top_logp"],
                         o["stats"], ws, size, stream_ptr() if stream is None else stream)
    o["ws"] = ws
    return o


def host(t):
    return t.double().cpu().numpy()


def check_logprobs(o, values, T, tokens, top, where):
    for r in range(len(values)):
        t = np.zeros(0, int) if tokens is None else tokens[r]
        w = R.logprobs(values[r], T, t, top)
        at = (where, "row", r)
        if o["logp"] is not None:
            R.check(host(o["logp"][r]), w["logp"], w["e_logp"] + R.TINY["f32"], at + ("logp",))
        if o["entropy"] is not None:
            R.check(host(o["entropy"][r]), w["entropy"], w["e_entropy"], at + ("entropy",))
        if top:
            assert np.array_equal(o["top"][r].cpu().numpy(), w["top"]), at
            R.check(host(o["top_logp"][r]), w["top_logp"], w["e_top"], at + ("top_logp",))
        if o["stats"] is not None:
            R.check(host(o["stats"][r]), w["stats"], [0.0, w["e_logs"], w["e_entropy"]], at + ("stats",))


def rows_of(rng, rows, V, kind, odd=True):
    """Rows of all sorts: plain, sure of one token, flat, masked, empty, marked, far from 0, ties, sorted, crowded."""
    x = rng.normal(0, 2.5, (rows, V))
    for r in range(rows):
        sort = int(rng.integers(0, 14)) if odd else 0
        if sort == 1:
            x[r, rng.integers(0, V)] += 30.0
        elif sort == 2:
            x[r] = 1.5
        elif sort == 3:
            x[r, rng.random(V) < 0.95] = -np.inf
        elif sort == 4:
            x[r] = -np.inf
        elif sort == 5:
            x[r, rng.integers(0, V)] = np.nan
        elif sort == 6:
            x[r, rng.integers(0, V)] = np.inf
        elif sort == 7:
            x[r] += 900.0 * (1 if rng.random() < 0.5 else -1)
        elif sort == 8:
            x[r] = np.round(x[r])
        elif sort == 9:
            x[r] = np.sort(x[r])[::int(rng.choice([-1, 1]))]
        elif sort == 10:   # the type's lowest value as a mask
            x[r, rng.random(V) < 0.9] = -R.LARGEST[kind]
        elif sort == 11:
            x[r] = -R.LARGEST[kind]
        elif sort == 12:   # a signed zero ties with the other
            x[r] = np.where(rng.random(V) < 0.5, 0.0, -0.0)
        elif sort == 13:   # the largest values in one place out of many
            x[r] -= 20.0 * (np.arange(V) % 4096 >= 8)
    return x


def tokens_of(rng, values, M, absent=True):
    rows, V = values.shape
    t = rng.integers(0, V, (rows, M))
    if absent:
        t[rng.random((rows, M)) < 0.1] = rng.choice([-1, V, 2 ** 31 - 1, -2 ** 31])
        if M > 1:
            t[:, 1] = np.where(rng.random(rows) < 0.5, t[:, 0], t[:, 1])
    return t


SIZES = [1, 2, 3, 5, 7, 8, 9, 15, 16, 17, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 500, 511, 512, 513, 1000, 1023, 1024, 1025, 1280,
         1281, 2047, 2048, 2049, 3001, 4095, 4096, 4097, 5000, 8191, 8192, 8193, 10007, 16383, 16385, 32001, 32768, 50000, 65537, 131072]


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("V", SIZES)
def test_logprobs_sizes(V, kind):
    rng = np.random.default_rng(7000 + V)
    for case in range(3):
        rows = int(rng.choice([1, 2, 5, 9])) if V < 20000 else int(rng.choice([1, 3]))
        stride, shift = V + int(rng.choice([0, 0, 3, 64])), int(rng.choice([0, 1, 2, 5]))
        T = float(rng.choice([1.0, 0.7, 2.0]))
        buf, view, values = place(rows_of(rng, rows, V, kind, case > 0), kind, stride, shift)
        M, top = int(rng.choice([0, 1, 2, 17, 64])), min(V, int(rng.choice([0, 1, 5, 20, 64])))
        tokens = tokens_of(rng, values, M) if M else None
        o = run_logprobs(view, kind, stride, V, T, None if tokens is None else dev(tokens.astype(np.int32)), top)
        check_logprobs(o, values, T, tokens, top, (V, kind, case, rows, stride, shift, T, M, top))


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("rows,V", [(70, 33), (300, 1025), (1000, 100), (130, 8192), (600, 2049), (40, 40000), (300, 9000)])
def test_logprobs_many_rows(rows, V, kind):
    rng = np.random.default_rng(rows + V)
    buf, view, values = place(rows_of(rng, rows, V, kind), kind)
    tokens = tokens_of(rng, values, 3)
    o = run_logprobs(view, kind, V, V, 1.0, dev(tokens.astype(np.int32)), 10)
    some = rng.permutation(rows)[:60]
    check_logprobs({k: None if v is None else v[torch.from_numpy(some).to(v.device)] for k, v in o.items() if k != "ws"}, values[some], 1.0,
                   tokens[some], 10, (rows, V, kind))


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("V", [600, 1025, 5000, 40000, 131072])
def test_alternatives_that_crowd(V, kind):
    """The largest values at one stride or in one run, equal or rising: more of them in one part of the row than any list of
    candidates should hold."""
    rng = np.random.default_rng(V)
    x = rng.normal(0, 1, (12, V))
    for r, step in enumerate([1, 4, 8, 64, 128, 256, 512, 1024, 2048, 4096, 8192, 16384]):
        at = np.arange(int(rng.integers(0, 16)), V, step)[:3000]
        x[r, at] = 20.0 + (0.0 if r % 3 == 0 else np.arange(len(at)) * 0.01 if r % 3 == 1 else -np.arange(len(at)) * 0.01)
    for top in (1, 20, 64):
        buf, view, values = place(x, kind)
        o = run_logprobs(view, kind, V, V, 1.0, None, top)
        check_logprobs(o, values, 1.0, None, top, (V, kind, top))


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("V", [1, 5, 40, 1025, 9000, 40000, 70001, 131072])
def test_small_log_probs_and_entropies(V, kind):
    """A token that has all but 1e-3 .. 1e-8 of a row: its log-prob and the entropy are as near, relative to themselves, as the
    probabilities of the others are (R: their sum, log p = -log(1 + R)), not only relative to 1."""
    rng = np.random.default_rng(V)
    x = np.where(rng.random((6, V)) < 30.0 / V, rng.uniform(-21, -10, (6, V)), -np.inf)
    at = np.array([0, V - 1, *rng.integers(0, V, 4)])
    x[np.arange(6), at] = np.array([0.0, 3.0, -2.0, 0.0, 5.5, 0.0])
    buf, view, values = place(x, kind)
    o = run_logprobs(view, kind, V, V, 1.0, dev(at[:, None].astype(np.int32)), min(V, 3))
    top = host(o["top_logp"])
    for r in range(6):
        d = values[r] - values[r].max()
        e = np.where(np.arange(V) == at[r], 0.0, np.exp(d))
        R_, far = e.sum(), np.abs(d[np.isfinite(d)]).max()
        off = R.U * (R.chain(V) + 16 + 8 * far)      # of every term and their sum, relative to it
        want = -np.log1p(R_)
        R.check(host(o["logp"])[r], [want], abs(want) * off, (V, kind, r, "logp"))
        R.check(top[r, :1], [want], abs(want) * off, (V, kind, r, "top"))
        H = np.log1p(R_) - (e[e > 0] * d[e > 0]).sum() / (1 + R_)
        R.check(host(o["entropy"])[r], H, H * 2 * off, (V, kind, r, "entropy"))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 5, 40, 1025, 9000, 33000, 131072])
def test_small_gradients_of_log_probs(V, kind):
    """The gradient of such a token's log-prob, R / (1 + R) on it, is as near relative to itself as R is; the others' as their
    probabilities."""
    rng = np.random.default_rng(V)
    x = np.where(rng.random((6, V)) < 30.0 / V, rng.uniform(-21, -10, (6, V)), -np.inf)
    at = np.array([0, V - 1, *rng.integers(0, V, 4)])
    x[np.arange(6), at] = np.array([0.0, 3.0, -2.0, 0.0, 5.5, 0.0])
    buf, view, values = place(x, kind)
    o = run_logprobs(view, kind, V, V, 1.0)
    g = np.array([[1.0], [-2.0], [0.5], [1.0], [3.0], [1.0]], np.float32)
    grad = torch.full((6, V), JUNK, dtype=KIND[kind][1], device=DEV)
    run_backward(view, kind, V, V, 1.0, o["stats"], dev(at[:, None].astype(np.int32)), dev(g), None, grad, V)
    for r in range(6):
        d = values[r] - values[r].max()
        e = np.where(np.arange(V) == at[r], 0.0, np.exp(d))
        R_, far = e.sum(), np.abs(d[np.isfinite(d)]).max()
        off = R.U * (R.chain(V) + 24 + 10 * far)
        want = -e / (1 + R_)
        want[at[r]] = R_ / (1 + R_)
        want *= g[r, 0]
        R.check(host(grad)[r], want, np.abs(want) * (off + R.HALF_STEP[kind]) + R.TINY[kind], (V, kind, r))


def test_widest_rows():
    V = 393216
    rng = np.random.default_rng(5)
    buf, view, values = place(rng.normal(0, 3, (2, V)), "bf16")
    tokens = np.array([[0, V - 1], [V, 7]])
    o = run_logprobs(view, "bf16", V, V, 1.0, dev(tokens.astype(np.int32)), 64)
    check_logprobs(o, values, 1.0, tokens, 64, V)
    t, l = teacher(rng, values, 64, 1.0)
    check_distill(rng, view, values, "bf16", V, 1.0, t, l, True, V)


def test_only_what_is_asked_for():
    rng = np.random.default_rng(3)
    buf, view, values = place(rows_of(rng, 6, 1025, "f32"), "f32")
    tokens = tokens_of(rng, values, 2)
    for M, top, ent, st in ((0, 0, True, False), (0, 0, False, True), (2, 0, False, False), (0, 3, False, False), (2, 3, False, True)):
        o = run_logprobs(view, "f32", 1025, 1025, 1.0, dev(tokens.astype(np.int32)) if M else None, top, ent, st)
        check_logprobs(o, values, 1.0, tokens if M else None, top, (M, top, ent, st))


# ---- gradient --------------------------------------------------------------------------------------------------------

def run_backward(view, kind, stride, V, T, stats, tokens, g, h, grad, grad_stride, stream=None):
    pb.pb_token_logprobs_backward(view, KIND[kind][0], stride, view.shape[0], V, T, stats, tokens, 0 if tokens is None else tokens.shape[1],
                                  g, h, grad, grad_stride, stream_ptr() if stream is None else stream)


def check_rows_behind(buf, shift, rows, stride, V):
    """Nothing but the rows was written."""
    flat = buf.double().cpu().numpy()
    keep = np.ones(len(flat), bool)
    for r in range(rows):
        keep[shift + r * stride:shift + r * stride + V] = False
    assert (flat[keep] == JUNK).all()


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("V", SIZES)
def test_backward_sizes(V, kind):
    rng = np.random.default_rng(9000 + V)
    for case in range(3):
        rows = int(rng.choice([1, 2, 5, 9])) if V < 20000 else int(rng.choice([1, 3]))
        stride, shift = V + int(rng.choice([0, 0, 3, 64])), int(rng.choice([0, 1, 2, 5]))
        T, M = float(rng.choice([1.0, 0.7, 2.0])), int(rng.choice([0, 1, 2, 17, 64]))
        buf, view, values = place(rows_of(rng, rows, V, kind, case > 0), kind, stride, shift)
        tokens = tokens_of(rng, values, M) if M else None
        g = rng.normal(0, 1, (rows, M)).astype(np.float32)
        h = rng.normal(0, 1, rows).astype(np.float32) if M == 0 or case != 1 else None
        if case == 2 and rows > 1:
            g[1:3], h[1:3] = 0.0, 0.0
        elif M:
            g[(tokens < 0) | (tokens >= V)] = np.nan    # (not looked at)
        d_tok = None if tokens is None else dev(tokens.astype(np.int32))
        stats = run_logprobs(view, kind, stride, V, T)["stats"]
        gs, gshift = V + int(rng.choice([0, 0, 5])), int(rng.choice([0, 1, 4]))
        gbuf = torch.full((gshift + rows * gs + 8,), JUNK, dtype=KIND[kind][1], device=DEV)
        grad = torch.as_strided(gbuf, (rows, V), (gs, 1), gshift)
        args = (d_tok, dev(g) if M else None, None if h is None else dev(h))
        run_backward(view, kind, stride, V, T, stats, *args, grad, gs)
        got = host(grad)
        for r in range(rows):
            t = tokens[r] if M else np.zeros(0, int)
            want, err = R.logprobs_grad(values[r], T, t, g[r].astype(np.float64), 0.0 if h is None else float(h[r]))
            R.check(got[r], want, R.rounded(err, want, kind), (V, kind, case, rows, stride, shift, gs, gshift, T, M, r))
        check_rows_behind(gbuf, gshift, rows, gs, V)
        run_backward(view, kind, stride, V, T, stats, *args, view, stride)   # in the logits' place: the same bits
        assert np.array_equal(host(view), got, equal_nan=True)
        check_rows_behind(buf, shift, rows, stride, V)


# ---- distillation ----------------------------------------------------------------------------------------------------

def teacher(rng, values, K, T, absent=0.0, twice=False):
    rows, V = values.shape
    t, l = np.zeros((rows, K), np.int64), np.zeros((rows, K), np.float32)
    for r in range(rows):
        x = np.where(np.isfinite(values[r]) & (np.abs(values[r]) < 1e4), values[r], 0.0) + rng.normal(0, 1, V)
        lp, _ = R.row_log_probs(x, T)
        first = np.argsort(-lp)[:K]
        t[r, :len(first)], l[r, :len(first)] = first, lp[first]
        t[r, len(first):] = -1
    if twice and K > 1 and V > 1:
        t[:, 1] = t[:, 0]
        l[:, :2] = l[:, :2].min(axis=1, keepdims=True) - 1.0
    gone = rng.random((rows, K)) < absent
    t[gone] = rng.choice([-1, V, 2 ** 31 - 1])
    l[gone] = np.nan
    return t, l


def run_distill(view, kind, stride, V, T, t, l, tail, w, loss, grad, gs, stream=None):
    rows = view.shape[0]
    size = pb.pb_distill_topk_workspace_bytes(KIND[kind][0], rows, V, t.shape[1])
    ws = workspace(size)
    pb.pb_distill_topk(view, KIND[kind][0], stride, rows, V, T, t, l, t.shape[1], pb.PB_DISTILL_TAIL if tail else pb.PB_DISTILL_RENORM, w,
                       loss, grad, gs, ws, size, stream_ptr() if stream is None else stream)
    return ws


def check_distill(rng, view, values, kind, stride, T, t, l, tail, where, weights=True):
    rows, V = values.shape
    w = rng.normal(0, 1, rows).astype(np.float32)
    if rows > 2:
        w[1] = 0.0
    d_w = dev(w) if weights else None
    if not weights:
        w[:] = 1.0
    gs, gshift = V + int(rng.choice([0, 0, 5])), int(rng.choice([0, 1, 4]))
    gbuf = torch.full((gshift + rows * gs + 8,), JUNK, dtype=KIND[kind][1], device=DEV)
    grad = torch.as_strided(gbuf, (rows, V), (gs, 1), gshift)
    loss = torch.full((rows,), JUNK, device=DEV)
    d_t, d_l = dev(t.astype(np.int32)), dev(l)
    run_distill(view, kind, stride, V, T, d_t, d_l, tail, d_w, loss, grad, gs)
    got, got_loss = host(grad), host(loss)
    for r in range(rows):
        want, g, e, eg = R.distill(values[r], T, t[r], l[r].astype(np.float64), tail, float(w[r]))
        R.check(got_loss[r], want, e * (1 + 2 ** -20) + R.U * abs(want) + 1e-37, (where, r, "loss"))
        R.check(got[r], g, R.rounded(eg, g, kind), (where, r, "grad"))
    check_rows_behind(gbuf, gshift, rows, gs, V)
    only = torch.full((rows,), JUNK, device=DEV)
    run_distill(view, kind, stride, V, T, d_t, d_l, tail, d_w, only, None, 0)          # the loss alone, the gradient alone
    assert np.array_equal(host(only), got_loss, equal_nan=True)
    grad.fill_(JUNK)
    run_distill(view, kind, stride, V, T, d_t, d_l, tail, d_w, None, grad, gs)
    assert np.array_equal(host(grad), got, equal_nan=True)
    run_distill(view, kind, stride, V, T, d_t, d_l, tail, d_w, only, view, stride)     # in the logits' place
    assert np.array_equal(host(view), got, equal_nan=True) and np.array_equal(host(only), got_loss, equal_nan=True)


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("V", SIZES)
def test_distill_sizes(V, kind):
    rng = np.random.default_rng(11000 + V)
    for case in range(4):
        rows = int(rng.choice([1, 2, 5, 9])) if V < 20000 else int(rng.choice([1, 3]))
        stride, shift = V + int(rng.choice([0, 0, 3, 64])), int(rng.choice([0, 1, 2, 5]))
        T, K = float(rng.choice([1.0, 0.7, 2.0])), int(rng.choice([1, 2, 8, 33, 64]))
        buf, view, values = place(rows_of(rng, rows, V, kind, case > 1), kind, stride, shift)
        t, l = teacher(rng, values, K, T, [0.0, 0.3, 0.3, 0.9][case], case == 1)
        if case == 2:
            t[-1] = -1                                  # a row of padding
            l[0, 0] = -np.inf                           # an entry without mass
        check_distill(rng, view, values, kind, stride, T, t, l, case % 2 == 0, (V, kind, case, rows, stride, shift, T, K), case != 1)
        check_rows_behind(buf, shift, rows, stride, V)


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("rows,V,K", [(70, 33, 8), (300, 1025, 8), (130, 8192, 16), (40, 40000, 32), (300, 9000, 5)])
def test_distill_many_rows(rows, V, K, tail, kind):
    rng = np.random.default_rng(rows + V)
    buf, view, values = place(rows_of(rng, rows, V, kind), kind)
    t, l = teacher(rng, values, K, 1.0, 0.1)
    check_distill(rng, view, values, kind, V, 1.0, t, l, tail, (rows, V, K, tail, kind))


@pytest.mark.parametrize("rows,V", [(9, 40), (9, 9000), (9, 70000), (9, 131072)])
def test_entries_that_are_no_numbers(rows, V):
    """An entry of NaN, of either sign, or +inf: loss and gradient are NaN (in the last case too where nothing else is listed);
    the rows beside it are what they are without it."""
    g = torch.Generator(device=DEV)
    g.manual_seed(V)
    view = torch.randn((rows, V), generator=g, device=DEV)
    t = torch.arange(5, dtype=torch.int32, device=DEV).repeat(rows, 1)
    l = torch.full((rows, 5), -2.0, device=DEV)
    nans = np.array([0x7fc00000, 0xffc00000, 0x7f800001, 0xff800001, 0x7f800000], np.uint32).view(np.float32)
    for tail in (False, True):
        out = []
        for odd in (False, True):
            k, listed = l.clone(), t.clone()
            if odd:
                k[1:6, 2] = dev(nans)
                listed[3, :2] = listed[3, 3:] = -1        # (nothing but that entry)
            loss, grad = torch.empty(rows, device=DEV), torch.empty((rows, V), device=DEV)
            run_distill(view, "f32", V, V, 1.0, listed, k, tail, None, loss, grad, V)
            out.append((host(loss), host(grad)))
        assert np.isnan(out[1][0][1:6]).all() and np.isnan(out[1][1][1:6]).all()
        for a, b in zip(*out):
            assert np.array_equal(a[[0, 6, 7, 8]], b[[0, 6, 7, 8]]) and np.isfinite(a).all()


# Rows of every kernel shape, as many as send the call there (the shape is chosen by vectors a row and rows): 8 rows of each
# call are compared.
MANY = [(1100, 4104), (1030, 6001), (1025, 16400), (70, 8200), (70, 20001), (70, 30000), (70, 33001), (70, 50000), (70, 70001),
        (170, 70000), (170, 131072), (72, 131072), (73, 131072), (30, 100001), (9, 300000), (300, 33000), (20, 41000), (64, 50001), (160, 70001), (260, 70001), (5000, 1030), (20, 30001),
        (90, 72000)]


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("rows,V", MANY)
def test_kernel_shapes(rows, V, kind):
    rng = np.random.default_rng(rows + V)
    some = np.unique(np.concatenate([[0, rows - 1], rng.integers(0, rows, 6)]))
    g = torch.Generator(device=DEV)
    g.manual_seed(rows + V)
    x = 2.5 * torch.randn((rows, V), generator=g, device=DEV)
    x[torch.from_numpy(some).to(DEV)] = dev(rows_of(rng, len(some), V, kind).astype(np.float32))
    shift = int(rng.integers(0, 8))
    buf = torch.full((shift + rows * V,), JUNK, dtype=KIND[kind][1], device=DEV)
    view = torch.as_strided(buf, (rows, V), (V, 1), shift)
    view.copy_(x)
    at = torch.from_numpy(some).to(DEV)
    values = host(view[at])
    tokens = tokens_of(rng, values, 2)
    all_tokens = rng.integers(0, V, (rows, 2))
    all_tokens[some] = tokens
    d_tokens = dev(all_tokens.astype(np.int32))
    for top, ent in ((0, True), (20, True), (7, False)):
        o = run_logprobs(view, kind, V, V, 1.0, d_tokens, top, ent, ent)
        check_logprobs({k: None if v is None else v[at] for k, v in o.items() if k != "ws"}, values, 1.0, tokens, top, (rows, V, kind, top))
    stats = run_logprobs(view, kind, V, V, 1.0)["stats"]
    gl, ge = rng.normal(0, 1, (rows, 2)).astype(np.float32), rng.normal(0, 1, rows).astype(np.float32)
    grad = torch.full_like(buf, JUNK)
    out = torch.as_strided(grad, (rows, V), (V, 1), shift)
    run_backward(view, kind, V, V, 1.0, stats, d_tokens, dev(gl), dev(ge), out, V)
    got = host(out[at])
    for i, r in enumerate(some):
        want, err = R.logprobs_grad(values[i], 1.0, tokens[i], gl[r].astype(np.float64), float(ge[r]))
        R.check(got[i], want, R.rounded(err, want, kind), (rows, V, kind, r))
    t, l = teacher(rng, values, 17, 1.0, 0.1)
    all_t, all_l = rng.integers(0, V, (rows, 17)), np.full((rows, 17), -4.0, np.float32)
    all_t[some], all_l[some] = t, l
    w = rng.normal(0, 1, rows).astype(np.float32)
    for tail in (False, True):
        loss = torch.full((rows,), JUNK, device=DEV)
        out.fill_(JUNK)
        run_distill(view, kind, V, V, 1.0, dev(all_t.astype(np.int32)), dev(all_l), tail, dev(w), loss, out, V)
        got, got_loss = host(out[at]), host(loss[at])
        for i, r in enumerate(some):
            want, gr, e, eg = R.distill(values[i], 1.0, t[i], l[i].astype(np.float64), tail, float(w[r]))
            R.check(got_loss[i], want, e * (1 + 2 ** -20) + R.U * abs(want) + 1e-37, (rows, V, kind, tail, r))
            R.check(got[i], gr, R.rounded(eg, gr, kind), (rows, V, kind, tail, r))
        assert not bool((out == JUNK).any())      # every element of every row was written


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_tensors_past_the_last_cache(kind):
    """Logits and gradients that do not fit in 256 MB together go past the caches: the same results as for a part of the rows."""
    V, rows = 17001, 4200
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    view = (2.5 * torch.randn((rows, V), generator=g, device=DEV)).to(KIND[kind][1])
    rng = np.random.default_rng(8)
    t = dev(np.stack([rng.permutation(V)[:9] for _ in range(rows)]).astype(np.int32))
    l = torch.full((rows, 9), -3.0, device=DEV)
    tok, ones = t[:, :1].contiguous(), torch.ones((rows, 1), device=DEV)
    stats = run_logprobs(view, kind, V, V, 1.0, tok)["stats"]
    whole, loss = [torch.empty_like(view) for _ in range(2)], torch.empty(rows, device=DEV)
    run_backward(view, kind, V, V, 1.0, stats, tok, ones, None, whole[0], V)
    run_distill(view, kind, V, V, 1.0, t, l, True, None, loss, whole[1], V)
    for lo, hi in ((0, 500), (3700, 4200)):
        part, some = [torch.empty_like(view[lo:hi]) for _ in range(2)], torch.empty(hi - lo, device=DEV)
        run_backward(view[lo:hi], kind, V, V, 1.0, stats[lo:hi], tok[lo:hi], ones, None, part[0], V)
        run_distill(view[lo:hi], kind, V, V, 1.0, t[lo:hi], l[lo:hi], True, None, some, part[1], V)
        assert torch.equal(part[0], whole[0][lo:hi]) and torch.equal(part[1], whole[1][lo:hi]) and torch.equal(some, loss[lo:hi])


@pytest.mark.parametrize("tail", [False, True])
def test_lists_that_cover_the_row(tail):
    """Every token listed, every token but one, all tokens with mass listed: nothing, or little, is left for the rest."""
    rng = np.random.default_rng(2)
    for V, masked in ((1, 0), (2, 0), (40, 0), (64, 0), (64, 30), (65, 0)):
        x = rng.normal(0, 2, (4, V))
        x[:, V - masked:] = -np.inf
        buf, view, values = place(x, "f32")
        K = min(64, V - masked)
        t, l = np.tile(rng.permutation(V - masked)[:K], (4, 1)), np.zeros((4, K), np.float32)
        for r in range(4):
            l[r] = R.row_log_probs(rng.normal(0, 1, V), 1.0)[0][t[r]]
        check_distill(rng, view, values, "f32", V, 1.0, t, l, tail, (V, masked))


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("V", [40, 1025, 9000, 70000])
def test_little_mass_for_the_rest_and_large_weights(V, kind):
    """A student that leaves e^-80 to the tokens that are not listed, most of them masked, rows weighted by a loss scale: q' / p'
    times the weight passes the fp32 range, the gradient does not."""
    rng = np.random.default_rng(V)
    for T in (1.0, 0.01):
        x = np.full((5, V), -np.inf)
        t = np.stack([rng.permutation(V)[:13] for _ in range(5)])
        for r in range(5):
            x[r, t[r]] = np.concatenate([rng.normal(0, 1, 8), rng.uniform(-82, -79, 5)]) * T
        buf, view, values = place(x, kind)
        t, l = t[:, :8], np.log(rng.dirichlet(np.ones(9), 5)[:, :8]).astype(np.float32)
        w = np.array([30000.0, -20000.0, 1.0, 0.25, 10000.0], np.float32) * np.float32(T)
        grad, loss = torch.full((5, V), JUNK, dtype=KIND[kind][1], device=DEV), torch.full((5,), JUNK, device=DEV)
        run_distill(view, kind, V, V, T, dev(t.astype(np.int32)), dev(l), True, dev(w), loss, grad, V)
        got, got_loss = host(grad), host(loss)
        for r in range(5):
            want, g, e, eg = R.distill(values[r], T, t[r], l[r].astype(np.float64), True, float(w[r]))
            R.check(got_loss[r], want, e * (1 + 2 ** -20) + R.U * abs(want) + 1e-37, (V, kind, T, r, "loss"))
            R.check(got[r], g, R.rounded(eg, g, kind), (V, kind, T, r, "grad"))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 5, 40, 1025, 9000, 33000, 70001, 131072])
def test_small_losses_and_gradients(V, kind):
    """The student has all but 1e-3 .. 1e-8 of a row on the one token that the teacher lists: loss log(1 + R) and gradient
    -R / (1 + R) on it are as near, relative to themselves, as R, the sum of the others, is."""
    rng = np.random.default_rng(V)
    x = np.where(rng.random((6, V)) < 30.0 / V, rng.uniform(-21, -10, (6, V)), -np.inf)
    at = np.array([0, V - 1, *rng.integers(0, V, 4)])
    x[np.arange(6), at] = np.array([0.0, 3.0, -2.0, 0.0, 5.5, 0.0])
    buf, view, values = place(x, kind)
    for tail in (False, True):
        loss, grad = torch.full((6,), JUNK, device=DEV), torch.full((6, V), JUNK, dtype=KIND[kind][1], device=DEV)
        run_distill(view, kind, V, V, 1.0, dev(at[:, None].astype(np.int32)), torch.zeros((6, 1), device=DEV), tail, None, loss, grad, V)
        for r in range(6):
            d = values[r] - values[r].max()
            e = np.where(np.arange(V) == at[r], 0.0, np.exp(d))
            R_, far = e.sum(), np.abs(d[np.isfinite(d)]).max()
            off = R.U * (R.chain(V) + 20 + 8 * far)
            R.check(host(loss)[r], np.log1p(R_), np.log1p(R_) * off, (V, kind, tail, r, "loss"))
            want = e / (1 + R_)
            want[at[r]] = -R_ / (1 + R_)
            R.check(host(grad)[r], want, np.abs(want) * (off + R.HALF_STEP[kind]) + R.TINY[kind], (V, kind, tail, r, "grad"))


# ---- together ----------------------------------------------------------------------------------------------------------

def test_confidence_of_what_a_decoder_emits_and_a_student_of_the_boosted_rows():
    """Greedy steps of the boosted decoder; the confidence of its tokens; the boosted rows' alternatives kept as a teacher; a
    student's loss and gradient on them; the tokens' own gradient."""
    import pb_workloads as W
    cfg = W.CONFIGS[1]
    toks, offs = W.make_phrases(cfg)
    V, B, steps, alpha, top = cfg.vocab_size, 4, 6, 0.5, 8
    tree = pb.pb_build(toks, offs, V, cfg.blank_id, device=0)
    logp = W.make_logp(cfg, steps=steps, batch=B, planting=W.Planting(toks, offs, cover=0.5))
    rng = np.random.default_rng(1)
    student = rng.normal(0, 2, (steps * B, V))
    s_buf, s_view, s_values = place(student, "bf16")
    states = torch.zeros(B, dtype=torch.int32, device=DEV)
    tokens = torch.empty((steps, B), dtype=torch.int32, device=DEV)
    fused = torch.empty((steps, B, V), device=DEV)
    score = torch.empty(B, device=DEV)
    boost = torch.empty((B, V), device=DEV)
    d_logp = dev(logp)
    for t in range(steps):
        pb.pb_score(tree, states, B, boost, None, stream_ptr())
        torch.add(d_logp[t], boost, alpha=alpha, out=fused[t])
        pb.pb_fuse_step(tree, d_logp[t], V, states, alpha, B, tokens[t], states, score, stream_ptr())
    rows = fused.reshape(steps * B, V)
    flat = tokens.reshape(-1, 1)
    kept = run_logprobs(rows, "f32", V, V, 1.0, flat, top)
    values = rows.double().cpu().numpy()
    check_logprobs(kept, values, 1.0, flat.cpu().numpy(), top, "teacher")
    assert np.array_equal(kept["top"][:, 0].cpu().numpy(), flat[:, 0].cpu().numpy())     # the greedy token comes first
    assert np.array_equal(host(kept["top_logp"][:, 0]), host(kept["logp"][:, 0]))
    for tail in (False, True):
        loss, grad = torch.empty(steps * B, device=DEV), torch.empty((steps * B, V), dtype=torch.bfloat16, device=DEV)
        run_distill(s_view, "bf16", V, V, 1.0, kept["top"], kept["top_logp"], tail, None, loss, grad, V)
        t, l = kept["top"].cpu().numpy(), host(kept["top_logp"])
        for r in range(steps * B):
            want, g, e, eg = R.distill(s_values[r], 1.0, t[r], l[r], tail, 1.0)
            R.check(host(loss[r]), want, e + R.U * abs(want), (tail, r))
            R.check(host(grad[r]), g, R.rounded(eg, g, "bf16"), (tail, r))
    g = torch.full((steps * B, 1), 1.0 / B, device=DEV)
    back = torch.empty_like(rows)
    run_backward(rows, "f32", V, V, 1.0, kept["stats"], flat, g, None, back, V)
    for r in range(steps * B):
        want, err = R.logprobs_grad(values[r], 1.0, flat[r].cpu().numpy(), np.full(1, float(np.float32(1.0 / B))), 0.0)
        R.check(host(back[r]), want, R.rounded(err, want, "f32"), r)
    pb.pb_free(tree)


@pytest.mark.parametrize("V", [40, 1025, 9000])
def test_gradient_is_a_difference_quotient_of_the_loss(V):
    """The loss along a direction u, both from the kernel: (L(x + s u) - L(x - s u)) / 2s against the gradient times u.  L is
    off by e (its bound above) on either side, so the quotient by e / s; its third derivative along u is at most
    6 max|u|^3, times s^2 / 6; the gradient's bound enters with |u|."""
    rng = np.random.default_rng(V)
    x = rng.normal(0, 2, (1, V))
    t, l = teacher(rng, x, 8, 1.0)
    u = rng.normal(0, 1, V) / 4
    s = 0.05
    out = []
    for k in (-1, 0, 1):
        buf, view, values = place(x + k * s * u, "f32")
        loss, grad = torch.empty(1, device=DEV), torch.empty((1, V), device=DEV)
        run_distill(view, "f32", V, V, 1.0, dev(t.astype(np.int32)), dev(l), True, None, loss, grad, V)
        _, _, e, eg = R.distill(values[0], 1.0, t[0], l[0].astype(np.float64), True, 1.0)
        out.append((float(host(loss)[0]), host(grad)[0], e + R.U, eg, values[0]))
    step = (out[2][4] - out[0][4]) / (2 * s)           # (the direction that the rounded inputs took)
    slope = (out[2][0] - out[0][0]) / (2 * s)
    bound = (out[0][2] + out[2][2]) / (2 * s) + np.abs(u).max() ** 3 * s * s + (out[1][3] * np.abs(u)).sum() + 1e-6
    assert abs(slope - float(out[1][1] @ step)) <= bound


SHAPES = [(3, 1025, "f32"), (2, 131072, "bf16"), (700, 257, "f16"), (64, 50000, "bf16"), (300, 9000, "f32")]


def _bundle(rng, rows, V, kind):
    buf, view, values = place(rows_of(rng, rows, V, kind, False), kind)
    t, l = teacher(rng, values[:1], 6, 1.0)
    t, l = np.tile(t, (rows, 1)), np.tile(l, (rows, 1))
    d = dict(view=view, tokens=dev(tokens_of(rng, values, 1, False).astype(np.int32)), t=dev(t.astype(np.int32)), l=dev(l),
             g=torch.ones((rows, 1), device=DEV), grad=torch.empty_like(view.contiguous()), grad2=torch.empty_like(view.contiguous()),
             loss=torch.empty(rows, device=DEV), o=dict(logp=torch.empty((rows, 1), device=DEV), entropy=torch.empty(rows, device=DEV),
                                                        top=torch.empty((rows, 7), dtype=torch.int32, device=DEV),
                                                        top_logp=torch.empty((rows, 7), device=DEV), stats=torch.empty((rows, 3), device=DEV)))
    k = KIND[kind][0]
    d["n1"], d["n2"] = pb.pb_token_logprobs_workspace_bytes(k, rows, V, 7), pb.pb_distill_topk_workspace_bytes(k, rows, V, 6)
    d["ws1"], d["ws2"] = workspace(max(16, d["n1"])), workspace(max(16, d["n2"]))
    return d


def _all_calls(d, kind, V, stream):
    k, rows, o = KIND[kind][0], d["view"].shape[0], d["o"]
    pb.pb_token_logprobs(d["view"], k, V, rows, V, 1.0, d["tokens"], 1, 7, o["logp"], o["entropy"], o["top"], o["top_logp"], o["stats"],
                         d["ws1"], d["n1"], stream)
    pb.pb_token_logprobs_backward(d["view"], k, V, rows, V, 1.0, o["stats"], d["tokens"], 1, d["g"], None, d["grad"], V, stream)
    pb.pb_distill_topk(d["view"], k, V, rows, V, 1.0, d["t"], d["l"], 6, pb.PB_DISTILL_TAIL, None, d["loss"], d["grad2"], V, d["ws2"], d["n2"],
                       stream)


def _outputs(d):
    return [host(x) for x in list(d["o"].values()) + [d["grad"], d["grad2"], d["loss"]]]


@pytest.mark.parametrize("rows,V,kind", SHAPES)
def test_captured_and_replayed(rows, V, kind):
    rng = np.random.default_rng(V)
    d, other = _bundle(rng, rows, V, kind), _bundle(rng, rows, V, kind)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        _all_calls(d, kind, V, int(side.cuda_stream))          # (before the capture: code is loaded)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _all_calls(d, kind, V, stream_ptr())
    for step in range(3):
        d["view"].copy_(dev(rows_of(rng, rows, V, kind, False).astype(np.float32)))
        for x in list(d["o"].values()) + [d["grad"], d["grad2"], d["loss"]]:
            x.fill_(-3)
        d["ws1"].fill_(step + 1)
        d["ws2"].fill_(step + 1)
        graph.replay()
        _all_calls(other, kind, V, stream_ptr())               # (eager work of its own between the replays)
        torch.cuda.synchronize()
        got = _outputs(d)
        _all_calls(d, kind, V, stream_ptr())
        torch.cuda.synchronize()
        for a, b in zip(got, _outputs(d)):
            assert np.array_equal(a, b, equal_nan=True), (rows, V, kind, step)


@pytest.mark.parametrize("rows,V,kind", SHAPES)
def test_two_streams_at_once(rows, V, kind):
    rng = np.random.default_rng(V + 1)
    both = [_bundle(rng, rows, V, kind) for _ in range(2)]
    want = []
    for d in both:
        _all_calls(d, kind, V, stream_ptr())
        torch.cuda.synchronize()
        want.append(_outputs(d))
        for x in list(d["o"].values()) + [d["grad"], d["grad2"], d["loss"]]:
            x.fill_(-3)
    streams = [torch.cuda.Stream() for _ in both]
    torch.cuda.synchronize()
    for _ in range(5):
        for d, s in zip(both, streams):
            _all_calls(d, kind, V, int(s.cuda_stream))
    torch.cuda.synchronize()
    for d, w in zip(both, want):
        for a, b in zip(_outputs(d), w):
            assert np.array_equal(a, b, equal_nan=True)


def test_rows_past_32_bits():
    """Rows whose offsets in elements and bytes do not fit 32 bits: the last row of a buffer of 2^32 + elements."""
    V, stride, rows, kind = 1025, 1 << 26, 70, "f16"
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("not enough memory")
    rng = np.random.default_rng(0)
    buf = torch.empty(rows * stride, dtype=torch.float16, device=DEV)
    view = torch.as_strided(buf, (rows, V), (stride, 1))
    x = rows_of(rng, rows, V, kind, False).astype(np.float32)
    view.copy_(dev(x))
    values = x.astype(np.float16).astype(np.float64)
    tokens = rng.integers(0, V, (rows, 2))
    d_tokens = dev(tokens.astype(np.int32))
    o = run_logprobs(view, kind, stride, V, 1.0, d_tokens, 5)
    check_logprobs(o, values, 1.0, tokens, 5, "far rows")
    g, l = torch.ones((rows, 2), device=DEV), torch.full((rows, 2), -1.5, device=DEV)
    loss = torch.empty(rows, device=DEV)
    run_backward(view, kind, stride, V, 1.0, o["stats"], d_tokens, g, None, view, stride)
    got = host(view)
    for r in range(rows):
        want, err = R.logprobs_grad(values[r], 1.0, tokens[r], np.ones(2), 0.0)
        R.check(got[r], want, R.rounded(err, want, kind), r)
    view.copy_(dev(x))
    run_distill(view, kind, stride, V, 1.0, d_tokens, l, True, None, loss, view, stride)
    got, got_loss = host(view), host(loss)
    for r in range(rows):
        want, grad, e, eg = R.distill(values[r], 1.0, tokens[r], np.full(2, -1.5), True, 1.0)
        R.check(got_loss[r], want, e + R.U * abs(want), r)
        R.check(got[r], grad, R.rounded(eg, grad, kind), r)
