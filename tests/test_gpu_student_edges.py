"""More of the calls around a student on the GPU: handles that are gone, log-probs of near-certain tokens, what
is left of rows that differ in two places, sums that are exact, sums of few terms, the largest layouts of the verification, sets past the last cache,
subnormal numbers, temperatures at their ends, gradients that are not finite, nothing but absent tokens."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import logit_rows as R  # noqa: E402
import paper_2508_07014_amd as pb  # noqa: E402
import student as S  # noqa: E402
from gpu_helpers import DEV, dev, stream_ptr  # noqa: E402
from test_gpu_logits import JUNK, KIND, host, place  # noqa: E402
from test_gpu_student import block, check_verify, numbers_of, rows_for, run_backward, run_norm, run_verify, set_of, tokens_for, tokens_of  # noqa: E402


def test_a_closed_set_to_write_to_is_refused():
    x, y, norm = torch.arange(1.0, 9.0, device=DEV), torch.zeros(8, device=DEV), torch.full((1,), 8.0, device=DEV)
    grads, out = (pb.pb_tensors_build([t], [8], [pb.PB_F32]) for t in (x, y))
    before = x.clone()
    pb.pb_tensors_free(out)
    with pytest.raises(pb.PbError) as e:
        pb.pb_grad_clip(grads, norm, 1.0, out, stream_ptr())
    assert e.value.code == pb.PB_EINVAL and torch.equal(x, before) and not y.any()
    grads.close()
    with pytest.raises(pb.PbError) as e:
        pb.pb_grad_clip(grads, norm, 1.0, None, stream_ptr())
    assert e.value.code == pb.PB_EINVAL and torch.equal(x, before)


def beside_error(x, T):
    """How far a log-prob may be off by what an fp32 evaluation of the row's tokens below its largest is: each exponent t by three
    roundings, 3 ln 2 |t| U of its weight, an exponential by 2 U and its sum by 13 additions one after the other (17 with two to spare); a
    weight below 2^-126 is none.  From 2^-20 on the sum may be one in 64 bits with the largest one's 1 in it, which leaves 2^-30 of it."""
    t = (x - x.max()) / T / np.log(2.0)
    e = np.where(t < 0, np.exp2(t), 0.0)
    return (e * ((2.1 * -np.maximum(t, -1e4) + 17.0) * S.U + 2.0 ** -30)).sum() + len(x) * 2.0 ** -126


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("V,n,sure", [(600, 2, False), (600, 2, True), (600, 0, True), (9001, 3, False), (16001, 3, True), (40000, 2, False), (131072, 1, False), (40000, 2, True),
                                      (90000, 8, True), (40000, 0, True), (131072, 0, True)])
def test_log_probs_of_near_certain_tokens(V, n, sure, kind):
    """Everything else lies by up to 82 below the largest logit (one, or three of the same): the log-prob is the others' weight, not the 0 that its sum
    with 1 leaves.  Of accepted tokens and of drawn ones, behind a full draft and behind a refusal."""
    rng = np.random.default_rng(V + n)
    gaps = [6.0, 12.0, 18.0, 21.0, 26.0, 33.0, 41.0, 55.0, 70.0, 82.0]
    B, T = 2 * len(gaps), 1.0
    x = np.empty((B, n + 1, V))
    for b in range(B):
        x[b] = -gaps[b // 2] + rng.uniform(-1.5, 1.5, (n + 1, V))
    top = rng.integers(3, V, (B, n + 1))
    np.put_along_axis(x, top[:, :, None], 0.0, 2)
    x[3, :, :3] = 0.0  # (and two with four of them)
    x[13, :, :3] = 0.0
    y = x[:, :n].copy()
    tokens, numbers = top[:, :n].copy(), np.full((B, n + 1), 0.25)
    if n:  # (every other sequence: the draft is sure of another token, which is refused)
        tokens[::2, n - 1] = (top[::2, n - 1] + 1) % V
        y[::2, n - 1] = -30.0
        np.put_along_axis(y[::2, n - 1], tokens[::2, n - 1:], 0.0, 1)
    bx, px, xv = block(x, kind, V, (n + 1) * V)
    py, yv = None, None
    if n and not sure:
        by, py, yv = block(y, kind, V, n * V)
    out, acc, lp = run_verify(px, py, kind, (V, (n + 1) * V), (V, n * V), B, n, V, T, T, tokens, numbers)
    for b in range(B):
        want, k, want_lp = S.verify(xv[b], None if yv is None else yv[b], T, T, tokens[b], numbers[b])
        assert acc[b] == k and np.array_equal(out[b], want), (b, out[b], want)
        for i in range(k + 1):
            # (beside that the last rounding, and 64 bits' of the difference from the largest and of the logarithm of how many there are)
            room = S.U * abs(want_lp[i]) + beside_error(xv[b, i], T) + 2.0 ** -50 * (abs(xv[b, i, want[i]]) + (xv[b, i] == 0).sum() - 1)
            assert abs(lp[b, i] - want_lp[i]) <= room, (b, i, lp[b, i], want_lp[i], room)


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("V", [40, 600, 5000, 20011, 131072])
def test_rows_that_differ_in_two_places(V, kind):
    """A draft's row is the target's with two logits exchanged: p = q but for these, and nothing but the one that has more of the target's is left,
    though the two sums are of other orders and differ in their last bits.  A number of 0, at which the first token with any rest is drawn, finds it too."""
    rng = np.random.default_rng(V)
    B = 12
    x = rng.normal(0, 2, (B, 2, V))
    at = np.array([rng.permutation(np.arange(V // 2, V))[:2] for _ in range(B)])
    for b in range(B):
        x[b, 0, at[b]] = [3.0, 1.5]
    y = x[:, :1].copy()
    for b in range(B):
        y[b, 0, at[b]] = [1.5, 3.0]
    bx, px, xv = block(x, kind, V, 2 * V)
    by, py, yv = block(y, kind, V + 3, V + 3, 1)
    for w in (0.0, 0.5, S.BELOW_1):
        numbers = np.tile([0.5, w], (B, 1))  # (p / q = e^-1.5)
        out, acc, lp = run_verify(px, py, kind, (V, 2 * V), (V + 3, V + 3), B, 1, V, 1.0, 1.0, at[:, 1:], numbers)
        assert not acc.any() and np.array_equal(out[:, 0], at[:, 0]), (w, out[:, 0], at[:, 0])


@pytest.mark.parametrize("n,V,dim,hot", [(500, 1025, 640, 0.9), (1000, 3000, 64, 0.5), (4096, 4096, 64, 0.9), (16384, 1000, 64, 0.9), (16384, 166, 3, 0.5),   # a workgroup a token
                                         (1024, 32001, 320, 0.9), (1000, 131072, 24, 0.5), (90, 9001, 1030, 0.6),                                            # some rows a workgroup
                                         (8192, 300, 512, 0.9), (20000, 32001, 256, 0.6), (40959, 4097, 128, 0.7), (24000, 131072, 24, 0.9), (5000, 70001, 3, 0.3),  # sorted at once
                                         (131072, 5000, 4, 0.3), (40960, 300, 100, 0.5), (70000, 32001, 256, 0.35), (131072, 131072, 40, 0.2), (131073, 193, 17, 0.0),  # split first
                                         (60000, 50000, 512, 0.4), (5000000, 1000, 1, 0.3)])
def test_table_gradient_of_whole_numbers(n, V, dim, hot):
    """Every sum of small whole numbers is exact in fp32, in any order: a position that is lost, or counted twice, shows however many a token has."""
    rng = np.random.default_rng(n + V + dim)
    tokens = tokens_for(rng, n, V, 0.1, hot)
    inside = (tokens >= 0) & (tokens < V)
    g = rng.integers(-3, 4, (n, dim), dtype=np.int8)
    # (float32: no sum passes 3 n < 2^24)
    want = torch.zeros((V, dim)).index_add_(0, torch.from_numpy(tokens[inside]), torch.from_numpy(g[inside]).float()).to(DEV)
    occurs = torch.from_numpy(np.bincount(tokens[inside], minlength=V) > 0).to(DEV)
    for kind, tkind, accumulate in (("f32", "f32", 0), ("bf16", "f32", 1), ("f16", "bf16", 0), ("bf16", "bf16", 0)):
        grad = torch.from_numpy(g).to(DEV).to(KIND[kind][1])
        out = torch.full((V, dim), 5.0 if accumulate else JUNK, dtype=KIND[tkind][1], device=DEV)
        run_backward(grad, kind, dim, tokens, V, dim, 0.5, accumulate, out, tkind, dim)
        ref = want * 0.5
        if accumulate:
            ref = torch.where(occurs[:, None], ref + 5.0, torch.full_like(ref, 5.0))
        assert torch.equal(out, ref.to(KIND[tkind][1])), (kind, tkind, accumulate)


@pytest.mark.parametrize("n,V,dim", [(64, 1000, 65), (900, 700, 130), (1000, 40000, 96), (4000, 3000, 33), (9000, 9000, 200), (39000, 30000, 24), (50000, 70000, 40), (16000, 40, 3)])
def test_table_gradient_of_few_terms(n, V, dim):
    """c terms are summed by c - 1 additions, in any order, and one product: off by c U of their absolute values' sum at most (2^-10 more for products
    of roundings).  That leaves next to nothing where a token occurs once or twice."""
    rng = np.random.default_rng(n)
    tokens = tokens_for(rng, n, V)
    buf, view, values = place(rng.normal(0, 1, (n, dim)), "f32")
    out = torch.full((V, dim), JUNK, device=DEV)
    scale = float(np.float32(0.3))
    run_backward(view, "f32", dim, tokens, V, dim, scale, 0, out, "f32", dim)
    inside = (tokens >= 0) & (tokens < V)
    total, size = np.zeros((V, dim)), np.zeros((V, dim))
    np.add.at(total, tokens[inside], values[inside])
    np.add.at(size, tokens[inside], np.abs(values[inside]))
    count = np.bincount(tokens[inside], minlength=V)
    assert (np.abs(host(out) - total * scale) <= size * scale * S.U * count[:, None] * (1 + 2.0 ** -10)).all()


def some_of(x, sequences):
    return None if x is None else x[torch.from_numpy(np.asarray(sequences)).to(x.device)]


def verify_on_device(x, y, kind, T, tokens, numbers):
    """run_verify of contiguous rows that are on the device already."""
    B, n1, V = x.shape
    return run_verify(x, y, kind, (V, n1 * V), (V, (n1 - 1) * V), B, n1 - 1, V, T, T, tokens, numbers)


@pytest.mark.parametrize("kind", list(KIND))
def test_verify_rows_that_few_workgroups_sum(kind):
    """140 sequences of long rows: the workgroups of a sequence take slices several times over.  As calls of ten sequences, bit for bit."""
    rng = np.random.default_rng(14)
    B, V = 140, 65537
    g = torch.Generator(device=DEV)
    g.manual_seed(7)
    x = (torch.randn((B, 2, V), generator=g, device=DEV) * 2).to(KIND[kind][1])
    y = (0.9 * x[:, :1].float() + 0.7 * torch.randn((B, 1, V), generator=g, device=DEV)).to(KIND[kind][1])
    tokens = y.float().argmax(dim=2).cpu().numpy()
    numbers = rng.random((B, 2)).astype(np.float32)
    tokens[::3] = (y[::3].float() - x[::3, :1].float()).argmax(dim=2).cpu().numpy()  # (refused)
    numbers[::3, 0] = S.BELOW_1
    out, acc, lp = verify_on_device(x, y, kind, 1.0, tokens, numbers)
    assert 0 < acc.sum() < B
    for b in range(0, B, 10):
        few = verify_on_device(x[b:b + 10], y[b:b + 10], kind, 1.0, tokens[b:b + 10], numbers[b:b + 10])
        for whole, part in zip((out, acc, lp), few):
            assert np.array_equal(whole[b:b + 10], part, equal_nan=part.dtype.kind == "f")
    rows = [0, 1, 69, 138, 139]
    check_verify((out[rows], acc[rows], lp[rows]), host(some_of(x, rows)), host(some_of(y, rows)), 1.0, 1.0, tokens[rows], numbers[rows], kind)


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("V", [9001, 16000, 16384])
def test_verify_more_sequences_of_middling_rows(V, kind):
    """130 sequences are decided and drawn from in one launch where 16-bit rows of 128 take two; both draw the same tokens."""
    rng = np.random.default_rng(V)
    B, n = 130, 8
    g = torch.Generator(device=DEV)
    g.manual_seed(V)
    x = (torch.randn((B, n + 1, V), generator=g, device=DEV) * 2).to(KIND[kind][1])
    y = (0.95 * x[:, :n].float() + 0.3 * torch.randn((B, n, V), generator=g, device=DEV)).to(KIND[kind][1])
    tokens = y.float().argmax(dim=2).cpu().numpy()
    tokens[rng.random((B, n)) < 0.03] = -1
    numbers = numbers_of(rng, B, n, True)
    out, acc, lp = verify_on_device(x, y, kind, 0.75, tokens, numbers)
    two = verify_on_device(x[:128], y[:128], kind, 0.75, tokens[:128], numbers[:128])
    assert np.array_equal(out[:128], two[0]) and np.array_equal(acc[:128], two[1])
    # (the rows' sums are of the same terms in two orders, 64 bits: a last rounding may fall to either side)
    some = ~np.isnan(two[2])
    assert np.array_equal(~np.isnan(lp[:128]), some) and (np.abs(lp[:128][some] - two[2][some]) <= 2 * S.U * np.abs(two[2][some]) + 2.0 ** -45).all()
    rows = [0, 63, 127, 128, 129]
    check_verify((out[rows], acc[rows], lp[rows]), host(some_of(x, rows)), host(some_of(y, rows)), 0.75, 0.75, tokens[rows], numbers[rows], (V, kind))


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("n,V", [(15, 500), (16, 500), (31, 1025), (63, 40), (63, 3001), (63, 9001), (40, 20011)])
def test_verify_long_drafts(n, V, kind):
    rng = np.random.default_rng(V + n)
    for B in (1, 3):
        x, y = rows_for(rng, B, n, V, kind, True)
        y[0] = x[0, :n]   # (a draft that is its target: all are accepted but where a row is marked)
        bx, px, xv = block(x, kind, V + 1, (n + 1) * (V + 1))
        by, py, yv = block(y, kind, V, n * V)
        tokens, numbers = tokens_of(rng, xv, yv, B > 1), numbers_of(rng, B, n, True)
        check_verify(run_verify(px, py, kind, (V + 1, (n + 1) * (V + 1)), (V, n * V), B, n, V, 1.0, 1.0, tokens, numbers), xv, yv, 1.0, 1.0, tokens, numbers, (n, V, kind, B))


@pytest.mark.parametrize("kind,size", [("bf16", 140_000_001), ("f16", 134_300_000), ("f32", 70_000_003)])
def test_sets_past_the_last_cache(kind, size):
    """More than 256 MiB, odd tensors that begin at any element among them: read past the caches; clipped into other buffers and in place."""
    g = torch.Generator(device=DEV)
    g.manual_seed(size)
    spec = [(77, "f32"), (size, kind), (1, "bf16"), (16385, "f16"), (3_000_001, "bf16")]

    def buffers():
        bufs = [torch.full((n + 8,), JUNK, dtype=KIND[k][1], device=DEV) for n, k in spec]
        return bufs, [b[at:at + n] for at, (b, (n, _)) in enumerate(zip(bufs, spec), 1)]
    bufs, views = buffers()
    for v in views:
        v.copy_(torch.randn(v.numel(), generator=g, device=DEV))
    grads = set_of([(None, v, k) for v, (_, k) in zip(views, spec)])
    norm = run_norm(grads)
    want = float(torch.sqrt(sum((v[i:i + (1 << 26)].double().square().sum() for v in views for i in range(0, v.numel(), 1 << 26)))))
    # (sums in 64 bits: what is left is the last rounding; 2^-30 is room for n 2^-53)
    assert abs(float(norm) - want) <= want * (S.U + 2.0 ** -30)
    max_norm = want / 3
    by = torch.tensor(np.float32(max_norm) / np.float32(float(norm)), device=DEV)
    obufs, outs = buffers()
    pb.pb_grad_clip(grads, norm, max_norm, set_of([(None, v, k) for v, (_, k) in zip(outs, spec)]), stream_ptr())
    torch.cuda.synchronize()
    for v, o, b in zip(views, outs, obufs):
        assert torch.equal(o, (v.float() * by).to(v.dtype)) and bool((b[:o.storage_offset()] == JUNK).all()) and bool((b[o.storage_offset() + o.numel():] == JUNK).all())
    pb.pb_grad_clip(grads, norm, 2 * want, None, stream_ptr())   # (not clipped: nothing changes)
    pb.pb_grad_clip(grads, norm, max_norm, None, stream_ptr())
    torch.cuda.synchronize()
    for v, o, b in zip(views, outs, bufs):
        assert torch.equal(v, o) and bool((b[:v.storage_offset()] == JUNK).all()) and bool((b[v.storage_offset() + v.numel():] == JUNK).all())


PATHS = [(500, 1025, 40), (9000, 300, 12), (300, 3, 2), (1000, 20000, 65), (20000, 32001, 9), (6000, 70001, 130), (50000, 3000, 33), (41000, 393216, 3)]


@pytest.mark.parametrize("n,V,dim", PATHS)
@pytest.mark.parametrize("kind,tkind", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32")])
def test_table_gradient_of_absent_tokens_alone(n, V, dim, kind, tkind):
    tokens = np.random.default_rng(n).choice([-1, V, 2 ** 31 - 1, -2 ** 31], n)
    grad = torch.full((n, dim), float("nan"), dtype=KIND[kind][1], device=DEV)
    for accumulate in (0, 1):
        out = torch.full((V, dim), 3.0, dtype=KIND[tkind][1], device=DEV)
        run_backward(grad, kind, dim, tokens, V, dim, 2.0, accumulate, out, tkind, dim)
        assert bool((out == (3.0 if accumulate else 0.0)).all())


@pytest.mark.parametrize("n,V,dim", PATHS)
@pytest.mark.parametrize("kind,tkind", [("f32", "f32"), ("bf16", "f32"), ("f16", "bf16")])
def test_table_gradient_that_is_not_finite(n, V, dim, kind, tkind):
    """An infinity or a NaN in a column of a gradient is one in that column of its token's row, and nowhere else."""
    rng = np.random.default_rng(V)
    tokens = tokens_for(rng, n, V, 0.1, 0.2)
    g = rng.integers(-3, 4, (n, dim)).astype(np.float32)
    for value in (np.inf, -np.inf, np.nan):
        g[rng.integers(0, n, 4), rng.integers(0, dim, 4)] = value
    inside = (tokens >= 0) & (tokens < V)
    want = torch.zeros((V, dim)).index_add_(0, torch.from_numpy(tokens[inside]), torch.from_numpy(g[inside]))
    out = torch.full((V, dim), JUNK, dtype=KIND[tkind][1], device=DEV)
    run_backward(torch.from_numpy(g).to(DEV).to(KIND[kind][1]), kind, dim, tokens, V, dim, 1.0, 0, out, tkind, dim)
    want = want.to(KIND[tkind][1]).float()
    assert not torch.isfinite(want).all() and torch.equal(torch.nan_to_num(out.float().cpu(), nan=-12345.0, posinf=1e30, neginf=-1e30), torch.nan_to_num(want, nan=-12345.0, posinf=1e30, neginf=-1e30))


@pytest.mark.parametrize("kind", list(KIND))
def test_subnormal_numbers(kind):
    """Values, products and sums below the smallest normal number of their type keep what the type holds of them."""
    low = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}[kind]  # the type's smallest
    dim, V = 37, 5
    table = (torch.arange(V * dim, device=DEV, dtype=torch.float64).view(V, dim) * low).to(torch.float32).to(KIND[kind][1])
    assert int((table != 0).sum()) == V * dim - 1
    tokens, out = np.array([4, 0, 3, 3, 1]), torch.full((5, dim), JUNK, dtype=KIND[kind][1], device=DEV)
    for scale in (1.0, 0.5, 3.0):
        pb.pb_embed_tokens(table, KIND[kind][0], dim, V, dim, scale, dev(tokens.astype(np.int32)), 5, out, KIND[kind][0], dim, stream_ptr())
        want = (table.double().cpu() * scale)[torch.from_numpy(tokens)].to(KIND[kind][1])  # (whole multiples of half the smallest: no second rounding)
        assert torch.equal(out.cpu(), want), scale
        grad = torch.full((V, dim), JUNK, dtype=KIND[kind][1], device=DEV)
        run_backward(table, kind, dim, tokens, V, dim, scale, 0, grad, kind, dim)
        sums = torch.zeros((V, dim), dtype=torch.float64).index_add_(0, torch.from_numpy(tokens), table.double().cpu())
        assert torch.equal(grad.cpu(), (sums * scale).to(KIND[kind][1])), scale
    grads = set_of([(None, table.view(-1), kind)])
    norm = run_norm(grads)
    want = float(table.double().square().sum().sqrt())
    assert abs(float(norm) - want) <= want * S.U + 2.0 ** -150  # (half a step of fp32's own)
    by = torch.full((1,), 4.0, device=DEV)
    pb.pb_grad_clip(grads, by, 1.0, set_of([(None, out.view(-1), kind)]), stream_ptr())
    assert torch.equal(out.cpu(), (table.double().cpu() / 4).to(KIND[kind][1]))


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("T", [1e-4, 1e4])
@pytest.mark.parametrize("V,n,sure", [(900, 3, False), (7000, 2, False), (40000, 2, False), (40000, 2, True), (40000, 0, True)])
def test_verify_at_the_ends_of_temperature(V, n, sure, T, kind):
    rng = np.random.default_rng(V + n)
    B, T = 6, float(np.float32(T))
    for size in (1.0, 1e-4, 1e3):
        # (the types' lowest values, as masks, stay what they are or become -inf)
        x, y = (np.where(np.isfinite(r), np.maximum(r * size, -R.LARGEST["f32"]), r) for r in rows_for(rng, B, n, V, kind, True))
        bx, px, xv = block(x, kind, V, (n + 1) * V)
        py, yv = None, None
        if n and not sure:
            by, py, yv = block(y, kind, V, n * V)
        tokens, numbers = tokens_of(rng, xv, xv[:, :n], True), numbers_of(rng, B, n, False)
        tokens[::2] = xv[::2, :n].argmax(axis=2)
        out, acc, lp = run_verify(px, py, kind, (V, (n + 1) * V), (V, n * V), B, n, V, T, T, tokens, numbers)
        check_verify((out, acc, None), xv, yv, T, T, tokens, numbers, (V, T, kind, size))


def test_verify_more_sequences_than_a_launch_takes_with_a_draft():
    """Rows of both models, of middling length and long, in two slices; sequences on both sides as calls of their own."""
    for V in (9001, 20001):
        B, n, g = 32900, 1, torch.Generator(device=DEV)
        g.manual_seed(V)
        x, y = torch.empty((B, 2, V), dtype=torch.bfloat16, device=DEV), torch.empty((B, 1, V), dtype=torch.bfloat16, device=DEV)
        for s in range(0, B, 3000):
            some = torch.randn((min(3000, B - s), 2, V), generator=g, device=DEV) * 2
            x[s:s + 3000] = some
            y[s:s + 3000] = 0.9 * some[:, :1] + 0.7 * torch.randn((min(3000, B - s), 1, V), generator=g, device=DEV)
        tokens, numbers = y.argmax(dim=2).cpu().numpy(), torch.rand((B, 2), generator=g, device=DEV).cpu().numpy()
        out, acc, lp = verify_on_device(x, y, "bf16", 1.0, tokens, numbers)
        for first in (0, 32700):  # (200 sequences: laid out as all of them are)
            s = slice(first, first + 200)
            for whole, part in zip((out, acc, lp), verify_on_device(x[s], y[s], "bf16", 1.0, tokens[s], numbers[s])):
                assert np.array_equal(whole[s], part, equal_nan=part.dtype.kind == "f"), (V, first)
        rows = [0, 32767, 32768, B - 1]
        check_verify((out[rows], acc[rows], lp[rows]), host(some_of(x, rows)), host(some_of(y, rows)), 1.0, 1.0, tokens[rows], numbers[rows], V)
