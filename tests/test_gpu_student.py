"""The calls around a student on the GPU against the 64-bit definitions in student.py: rows for tokens and the table's gradient,
the norm over gradients and their clipping, and the verification of drafted tokens, at every type, odd sizes, strides and
alignments, absent tokens, rows whose mask leaves nothing, numbers on borders, graphs, streams, and all of them in a run."""
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

GUARD = 0x5a


def workspace(size, slack=64):
    """A workspace of exactly `size` bytes, with a guard behind it."""
    return torch.full((size + slack,), GUARD, dtype=torch.uint8, device=DEV)


def guard_ok(ws, size):
    return bool((ws[size:] == GUARD).all())


# ---- rows for tokens ---------------------------------------------------------------------------------------------------

def tokens_for(rng, n, V, absent=0.1, hot=0.0):
    t = rng.integers(0, V, n)
    t[rng.random(n) < hot] = rng.integers(0, V)
    t[rng.random(n) < absent] = rng.choice([-1, V, 2 ** 31 - 1, -2 ** 31])
    return t


DIMS = [1, 2, 3, 7, 8, 9, 15, 16, 17, 63, 64, 65, 100, 128, 250, 511, 512, 513, 640, 1000, 1024, 2048, 2050]


@pytest.mark.parametrize("out", list(KIND))
@pytest.mark.parametrize("table", list(KIND))
def test_lookup(table, out):
    rng = np.random.default_rng(11)
    for dim in DIMS:
        V, n = int(rng.integers(1, 60)), int(rng.choice([1, 2, 5, 33, 130]))
        stride, shift, out_stride, scale = dim + int(rng.choice([0, 3])), int(rng.choice([0, 1])), dim + int(rng.choice([0, 5])), float(rng.choice([1.0, 0.3, 22.6]))
        buf, view, _ = place(rng.normal(0, 1, (V, dim)), table, stride, shift)
        tokens = tokens_for(rng, n, V)
        to = torch.full((n * out_stride + 9,), JUNK, dtype=KIND[out][1], device=DEV)
        pb.pb_embed_tokens(view, KIND[table][0], stride, V, dim, scale, dev(tokens.astype(np.int32)), n, to[1:], KIND[out][0], out_stride, stream_ptr())
        got = torch.as_strided(to, (n, dim), (out_stride, 1), 1)
        there = torch.from_numpy((tokens >= 0) & (tokens < V)).to(DEV)
        rows = view[torch.from_numpy(np.where((tokens >= 0) & (tokens < V), tokens, 0)).to(DEV)]
        want = torch.where(there[:, None], rows.float() * torch.tensor(scale, dtype=torch.float32, device=DEV), 0.0).to(KIND[out][1])
        assert torch.equal(got, want), (dim, V, n)        # (one product in fp32, rounded once: the same bits)
        kept = torch.full_like(to, JUNK)
        torch.as_strided(kept, (n, dim), (out_stride, 1), 1).copy_(got)
        assert torch.equal(kept, to), (dim, "written beside the rows")


def test_lookup_of_odd_values():
    """Infinities and NaN of the table come through, a token that is absent looks at none of them."""
    table = torch.tensor([[np.inf, -np.inf, np.nan, 1.0], [1.0, 2.0, 3.0, 4.0]], device=DEV)
    out = torch.empty((3, 4), device=DEV)
    pb.pb_embed_tokens(table, pb.PB_F32, 4, 2, 4, -2.0, dev(np.array([0, -1, 1], np.int32)), 3, out, pb.PB_F32, 4, stream_ptr())
    got = out.cpu().numpy()
    assert got[0, 0] == -np.inf and got[0, 1] == np.inf and np.isnan(got[0, 2]) and (got[1] == 0).all() and list(got[2]) == [-2, -4, -6, -8]


def run_backward(grad, kind, stride, tokens, V, dim, scale, accumulate, table, tkind, tstride, stream=None):
    n = len(tokens)
    size = pb.pb_embed_tokens_backward_workspace_bytes(n, V, dim)
    ws = workspace(size)
    pb.pb_embed_tokens_backward(grad, KIND[kind][0], stride, dev(tokens.astype(np.int32)) if n else None, n, V, dim, scale, accumulate, table,
                                KIND[tkind][0], tstride, ws, size, stream_ptr() if stream is None else stream)
    assert guard_ok(ws, size)


def check_backward(rng, n, V, dim, kind, tkind, absent, hot, accumulate, where):
    stride, shift, tstride, scale = dim + int(rng.choice([0, 3])), int(rng.choice([0, 1])), dim + int(rng.choice([0, 5])), float(np.float32(rng.choice([1.0, 0.3, 22.6])))
    tokens = tokens_for(rng, n, V, absent, hot)
    x = rng.normal(0, 1, (max(n, 1), dim))
    inside = (tokens >= 0) & (tokens < V)
    x[:n][~inside & (rng.random(n) < 0.5)] = np.nan       # (not looked at)
    buf, view, values = place(x, kind, stride, shift)
    to = torch.full((V * tstride + 9,), 3.0, dtype=KIND[tkind][1], device=DEV)
    before = to.clone()
    run_backward(view, kind, stride, tokens, V, dim, scale, accumulate, to[1:], tkind, tstride)
    total, bound, count = S.table_gradient(np.where(inside[:, None], values[:n], 0.0), tokens, V, scale)
    if accumulate:
        bound = bound + S.U * (np.abs(total) + 3.0 + bound)
        total = total + 3.0
    got = torch.as_strided(to, (V, dim), (tstride, 1), 1)
    R.check(host(got), total, np.where(count[:, None] > 0, R.rounded(bound, total, tkind), 0.0), where)
    torch.as_strided(before, (V, dim), (tstride, 1), 1).copy_(got)
    assert torch.equal(before, to), (where, "written beside the rows")
    if accumulate:
        assert bool((got[torch.from_numpy(count == 0).to(DEV)] == 3.0).all()), where


@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("tkind", list(KIND))
@pytest.mark.parametrize("kind", list(KIND))
def test_table_gradient(kind, tkind, accumulate):
    rng = np.random.default_rng(5)
    for dim in DIMS:
        n, V = int(rng.choice([0, 1, 2, 63, 64, 65, 129, 500, 1000])), int(rng.choice([1, 2, 7, 100, 257, 1025]))
        check_backward(rng, n, V, dim, kind, tkind, 0.2, float(rng.choice([0.0, 0.6])), accumulate, (n, V, dim))


@pytest.mark.parametrize("n,V,dim,hot", [(1, 393216, 3, 0.0), (5000, 393216, 8, 0.3), (4095, 1, 40, 0.0), (4096, 2, 33, 0.5), (4097, 3, 512, 0.0),
                                         (20000, 1025, 16, 0.08), (20000, 1, 8, 0.0), (131072, 5000, 4, 0.2), (70001, 131072, 5, 0.01), (16384, 256, 1030, 0.9),
                                         (12345, 257, 64, 0.05), (8192, 64, 7, 0.0), (130, 2, 2048, 1.0), (16384, 1000, 5, 0.2), (16383, 90, 60, 0.0), (5001, 300, 128, 0.4), (4097, 6144, 3, 0.0),
                                         (4096, 61, 2500, 0.9), (1025, 5, 300, 0.0), (1024, 5, 300, 0.5), (16385, 1000, 5, 0.1), (64 * 40, 40, 9, 0.0), (24575, 700, 6, 0.3), (40959, 300, 10, 0.3), (40960, 5000, 7, 0.1),
                                         (24576, 393216, 2, 0.1), (28673, 1, 9, 0.0), (40000, 256, 12, 0.5), (65536, 257, 33, 0.02), (300000, 513, 3, 0.4)])
def test_table_gradient_sizes(n, V, dim, hot):
    rng = np.random.default_rng(n + V)
    for kind, tkind, accumulate in (("f32", "f32", 0), ("bf16", "f32", 1), ("bf16", "bf16", 0)):
        check_backward(rng, n, V, dim, kind, tkind, 0.1, hot, accumulate, (n, V, dim, kind))


@pytest.mark.parametrize("n,V,dim,hot", [(4095, 65536, 5, 0.1), (4096, 65536, 5, 0.1), (4096, 65537, 4, 0.1), (20000, 32001, 250, 0.05), (300, 70001, 200, 0.2), (40959, 20001, 256, 0.3),
                                         (9000, 200001, 22, 0.2), (7000, 33001, 300, 0.0), (41000, 16385, 511, 0.1), (4096, 16385, 256, 0.9), (1, 16385, 255, 0.0), (0, 16385, 256, 0.0),
                                         (33000, 6145, 3, 0.02), (16385, 129, 3, 0.5), (32768, 65536, 2, 0.9)])
def test_table_gradient_of_large_tables(n, V, dim, hot):
    """Positions that two workgroups a range place, rows that lanes take several of."""
    rng = np.random.default_rng(n + V)
    for kind, tkind, accumulate in (("f32", "f32", 1), ("bf16", "f32", 0), ("f16", "bf16", 0), ("bf16", "bf16", 1)):
        check_backward(rng, n, V, dim, kind, tkind, 0.1, hot, accumulate, (n, V, dim, kind))


@pytest.mark.parametrize("n,V,dim,hot", [(1024, 4609, 64, 0.1), (1025, 4609, 64, 0.1), (1024, 6145, 8, 1.0), (1, 32769, 130, 0.0), (0, 20000, 9, 0.0), (1000, 16384, 257, 0.0), (1000, 16385, 12, 0.3),
                                         (700, 32768, 300, 0.05), (257, 40007, 1030, 0.0), (256, 131072, 8, 0.9), (1023, 393216, 16, 0.0), (300, 2400, 700, 0.2), (64, 9001, 7, 0.0), (64, 9001, 3, 0.0)])
def test_table_gradient_of_few_tokens(n, V, dim, hot):
    """One launch whose workgroups take some rows each."""
    rng = np.random.default_rng(n + V)
    for kind, tkind, accumulate in (("f32", "f32", 1), ("bf16", "f32", 0), ("f16", "bf16", 0), ("bf16", "bf16", 1)):
        check_backward(rng, n, V, dim, kind, tkind, 0.1, hot, accumulate, (n, V, dim, kind))


def test_table_gradient_of_runs():
    """Tokens in runs whose lengths lie around the lengths that are summed at once: ends of runs on and beside every border."""
    rng = np.random.default_rng(9)
    for lengths in ([64, 65, 63, 64, 1, 128, 129, 127, 2, 66], [65] * 20, [1] * 63 + [65, 64, 192, 193], [200, 1, 63, 300], [64] * 10, [1000]):
        tokens = rng.permutation(np.repeat(np.arange(len(lengths)), lengths))
        g = rng.normal(0, 1, (len(tokens), 12))
        buf, view, values = place(g, "f32")
        out = torch.full((len(lengths) + 2, 12), JUNK, device=DEV)
        run_backward(view, "f32", 12, tokens, len(lengths) + 2, 12, 1.0, 0, out, "f32", 12)
        total, bound, _ = S.table_gradient(values, tokens, len(lengths) + 2, 1.0)
        R.check(host(out), total, R.rounded(bound, total, "f32"), lengths)
        again = torch.full_like(out, JUNK)
        run_backward(view, "f32", 12, tokens, len(lengths) + 2, 12, 1.0, 0, again, "f32", 12)
        assert torch.equal(out, again)      # the same bits every time


def test_rows_past_32_bits():
    """Tables, gradients and outputs whose rows lie more than 2^32 bytes and 2^31 elements apart."""
    dim, far = 40, (1 << 31) + 24
    big = torch.zeros(far + 2 * dim, dtype=torch.bfloat16, device=DEV)
    two = torch.as_strided(big, (2, dim), (far, 1))
    two.copy_(torch.randn((2, dim), device=DEV))
    tokens = dev(np.array([1, 0, 1, -1], np.int32))
    out = torch.empty((4, dim), dtype=torch.bfloat16, device=DEV)
    pb.pb_embed_tokens(two, pb.PB_BF16, far, 2, dim, 1.0, tokens, 4, out, pb.PB_BF16, dim, stream_ptr())
    assert torch.equal(out[0], two[1]) and torch.equal(out[1], two[0]) and torch.equal(out[2], two[1]) and not out[3].any()
    want = two.clone()
    grad, ws = torch.empty((3, dim), dtype=torch.bfloat16, device=DEV), workspace(pb.pb_embed_tokens_backward_workspace_bytes(2, 3, dim))
    pb.pb_embed_tokens_backward(two, pb.PB_BF16, far, dev(np.array([2, 0], np.int32)), 2, 3, dim, 1.0, 0, grad, pb.PB_BF16, dim, ws, ws.numel(), stream_ptr())
    assert torch.equal(grad[2], want[0]) and torch.equal(grad[0], want[1]) and not grad[1].any()
    pb.pb_embed_tokens(out, pb.PB_BF16, dim, 4, dim, 1.0, dev(np.array([3, 1], np.int32)), 2, two, pb.PB_BF16, far, stream_ptr())
    assert not two[0].any() and torch.equal(two[1], out[1])
    pb.pb_embed_tokens_backward(grad, pb.PB_BF16, dim, dev(np.array([1, 0, 1], np.int32)), 3, 2, dim, 1.0, 0, two, pb.PB_BF16, far, ws, ws.numel(), stream_ptr())
    assert torch.equal(two[0], grad[1]) and torch.equal(two[1], (grad[0].float() + grad[2].float()).bfloat16())
    # a verification: row strides and sequence strides
    x = torch.randn((2, dim), device=DEV)
    two.copy_(x)
    numbers = torch.tensor([[0.3], [0.8]], device=DEV)
    drawn, acc = torch.empty((2, 1), dtype=torch.int32, device=DEV), torch.empty(2, dtype=torch.int32, device=DEV)
    pb.pb_verify_draft(two, None, pb.PB_BF16, far, dim, 0, 0, 2, 0, dim, 1.0, 1.0, None, numbers, drawn, acc, None, None, 0, stream_ptr())
    for b in range(2):
        assert int(drawn[b, 0]) == S.drawn(S.probabilities(host(two[b]), 1.0)[0], float(numbers[b, 0]))
    pb.pb_verify_draft(two, two, pb.PB_BF16, 2 * far, far, far, dim, 1, 1, dim, 1.0, 1.0, two[0].argmax().view(1, 1).to(torch.int32), numbers, drawn, acc, None, None, 0,
                       stream_ptr())
    assert int(acc[0]) == 1 and int(drawn[1, 0]) == S.drawn(S.probabilities(host(two[1]), 1.0)[0], float(numbers[1, 0]))


@pytest.mark.parametrize("n,V,hot", [(5_000_000, 1000, 0.0), (4_500_000, 393216, 0.3)])
def test_table_gradient_of_millions(n, V, hot):
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    tokens = torch.randint(-1, V, (n,), generator=g, device=DEV, dtype=torch.int32)
    tokens[torch.rand(n, generator=g, device=DEV) < hot] = 77
    grad = torch.randn((n, 1), generator=g, device=DEV)
    out = torch.full((V, 1), JUNK, device=DEV)
    size = pb.pb_embed_tokens_backward_workspace_bytes(n, V, 1)
    ws = workspace(size)
    pb.pb_embed_tokens_backward(grad, pb.PB_F32, 1, tokens, n, V, 1, 0.5, 0, out, pb.PB_F32, 1, ws, size, stream_ptr())
    assert guard_ok(ws, size)
    at, x = tokens.cpu().numpy() + 1, host(grad[:, 0]) * 0.5   # (absent ones come first, and are dropped)
    want, sizes, count = (np.bincount(at, weights=w, minlength=V + 1)[1:] for w in (x, np.abs(x), np.ones(n)))
    # (as in table_gradient; the pieces' sums once more in up to 1024 shares)
    bound = sizes * S.U * (np.minimum(count, S.FEW) + count // S.FEW + 1024 + 3) + S.U * np.abs(want)
    assert (np.abs(host(out[:, 0]) - want) <= bound).all()


# ---- norm and clipping -------------------------------------------------------------------------------------------------

def tensors_of(rng, spec, shift=False):
    out = []
    for k, (n, kind) in enumerate(spec):
        buf = torch.full((n + 8,), JUNK, dtype=KIND[kind][1], device=DEV)
        at = 1 + k % 7 if shift else 0
        buf[at:at + n] = torch.from_numpy(rng.normal(0, 0.5, n).astype(np.float32)).to(DEV).to(KIND[kind][1])
        out.append((buf, buf[at:at + n], kind))
    return out


def set_of(tensors):
    return pb.pb_tensors_build([t for _, t, _ in tensors], [t.numel() for _, t, _ in tensors], [KIND[k][0] for _, _, k in tensors])


def run_norm(grads, stream=None):
    norm = torch.full((2,), JUNK, device=DEV)
    size = pb.pb_grad_norm_workspace_bytes(grads)
    ws = workspace(size)
    pb.pb_grad_norm(grads, norm, ws, size, stream_ptr() if stream is None else stream)
    assert guard_ok(ws, size) and norm[1] == JUNK
    return norm[:1]


SPECS = [[(1, "f32")], [(5, "bf16"), (0, "f16"), (9, "f16"), (3, "f32")], [(16384, "f32"), (16385, "bf16"), (16383, "f16"), (1, "bf16")],
         [(100000, "bf16"), (7, "f32"), (300001, "f32"), (77777, "f16")], [(n, k) for n in range(1, 40) for k in KIND], [(0, "f32")],
         [(50_000_000, "bf16"), (3, "f32")], [(1 + k, "f16") for k in range(64)], [(1, "f32")] * 65, [(2048 * 64, "bf16")], [(2048 * 63 + 1, "f32"), (1, "bf16")],
         [(2047, k) for k in KIND] * 16 + [(2049, "f32")] * 8]


@pytest.mark.parametrize("spec", SPECS, ids=range(len(SPECS)))
@pytest.mark.parametrize("shift", [False, True])
def test_norm_and_clipping(spec, shift):
    rng = np.random.default_rng(len(spec))
    tensors = tensors_of(rng, spec, shift)
    grads = set_of(tensors)
    norm = run_norm(grads)
    want = float(torch.sqrt(sum(t.double().square().sum() for _, t, _ in tensors)))
    # (sums in 64 bits: what is left is the last rounding; 2^-30 is room for n 2^-53)
    assert abs(float(norm) - want) <= want * (S.U + 2.0 ** -30)
    for max_norm in (want * 0.25, want * 2 + 1.0, float(norm), 0.0):
        into = [(torch.full_like(b, JUNK), None, k) for b, _, k in tensors]
        into = [(b, b[t.storage_offset():t.storage_offset() + t.numel()], k) for (b, _, k), (_, t, _) in zip(into, tensors)]
        out = set_of(into)
        pb.pb_grad_clip(grads, norm, max_norm, out, stream_ptr())
        by = np.float32(max_norm) / np.float32(float(norm)) if np.float32(float(norm)) > np.float32(max_norm) else np.float32(1.0)
        copies = [(b.clone(), None, k) for b, _, k in tensors]
        copies = [(b, b[t.storage_offset():t.storage_offset() + t.numel()], k) for (b, _, k), (_, t, _) in zip(copies, tensors)]
        pb.pb_grad_clip(set_of(copies), norm, max_norm, None, stream_ptr())
        torch.cuda.synchronize()
        for (src, t, _), (b, o, _), (cb, c, _) in zip(tensors, into, copies):
            x = (t.float() * torch.tensor(by, device=DEV)).to(t.dtype)
            assert torch.equal(o, x) and torch.equal(c, x)
            at = o.storage_offset()
            assert bool((b[:at] == JUNK).all()) and bool((b[at + o.numel():] == JUNK).all())
            assert torch.equal(cb[:at], src[:at]) and torch.equal(cb[at + o.numel():], src[at + o.numel():])


@pytest.mark.parametrize("value,want", [(1e30, "big"), (3e38, "inf"), (1e-30, "small"), (float("nan"), "nan"), (float("inf"), "inf")])
def test_norms_out_of_the_ordinary(value, want):
    t = torch.full((1000,), value, device=DEV)
    grads = set_of([(t, t, "f32")])
    norm = run_norm(grads)
    got = float(norm)
    if want in ("big", "small"):
        exact = float(t[0].double()) * np.sqrt(1000.0)
        assert abs(got - exact) <= exact * 2 * S.U
    else:
        assert np.isnan(got) if want == "nan" else got == np.inf
        before = t.clone()
        pb.pb_grad_clip(grads, norm, 1.0, None, stream_ptr())
        out = torch.zeros_like(t)
        pb.pb_grad_clip(grads, norm, 1.0, set_of([(out, out, "f32")]), stream_ptr())
        assert torch.equal(t.view(torch.int32), before.view(torch.int32)) and torch.equal(out.view(torch.int32), before.view(torch.int32))


def test_clip_refuses_another_set():
    a, b = torch.zeros(4, device=DEV), torch.zeros(5, device=DEV)
    norm = torch.ones(1, device=DEV)
    grads = set_of([(a, a, "f32")])
    for other in (set_of([(b, b, "f32")]), pb.pb_tensors_build([b], [4], [pb.PB_F16]), pb.pb_tensors_build([b, b], [2, 2], [pb.PB_F32] * 2)):
        with pytest.raises(pb.PbError) as e:
            pb.pb_grad_clip(grads, norm, 1.0, other, stream_ptr())
        assert e.value.code == pb.PB_EINVAL
    for bad in (-1.0, float("nan"), float("inf")):
        with pytest.raises(pb.PbError) as e:
            pb.pb_grad_clip(grads, norm, bad, None, stream_ptr())
        assert e.value.code == pb.PB_ERANGE
    for change in (dict(d_norm=None), dict(workspace_bytes=0), dict(d_workspace=None), dict(workspace_bytes=-1)):
        ws = workspace(64)
        call = dict(d_norm=norm, d_workspace=ws, workspace_bytes=64, stream=stream_ptr())
        with pytest.raises(pb.PbError) as e:
            pb.pb_grad_norm(grads, **dict(call, **change))
        assert e.value.code == pb.PB_EINVAL


def test_tensors_that_share_memory():
    x, norm, ws = torch.arange(1.0, 17.0, device=DEV), torch.full((1,), 8.0, device=DEV), workspace(64)
    f32 = lambda *parts: pb.pb_tensors_build(list(parts), [p.numel() for p in parts], [pb.PB_F32] * len(parts))  # noqa: E731
    lo, mid, hi, y = x[:4], x[2:6], x[4:8], torch.zeros(8, device=DEV)
    none = x[:0]
    for grads, out in ((f32(lo, lo), None), (f32(lo, mid), None), (f32(lo, hi), f32(hi, lo)), (f32(lo, hi), f32(y[:4], y[2:6])), (f32(lo), f32(mid)),
                       (f32(lo, hi), f32(x[8:12], lo)), (f32(lo, mid), f32(lo, y[:4])), (f32(lo, hi, x[8:12]), f32(lo, hi, x[7:11])),
                       (f32(x[:8], y), f32(x[1:9], y))):
        before = x.clone()
        with pytest.raises(pb.PbError) as e:
            pb.pb_grad_clip(grads, norm, 1.0, out, stream_ptr())
        assert e.value.code == pb.PB_EINVAL and torch.equal(x, before)
    # each counts in the norm; into other buffers, or the same ones by another set, they are clipped
    got = torch.zeros(1, device=DEV)
    pb.pb_grad_norm(f32(lo, mid), got, ws, 64, stream_ptr())
    want = float(torch.cat([lo, mid]).double().square().sum().sqrt())
    assert abs(float(got) - want) <= 2 * S.U * want
    pb.pb_grad_clip(f32(lo, mid), norm, 1.0, f32(y[:4], y[4:]), stream_ptr())
    assert torch.equal(y, torch.cat([lo, mid]) / 8)
    before = x.clone()
    pb.pb_grad_clip(f32(hi, none, lo), norm, 1.0, f32(hi, y[:0], lo), stream_ptr())
    assert torch.equal(x[:8], before[:8] / 8) and torch.equal(x[8:], before[8:])
    pb.pb_grad_clip(f32(x[8:12], hi, lo), norm, 1.0, f32(x[8:12], y[:4], lo), stream_ptr())
    assert torch.equal(x[8:12], before[8:12] / 8) and torch.equal(y[:4], before[4:8] / 64) and torch.equal(x[4:8], before[4:8] / 8)


# ---- verification ------------------------------------------------------------------------------------------------------

def block(x, kind, row_stride, seq_stride, shift=0):
    """x [B, n, V] on the device at the given strides, junk between; the buffer, its first element, the float64 values."""
    B, n, V = x.shape
    buf = torch.full((shift + (B - 1) * seq_stride + (n - 1) * row_stride + V + 8,), JUNK, dtype=KIND[kind][1], device=DEV)
    view = torch.as_strided(buf, (B, n, V), (seq_stride, row_stride, 1), shift)
    view.copy_(torch.from_numpy(x.astype(np.float32)).to(DEV))
    return buf, buf[shift:], view.double().cpu().numpy()


def layout(rng, B, n, V):
    """(row stride, sequence stride): rows of a sequence together, padded, or sequences side by side for each place."""
    pad = V + int(rng.choice([0, 0, 1, 5, 64]))
    if rng.random() < 0.3:
        return B * pad, pad
    return pad, n * pad + int(rng.choice([0, 3]))


def run_verify(x, y, kind, xs, ys, B, n, V, T, Ty, tokens, numbers, logp=True, stream=None):
    out = torch.full((B * (n + 1) + 4,), -7, dtype=torch.int32, device=DEV)
    acc = torch.full((B + 4,), -7, dtype=torch.int32, device=DEV)
    lp = torch.full((B * (n + 1) + 4,), JUNK, device=DEV) if logp else None
    size = pb.pb_verify_draft_workspace_bytes(KIND[kind][0], B, n, V)
    ws = workspace(size)
    pb.pb_verify_draft(x, y, KIND[kind][0], xs[1], xs[0], ys[1], ys[0], B, n, V, T, Ty, dev(tokens.astype(np.int32)) if n else None,
                       dev(numbers.astype(np.float32)), out, acc, lp, ws, size, stream_ptr() if stream is None else stream)
    assert guard_ok(ws, size)
    assert bool((out[B * (n + 1):] == -7).all()) and bool((acc[B:] == -7).all()) and (lp is None or bool((lp[B * (n + 1):] == JUNK).all()))
    shape = (B, n + 1)
    return out[:B * (n + 1)].view(shape).cpu().numpy(), acc[:B].cpu().numpy(), lp[:B * (n + 1)].view(shape).double().cpu().numpy() if logp else None


def check_verify(got, xv, yv, T, Ty, tokens, numbers, where):
    out, acc, lp = got
    for b in range(len(out)):
        w_out, w_k, w_lp = S.verify(xv[b], None if yv is None else yv[b], T, Ty, tokens[b], numbers[b])
        assert acc[b] == w_k and np.array_equal(out[b], w_out), (where, b, acc[b], w_k, out[b], w_out)
        if lp is not None:  # (what lies beside a row's largest token is off by 2^-18 of itself at most; 2^-50 of its spread for what 64 bits
            # round; the sum of a row is 1 or more of its largest weight, rounded to 2^-53 of itself here and there, and so its logarithm)
            fin = ~np.isnan(w_lp)
            room = np.zeros(len(w_lp))
            for i in np.flatnonzero(fin):
                p, lps, _ = S.probabilities(xv[b, i], T)
                room[i] = 2.0 ** -18 * p[p < p.max()].sum() + 2.0 ** -50 * (lps.max() - w_lp[i])
            assert np.array_equal(np.isnan(lp[b]), ~fin), (where, b)
            assert (np.abs(lp[b][fin] - w_lp[fin]) <= S.U * np.abs(w_lp[fin]) + room[fin] + 2.0 ** -51).all(), (where, b, lp[b], w_lp)


def rows_for(rng, B, n, V, kind, odd):
    """Target and draft rows: the draft's the target's with noise; and rows of all sorts among them."""
    x = rng.normal(0, 2.5, (B, n + 1, V))
    y = 0.9 * x[:, :n] + 0.7 * rng.normal(0, 1, (B, n, V))
    for z in (x, y):
        for b in range(B):
            for i in range(z.shape[1]):
                sort = int(rng.integers(0, 16)) if odd else 0
                if sort == 1:
                    z[b, i, rng.integers(0, V)] += float(rng.choice([12.0, 20.0, 30.0]))
                elif sort == 2:
                    z[b, i] = 1.5
                elif sort == 3:
                    z[b, i, rng.random(V) < 0.95] = -np.inf
                elif sort == 4 and rng.random() < 0.3:
                    z[b, i] = -np.inf
                elif sort == 5 and rng.random() < 0.3:
                    z[b, i, rng.integers(0, V)] = np.nan
                elif sort == 6 and rng.random() < 0.3:
                    z[b, i, rng.integers(0, V)] = np.inf
                elif sort == 7:
                    z[b, i] += 900.0 * (1 if rng.random() < 0.5 else -1)
                elif sort == 8:
                    z[b, i] = np.round(z[b, i])
                elif sort == 9:
                    z[b, i, rng.random(V) < 0.9] = -R.LARGEST[kind]
                elif sort == 10 and rng.random() < 0.3:
                    z[b, i] = -R.LARGEST[kind]
                elif sort == 11 and i < n:
                    x[b, i] = y[b, i]
    return x, y


def tokens_of(rng, x, y, ragged):
    """Likely tokens of the draft, some unlikely, some absent ones."""
    B, n, V = y.shape
    t = rng.integers(0, V, (B, n))
    for b in range(B):
        for i in range(n):
            q = S.probabilities(y[b, i], 1.0)[0]
            if rng.random() < 0.9 and np.isfinite(q).all() and q.sum() > 0:
                t[b, i] = rng.choice(V, p=q / q.sum())
    if ragged:
        t[rng.random((B, n)) < 0.1] = rng.choice([-1, V, 2 ** 31 - 1, -2 ** 31])
    return t


def numbers_of(rng, B, n, odd):
    u = rng.random((B, n + 1)).astype(np.float32)
    if odd:
        at = rng.random(u.shape) < 0.15
        u[at] = rng.choice(np.array([0.0, 1.0 - 2.0 ** -24, 1.0, -1.0, 7.0, np.nan, -0.0, 0.5, np.inf, -np.inf], np.float32), at.sum())
    return u


SIZES = [1, 2, 3, 5, 8, 9, 15, 16, 17, 31, 64, 65, 100, 127, 129, 255, 257, 511, 512, 513, 1000, 1024, 1025, 2047, 2048, 2049, 3001, 4095, 4096, 4097,
         5000, 8191, 8193, 10007, 16384, 16385, 32001, 50000, 65537]


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("V", SIZES)
def test_verify_sizes(V, kind):
    rng = np.random.default_rng(V * 3 + 1)
    for case in range(4):
        B, n = (int(rng.choice([1, 2, 5, 9])), int(rng.choice([0, 1, 2, 4, 7]))) if V < 9000 else (int(rng.choice([1, 2])), int(rng.choice([0, 1, 3])))
        T, Ty = float(rng.choice([1.0, 0.75, 2.0])), float(rng.choice([1.0, 0.5]))
        x, y = rows_for(rng, B, n, V, kind, case > 0)
        xs, ys = layout(rng, B, n + 1, V), layout(rng, B, max(n, 1), V)
        bx, px, xv = block(x, kind, *xs, int(rng.choice([0, 1, 3])))
        by, py, yv = block(y, kind, *ys, int(rng.choice([0, 1, 3]))) if n and case != 2 else (None, None, None)
        tokens, numbers = tokens_of(rng, xv, yv if yv is not None else y, case == 3), numbers_of(rng, B, n, case > 0)
        got = run_verify(px, py, kind, xs, ys, B, n, V, T, Ty, tokens, numbers, logp=case != 1)
        check_verify(got, xv, yv, T, Ty, tokens, numbers, (V, kind, case, B, n, xs, ys, T, Ty))


@pytest.mark.parametrize("B,n,V", [(300, 3, 130), (70, 8, 1025), (2, 63, 700), (1, 63, 5000), (40, 1, 9001), (600, 0, 64), (33, 15, 257), (3, 20, 20000)])
def test_verify_batches(B, n, V):
    rng = np.random.default_rng(B + n + V)
    for kind in KIND:
        x, y = rows_for(rng, B, n, V, kind, True)
        xs, ys = layout(rng, B, n + 1, V), layout(rng, B, max(n, 1), V)
        bx, px, xv = block(x, kind, *xs, 1)
        by, py, yv = block(y, kind, *ys) if n else (None, None, None)
        tokens, numbers = tokens_of(rng, xv, yv if n else y, True), numbers_of(rng, B, n, True)
        check_verify(run_verify(px, py, kind, xs, ys, B, n, V, 1.0, 1.0, tokens, numbers), xv, yv, 1.0, 1.0, tokens, numbers, (B, n, V, kind))


@pytest.mark.parametrize("V", [131072, 393216])
@pytest.mark.parametrize("kind", list(KIND))
def test_verify_long_rows(kind, V):
    rng = np.random.default_rng(V)
    for B, n in ((1, 2), (2, 1)):
        x, y = rng.normal(0, 2, (B, n + 1, V)), None
        y = x[:, :n] + rng.normal(0, 0.5, (B, n, V))
        xs, ys = (V + 1, (n + 1) * (V + 1)), (V, n * V)
        bx, px, xv = block(x, kind, *xs, 1)
        by, py, yv = block(y, kind, *ys)
        for turn in range(4):
            tokens, numbers = yv.argmax(axis=2), rng.random((B, n + 1)).astype(np.float32)
            if turn > 1:  # (refused: the rest is drawn from)
                numbers[:, 0] = 1 - 2.0 ** -24
                tokens[:, 0] = (yv[:, 0] - xv[:, 0]).argmax(axis=1)
            check_verify(run_verify(px, py, kind, xs, ys, B, n, V, 1.0, 1.0, tokens, numbers), xv, yv, 1.0, 1.0, tokens, numbers, (V, kind, B, n, turn))


def test_verify_borders():
    """Flat rows, whose sums are whole numbers: numbers that lie on borders decide as the definition says."""
    V = 8
    x = np.zeros((9, 2, V))
    y = np.full((9, 1, V), -np.inf)
    y[:, 0, :4] = 0.0                                  # p = 1/8, q = 1/4 on the first four: accepted below 1/2
    tokens = np.full((9, 1), 2)
    numbers = np.array([[0.5, w / 8] for w in range(8)] + [[0.5 - 2.0 ** -25, 0.875]])
    bx, px, xv = block(x, "f32", V, 2 * V)
    by, py, yv = block(y, "f32", V, V)
    got = run_verify(px, py, "f32", (V, 2 * V), (V, V), 9, 1, V, 1.0, 1.0, tokens, numbers)
    check_verify(got, xv, yv, 1.0, 1.0, tokens, numbers, "borders")
    assert list(got[1]) == [0] * 8 + [1] and [int(t) for t in got[0][:8, 0]] == [4, 4, 5, 5, 6, 6, 7, 7] and list(got[0][8]) == [2, 7]


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("V", [50, 1025, 5000, 20011])
def test_verify_equal_rows(V, kind):
    """A draft that is its target accepts whatever it draws; a token that both bar is refused, and the target's row drawn from; rows
    lie at other alignments."""
    rng = np.random.default_rng(V)
    x = rng.normal(0, 2, (6, 3, V))
    x[:, :, 7] = -np.inf
    bx, px, xv = block(x, kind, V + 1, 3 * (V + 1), 1)
    by, py, yv = block(x[:, :2], kind, V, 2 * V + 3, 2)
    tokens = np.where(np.arange(6)[:, None] < 3, xv[:, :2].argmax(axis=2), np.array([[9, 7]]))
    numbers = np.full((6, 3), S.BELOW_1)
    numbers[:, 2] = rng.random(6)
    got = run_verify(px, py, kind, (V + 1, 3 * (V + 1)), (V, 2 * V + 3), 6, 2, V, 1.0, 1.0, tokens, numbers)
    check_verify(got, xv, yv, 1.0, 1.0, tokens, numbers, V)
    assert list(got[1]) == [2, 2, 2, 1, 1, 1] and (got[0][3:, 1] >= 0).all()


def refused(y, x):
    """A token whose p lies as far below its q as any, and a number that refuses it."""
    q = np.array([S.probabilities(r, 1.0)[0] for r in y])
    p = np.array([S.probabilities(r, 1.0)[0] for r in x])
    return (p / q).argmin(axis=1), S.BELOW_1


@pytest.mark.parametrize("V", [700, 5000, 20011, 131072])
def test_verify_tokens_on_the_line(V):
    """Draft and target agree on most tokens, and what some have more the others have less, so that p / q is 1 within 1e-8 on the many:
    on which side they lie is for the last bits of the two sums to say."""
    rng = np.random.default_rng(V)
    B = 4
    y = rng.normal(0, 1.5, (B, 1, V)).astype(np.float32).astype(np.float64)
    x = np.repeat(y, 2, axis=1)
    up, down = np.arange(V) % 50 == 3, np.arange(V) % 50 == 7
    for b in range(B):
        e = np.exp(y[b, 0])
        more = (e[up] * (np.e - 1)).sum()
        if more >= 0.9 * e[down].sum():
            more, scale = 0.5 * e[down].sum(), np.log1p(0.5 * e[down].sum() / e[up].sum())
        else:
            scale = 1.0
        x[b, 0, up] += np.float32(scale)
        x[b, 0] = x[b, 0].astype(np.float32)
        gain = (np.exp(x[b, 0, up]) - e[up]).sum()
        x[b, 0, down] += np.float32(np.log1p(-gain / e[down].sum()))
        x[b, 0] = x[b, 0].astype(np.float32)
        # (both sides of the line, and nearer to it than roundings of the shifted ones allow: one token takes up the rest)
        at = np.flatnonzero(down)[0]
        left = np.exp(x[b, 0]).sum() - e.sum() - np.exp(x[b, 0, at])
        x[b, 0, at] = np.float32(np.log(max(1e-30, -left) * (1 + (1e-6 if b % 2 else -1e-6))))
    bx, px, xv = block(x, "f32", V, 2 * V)
    by, py, yv = block(y, "f32", V, V)
    tokens, u = refused(yv[:, 0], xv[:, 0])
    for w in (0.0, 0.01, 0.3, 0.999):
        numbers = np.tile([u, w], (B, 1))
        got = run_verify(px, py, "f32", (V, 2 * V), (V, V), B, 1, V, 1.0, 1.0, tokens[:, None], numbers)
        check_verify(got, xv, yv, 1.0, 1.0, tokens[:, None], numbers, (V, w))
        assert (got[1] == 0).all()


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("V", [700, 5000, 20011, 131072])
def test_verify_rows_that_are_all_but_equal(V, kind):
    """Flat rows but for a few tokens that differ by 1e-5 (1e-2 in one case): numbers next to p / q, a rest of next to nothing."""
    rng = np.random.default_rng(V + 1)
    B = 6
    y = np.zeros((B, 1, V))
    x = np.zeros((B, 2, V))
    for b in range(B):
        size = 1e-2 if b == 5 else 1e-5
        x[b, 0, rng.integers(0, V, 5)] = size
        y[b, 0, rng.integers(0, V, 5)] = size * 2
    bx, px, xv = block(x, kind, V, 2 * V)
    by, py, yv = block(y, kind, V, V)
    tokens, u = refused(yv[:, 0], xv[:, 0])
    p = np.array([S.probabilities(xv[b, 0], 1.0)[0][tokens[b]] / S.probabilities(yv[b, 0], 1.0)[0][tokens[b]] for b in range(B)])
    for shift in (-2, -1, 1, 2):    # (fp32 numbers on either side of the line, but not on it)
        number = (np.float32(p) + shift * np.spacing(np.float32(p))).astype(np.float32)
        numbers = np.stack([number, rng.random(B).astype(np.float32)], axis=1)
        got = run_verify(px, py, kind, (V, 2 * V), (V, V), B, 1, V, 1.0, 1.0, tokens[:, None], numbers)
        check_verify(got, xv, yv, 1.0, 1.0, tokens[:, None], numbers, (V, kind, shift))
        assert (got[1] == (shift < 0)).all()


@pytest.mark.parametrize("V,sure", [(1025, False), (12000, False), (40000, False), (1025, True), (40000, True), (400000 - 7000, True)])
def test_verify_rows_behind_the_end_are_not_read(V, sure):
    n = 4
    rng = np.random.default_rng(0)
    x, y = rng.normal(0, 2, (3, n + 1, V)), rng.normal(0, 2, (3, n, V))
    tokens = y.argmax(axis=2)
    for b, end in enumerate((0, 1, 3)):
        tokens[b, end] = -1
        x[b, end + 1:], y[b, end:] = np.nan, np.nan
    bx, px, xv = block(x, "bf16", V, (n + 1) * V)
    by, py, yv = block(y, "bf16", V, n * V)
    numbers = np.zeros((3, n + 1))
    got = run_verify(px, None if sure else py, "bf16", (V, (n + 1) * V), (V, n * V), 3, n, V, 1.0, 1.0, tokens, numbers)
    assert list(got[1]) == [0, 1, 3]
    check_verify(got, xv, None if sure else yv, 1.0, 1.0, tokens, numbers, "ends")


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("B,n,V", [(1, 0, 393216), (3, 0, 16385), (40, 0, 50001), (2, 1, 131072), (5, 2, 33000), (2, 63, 16390), (1, 4, 393215), (5, 9, 150001), (6, 9, 150001), (300, 0, 17000)])
def test_verify_long_rows_without_a_draft(kind, B, n, V):
    """Rows without a draft's, few elements and many: summed in 64 bits at once, or in three steps."""
    rng = np.random.default_rng(V + n)
    x, y = rows_for(rng, B, n, V, kind, True)
    tokens, numbers = tokens_of(rng, x, x[:, :n], True), numbers_of(rng, B, n, True)
    if n:  # (a token that has all of its row: nothing is left beside it)
        x[0, 0], tokens[0, 0], numbers[0, 0] = -np.inf, V // 2, 1.0
        x[0, 0, V // 2] = 1.0
        x[-1, 0, V // 3], tokens[-1, 0], numbers[-1, 0] = 40.0, V // 3, np.nan
    T, pad = float(rng.choice([0.5, 1.0, 1.25])), int(rng.choice([0, 3]))
    bx, px, xv = block(x, kind, V + pad, (n + 1) * (V + pad), int(rng.choice([0, 1])))
    got = run_verify(px, None, kind, (V + pad, (n + 1) * (V + pad)), (0, 0), B, n, V, T, 1.0, tokens, numbers)
    check_verify(got, xv, None, T, 1.0, tokens, numbers, (kind, B, n, V))


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("V", [600, 6000, 40000, 131072])
@pytest.mark.parametrize("drafted", [False, True, None])
def test_weights_that_are_none_each(kind, V, drafted):
    """Thousands of tokens with weights just below those that count, in front of the one that has all: not drawn at a number of 0."""
    n = 0 if drafted is None else 1
    x, y = np.full((2, n + 1, V), -np.inf), np.full((2, n, V), -np.inf)
    x[:, :, :V - 100] = -668.0
    x[:, :, V - 50] = 0.0
    x[1, :, V - 70] = -664.0  # (this one counts)
    if n:
        y[:, :, V - 10] = 0.0
    tokens, numbers = np.full((2, n), V - 10), np.zeros((2, n + 1))
    bx, px, xv = block(x, kind, V, (n + 1) * V)
    py, yv = None, None
    if drafted:
        by, py, yv = block(y, kind, V, n * V)
    got = run_verify(px, py, kind, (V, (n + 1) * V), (V, n * V), 2, n, V, 1.0, 1.0, tokens, numbers)
    assert list(got[1]) == [0, 0] and list(got[0][:, 0]) == [V - 50, V - 70]


@pytest.mark.parametrize("n,V", [(0, 20000), (1, 600)])
def test_verify_more_sequences_than_a_launch_takes(n, V):
    B, g = 33000, torch.Generator(device=DEV)
    g.manual_seed(V)
    x = torch.empty((B, n + 1, V), dtype=torch.bfloat16, device=DEV)
    for s in range(0, B, 3000):
        x[s:s + 3000] = (torch.randn((min(3000, B - s), n + 1, V), generator=g, device=DEV) * 2).bfloat16()
    tokens = torch.randint(0, V, (B, n), generator=g, device=DEV, dtype=torch.int32)
    numbers = torch.rand((B, n + 1), generator=g, device=DEV)

    def run(first, count):
        out, acc = torch.full((count, n + 1), -7, dtype=torch.int32, device=DEV), torch.full((count,), -7, dtype=torch.int32, device=DEV)
        lp = torch.full((count, n + 1), JUNK, device=DEV)
        size = pb.pb_verify_draft_workspace_bytes(pb.PB_BF16, count, n, V)
        ws = workspace(size)
        pb.pb_verify_draft(x[first:], None, pb.PB_BF16, (n + 1) * V, V, V, V, count, n, V, 1.0, 1.0, tokens[first:] if n else None, numbers[first:], out, acc,
                           lp, ws, size, stream_ptr())
        assert guard_ok(ws, size)
        return out, acc, torch.nan_to_num(lp, nan=9.0)
    whole = run(0, B)
    for first in (0, 16500, 32700):
        for a, b in zip(whole, run(first, 300)):
            # (log-probs of accepted tokens: sums are the same in any call)
            assert torch.equal(a[first:first + 300], b)
    rows = [0, 1, 32767, 32768, B - 1]
    got = [w[rows].cpu().numpy() for w in whole]
    check_verify((got[0], got[1], None), host(x[rows]), None, 1.0, 1.0, tokens[rows].cpu().numpy(), numbers[rows].cpu().numpy(), "sequences")


def test_verify_two_calls_at_once():
    """On two streams, a workspace each; equal to one after the other."""
    rng = np.random.default_rng(8)
    V, n = 40000, 3
    calls = []
    for k in range(2):
        x = torch.from_numpy(rng.normal(0, 2, (16, n + 1, V)).astype(np.float32)).to(DEV)
        y = (x[:, :n] + torch.randn((16, n, V), device=DEV)).contiguous()
        calls.append((x, y, y.argmax(dim=2).to(torch.int32), torch.rand((16, n + 1), device=DEV)))
    size = pb.pb_verify_draft_workspace_bytes(pb.PB_F32, 16, n, V)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()

    def go(k, stream, ws):
        x, y, t, u = calls[k]
        out, acc = torch.empty((16, n + 1), dtype=torch.int32, device=DEV), torch.empty(16, dtype=torch.int32, device=DEV)
        pb.pb_verify_draft(x, y, pb.PB_F32, (n + 1) * V, V, n * V, V, 16, n, V, 1.0, 1.0, t, u, out, acc, None, ws, size, stream)
        return out, acc
    spaces = [workspace(size) for _ in range(2)]
    torch.cuda.synchronize()
    for turn in range(5):
        at_once = [go(k, int(streams[k].cuda_stream), spaces[k]) for k in range(2)]
        torch.cuda.synchronize()
        for k in range(2):
            one = go(k, stream_ptr(), spaces[0])
            torch.cuda.synchronize()
            assert torch.equal(one[0], at_once[k][0]) and torch.equal(one[1], at_once[k][1])


# ---- graphs, streams, a run of them ------------------------------------------------------------------------------------

@pytest.mark.parametrize("n,V,N,rows,dim", [(3, 5000, 3000, 700, 96), (0, 40001, 9000, 9000, 96), (2, 30000, 50000, 70001, 40), (3, 9001, 5000, 20001, 200), (1, 600, 100, 30, 1)])
def test_captured_and_replayed(n, V, N, rows, dim):
    """Two graphs with a workspace each, replayed in turn with eager calls between them; every replay equals the eager result."""
    rng = np.random.default_rng(2)
    B = 4
    x, y = rng.normal(0, 2, (B, n + 1, V)), rng.normal(0, 2, (B, n, V))
    X, Y = (torch.from_numpy(a.astype(np.float32)).to(DEV) for a in (x, y))
    Y = Y if n else None
    tokens, numbers = dev(y.argmax(axis=2).astype(np.int32)) if n else None, dev(rng.random((B, n + 1)).astype(np.float32))
    toks = dev(tokens_for(rng, N, rows, 0.1, 0.2).astype(np.int32))
    table, grad = torch.randn((rows, dim), device=DEV), torch.randn((N, dim), device=DEV)

    class Run:
        def __init__(self):
            self.out = torch.zeros((B, n + 1), dtype=torch.int32, device=DEV)
            self.acc, self.lp = torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros((B, n + 1), device=DEV)
            self.looked, self.tg, self.norm = torch.zeros((N, dim), device=DEV), torch.zeros((rows, dim), device=DEV), torch.zeros(1, device=DEV)
            self.clipped = torch.zeros((rows, dim), device=DEV)
            self.set, self.to = (pb.pb_tensors_build([t], [t.numel()], [pb.PB_F32]) for t in (self.tg, self.clipped))
            sizes = (pb.pb_verify_draft_workspace_bytes(pb.PB_F32, B, n, V), pb.pb_embed_tokens_backward_workspace_bytes(N, rows, dim),
                     pb.pb_grad_norm_workspace_bytes(self.set))
            self.ws = [workspace(s, 0) for s in sizes]

        def go(self):
            s = int(torch.cuda.current_stream().cuda_stream)
            pb.pb_verify_draft(X, Y, pb.PB_F32, (n + 1) * V, V, n * V, V, B, n, V, 1.0, 1.0, tokens, numbers, self.out, self.acc, self.lp, self.ws[0],
                               self.ws[0].numel(), s)
            pb.pb_embed_tokens(table, pb.PB_F32, dim, rows, dim, 0.5, toks, N, self.looked, pb.PB_F32, dim, s)
            pb.pb_embed_tokens_backward(grad, pb.PB_F32, dim, toks, N, rows, dim, 0.5, 0, self.tg, pb.PB_F32, dim, self.ws[1], self.ws[1].numel(), s)
            pb.pb_grad_norm(self.set, self.norm, self.ws[2], self.ws[2].numel(), s)
            pb.pb_grad_clip(self.set, self.norm, 1.0, self.to, s)

        def results(self):
            return [t.clone() for t in (self.out, self.acc, self.lp, self.looked, self.tg, self.norm, self.clipped)]

    eager, runs, graphs = Run(), [Run(), Run()], []
    for r in runs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r.go()
        graphs.append(g)
    for turn in range(4):
        X.copy_(X.roll(1, 0) + 0.1)
        numbers.copy_(torch.rand((B, n + 1), device=DEV))
        toks.copy_(toks.roll(7))
        grad.mul_(1.25)
        for g, r in zip(graphs, runs):
            g.replay()
        eager.go()
        torch.cuda.synchronize()
        for r in runs:
            for a, b in zip(r.results(), eager.results()):
                assert torch.equal(torch.nan_to_num(a, nan=-9.0) if a.is_floating_point() else a, torch.nan_to_num(b, nan=-9.0) if b.is_floating_point() else b), turn


def test_another_stream():
    rng = np.random.default_rng(6)
    side = torch.cuda.Stream()
    V, N, dim = 300, 2000, 40
    with torch.cuda.stream(side):
        g = torch.randn((N, dim), device=DEV)
        tokens = tokens_for(rng, N, V, 0.1, 0.3)
        out = torch.full((V, dim), JUNK, device=DEV)
        run_backward(g, "f32", dim, tokens, V, dim, 1.0, 0, out, "f32", dim)
        norm = run_norm(set_of([(out, out, "f32")]))
    side.synchronize()
    total, bound, _ = S.table_gradient(host(g), tokens, V, 1.0)
    R.check(host(out), total, R.rounded(bound, total, "f32"), "stream")
    assert abs(float(norm) - S.norm([host(out)])) <= float(norm) * 2 * S.U


def test_a_students_step_and_its_drafts():
    """Lookup, a head, distillation from a teacher's alternatives, the gradients back to the table, their norm and clipping, held
    to the same step in 64 bits; then the student drafts, and the teacher's rows verify."""
    rng = np.random.default_rng(4)
    N, V, dim, K, T, scale = 96, 257, 48, 8, 1.0, 4.0
    s = stream_ptr()
    table, head = (torch.from_numpy(rng.normal(0, 0.5, sh).astype(np.float32)).to(DEV) for sh in ((V, dim), (V, dim)))
    tokens = tokens_for(rng, N, V, 0.0, 0.5)
    toks = dev(tokens.astype(np.int32))
    teacher = torch.from_numpy(rng.normal(0, 2, (N, V)).astype(np.float32)).to(DEV)
    top, top_lp = torch.empty((N, K), dtype=torch.int32, device=DEV), torch.empty((N, K), device=DEV)
    pb.pb_token_logprobs(teacher, pb.PB_F32, V, N, V, T, None, 0, K, None, None, top, top_lp, None, None, 0, s)
    rows, logits_grad, loss = torch.empty((N, dim), device=DEV), torch.empty((N, V), device=DEV), torch.empty(N, device=DEV)
    pb.pb_embed_tokens(table, pb.PB_F32, dim, V, dim, scale, toks, N, rows, pb.PB_F32, dim, s)
    logits = rows @ head.t().contiguous()
    pb.pb_distill_topk(logits, pb.PB_F32, V, N, V, T, top, top_lp, K, pb.PB_DISTILL_TAIL, torch.full((N,), 1.0 / N, device=DEV), loss, logits_grad, V, None, 0, s)
    rows_grad, head_grad = logits_grad @ head, logits_grad.t().contiguous() @ rows
    table_grad = torch.empty_like(table)
    size = pb.pb_embed_tokens_backward_workspace_bytes(N, V, dim)
    ws = workspace(size, 0)
    pb.pb_embed_tokens_backward(rows_grad, pb.PB_F32, dim, toks, N, V, dim, scale, 0, table_grad, pb.PB_F32, dim, ws, size, s)
    grads = pb.pb_tensors_build([table_grad, head_grad], [V * dim] * 2, [pb.PB_F32] * 2)
    norm = run_norm(grads)
    before = [host(table_grad), host(head_grad)]
    pb.pb_grad_clip(grads, norm, float(norm) / 3, None, s)
    # the same in 64 bits
    w, h = (t.double().cpu().requires_grad_() for t in (table, head))
    lp = torch.log_softmax((w[torch.from_numpy(tokens)] * scale) @ h.t() / T, dim=1)
    q, at = top_lp.double().cpu().exp(), top.long().cpu()
    rest = 1 - q.sum(dim=1)
    p_rest = 1 - lp.exp().gather(1, at).sum(dim=1)
    want = ((q * (q.log() - lp.gather(1, at))).sum(dim=1) + rest * (rest.log() - p_rest.log())).mean()
    want.backward()
    assert abs(loss.double().mean().item() - want.item()) <= 1e-5 * want.item()
    # (fp32 products over V = 257 and N = 96 terms and the loss' own 1e-6: 1e-5 of the norm is room for the chain of them)
    for got, ref in zip(before, (w.grad, h.grad)):
        assert np.linalg.norm(got - ref.numpy()) <= 1e-5 * np.linalg.norm(ref.numpy())
    full = S.norm([w.grad.numpy(), h.grad.numpy()])
    assert abs(float(norm) - full) <= 1e-5 * full
    for got, ref in zip((table_grad, head_grad), before):
        assert np.abs(host(got) - ref / 3).max() <= 4 * S.U * np.abs(ref).max()
    # drafting: tokens drawn from the student's rows, verified by the teacher's
    B, n = 24, 3
    y, x = logits.view(B, N // B, V), teacher.view(B, N // B, V)
    drafts = torch.empty((B, N // B), dtype=torch.int32, device=DEV)
    drawn, none = torch.empty((N, 1), dtype=torch.int32, device=DEV), torch.empty(N, dtype=torch.int32, device=DEV)
    numbers = torch.from_numpy(rng.random((N, 1)).astype(np.float32)).to(DEV)
    size = pb.pb_verify_draft_workspace_bytes(pb.PB_F32, N, 0, V)
    ws = workspace(size, 0)
    pb.pb_verify_draft(logits, None, pb.PB_F32, V, V, 0, 0, N, 0, V, T, T, None, numbers, drawn, none, None, ws, size, s)
    drafts = drawn.view(B, N // B)[:, :n].contiguous()
    xv, yv = host(x), host(y)
    check = [S.drawn(S.probabilities(yv.reshape(N, V)[r], T)[0], float(numbers[r, 0])) for r in range(N)]
    assert drawn[:, 0].tolist() == check and not none.any()
    u = rng.random((B, n + 1))
    got = run_verify(x, y, "f32", (V, N // B * V), (V, N // B * V), B, n, V, T, T, drafts.cpu().numpy(), u)
    check_verify(got, xv[:, :n + 1], yv[:, :n], T, T, drafts.cpu().numpy(), u.astype(np.float32), "drafts")
