"""The calls around a student without a GPU: what is refused, workspace sizes, the binding, and the 64-bit definitions that the
GPU tests hold the kernels to."""
import ctypes as C

import numpy as np
import pytest

import paper_2508_07014_amd as pb
import student as S
from paper_2508_07014_amd import binding as B

P = 0x7f0000001000  # an address that no refused call looks at
BIG = 1 << 40

EMBED = dict(d_table=P, table_dtype=pb.PB_F32, table_stride=16, vocab_size=10, dim=16, scale=1.0, d_tokens=P, n_tokens=4, d_out=P,
             out_dtype=pb.PB_BF16, out_stride=16, stream=0)
GRAD = dict(d_grad_out=P, grad_dtype=pb.PB_BF16, grad_stride=16, d_tokens=P, n_tokens=4, vocab_size=10, dim=16, scale=1.0, accumulate=0,
            d_grad_table=P, table_dtype=pb.PB_F32, table_stride=16, d_workspace=P, workspace_bytes=BIG, stream=0)
VERIFY = dict(d_target_logits=P, d_draft_logits=P, dtype=pb.PB_F32, target_seq_stride=80, target_row_stride=16, draft_seq_stride=64,
              draft_row_stride=16, sequences=2, n_draft=4, vocab_size=16, temperature=1.0, draft_temperature=1.0, d_draft_tokens=P,
              d_uniforms=P, d_tokens=P, d_accepted=P, d_logp=P, d_workspace=P, workspace_bytes=BIG, stream=0)


def code(call, base, **change):
    try:
        call(**{**base, **change})
    except pb.PbError as e:
        return e.code
    return pb.PB_OK


TABLE = [(dict(n_tokens=-1), pb.PB_EINVAL), (dict(vocab_size=0), pb.PB_EINVAL), (dict(dim=0), pb.PB_EINVAL), (dict(dim=-4), pb.PB_EINVAL),
         (dict(table_dtype=3), pb.PB_EINVAL), (dict(table_dtype=-1), pb.PB_EINVAL), (dict(table_stride=15), pb.PB_EINVAL),
         (dict(table_stride=-16), pb.PB_EINVAL), (dict(d_tokens=None), pb.PB_EINVAL), (dict(d_tokens=P + 2), pb.PB_EINVAL),
         (dict(scale=float("nan")), pb.PB_ERANGE), (dict(scale=float("inf")), pb.PB_ERANGE), (dict(scale=1e39), pb.PB_ERANGE),
         (dict(n_tokens=(1 << 24) + 1), pb.PB_EUNSUPPORTED), (dict(vocab_size=393217), pb.PB_EUNSUPPORTED),
         (dict(dim=65537, table_stride=1 << 20, out_stride=1 << 20, grad_stride=1 << 20), pb.PB_EUNSUPPORTED)]


@pytest.mark.parametrize("change,want", TABLE + [
    (dict(out_dtype=3), pb.PB_EINVAL), (dict(out_stride=15), pb.PB_EINVAL), (dict(d_table=None), pb.PB_EINVAL), (dict(d_out=None), pb.PB_EINVAL),
    (dict(d_table=P + 2), pb.PB_EINVAL), (dict(d_out=P + 1), pb.PB_EINVAL), (dict(n_tokens=0), pb.PB_OK),
    (dict(n_tokens=0, d_table=None, d_tokens=None, d_out=None), pb.PB_OK)])
def test_embed_refusals(change, want):
    assert code(pb.pb_embed_tokens, EMBED, **{k: v for k, v in change.items() if k in EMBED}) == want


@pytest.mark.parametrize("change,want", TABLE + [
    (dict(grad_dtype=-1), pb.PB_EINVAL), (dict(grad_stride=15), pb.PB_EINVAL), (dict(d_grad_out=None), pb.PB_EINVAL),
    (dict(d_grad_out=P + 1), pb.PB_EINVAL), (dict(d_grad_table=None), pb.PB_EINVAL), (dict(d_grad_table=P + 2), pb.PB_EINVAL),
    (dict(accumulate=2), pb.PB_EINVAL), (dict(accumulate=-1), pb.PB_EINVAL), (dict(workspace_bytes=-1), pb.PB_EINVAL),
    (dict(n_tokens=0, accumulate=1), pb.PB_OK), (dict(n_tokens=0, d_grad_table=None), pb.PB_EINVAL)])
def test_embed_backward_refusals(change, want):
    assert code(pb.pb_embed_tokens_backward, GRAD, **{k: v for k, v in change.items() if k in GRAD}) == want


@pytest.mark.parametrize("change,want", [
    (dict(sequences=-1), pb.PB_EINVAL), (dict(n_draft=-1), pb.PB_EINVAL), (dict(vocab_size=0), pb.PB_EINVAL), (dict(dtype=3), pb.PB_EINVAL),
    (dict(target_row_stride=15), pb.PB_EINVAL), (dict(target_seq_stride=15), pb.PB_EINVAL), (dict(draft_row_stride=15), pb.PB_EINVAL),
    (dict(draft_seq_stride=-64), pb.PB_EINVAL), (dict(d_target_logits=None), pb.PB_EINVAL), (dict(d_target_logits=P + 2), pb.PB_EINVAL),
    (dict(d_draft_logits=P + 1), pb.PB_EINVAL), (dict(d_draft_tokens=None), pb.PB_EINVAL), (dict(d_uniforms=None), pb.PB_EINVAL),
    (dict(d_tokens=None), pb.PB_EINVAL), (dict(d_accepted=None), pb.PB_EINVAL), (dict(n_draft=0, d_draft_tokens=None), pb.PB_EINVAL),
    (dict(n_draft=0, d_draft_logits=None), pb.PB_EINVAL), (dict(d_logp=P + 2), pb.PB_EINVAL), (dict(d_accepted=P + 2), pb.PB_EINVAL),
    (dict(d_uniforms=P + 2), pb.PB_EINVAL), (dict(d_tokens=P + 1), pb.PB_EINVAL), (dict(d_draft_tokens=P + 1), pb.PB_EINVAL),
    (dict(temperature=0.0), pb.PB_ERANGE), (dict(temperature=float("nan")), pb.PB_ERANGE), (dict(draft_temperature=1e5), pb.PB_ERANGE),
    (dict(draft_temperature=-1.0), pb.PB_ERANGE), (dict(vocab_size=393217, target_row_stride=1 << 20), pb.PB_EUNSUPPORTED),
    (dict(n_draft=64), pb.PB_EUNSUPPORTED), (dict(workspace_bytes=-1), pb.PB_EINVAL), (dict(sequences=0), pb.PB_OK)])
def test_verify_refusals(change, want):
    assert code(pb.pb_verify_draft, VERIFY, **change) == want


def test_sets_of_tensors_refused():
    lib = pb.load()
    out = C.c_void_p()
    one = (C.c_void_p * 1)(P), (C.c_int64 * 1)(4), (C.c_int32 * 1)(0)
    for bufs, sizes, kinds, n, device in ((None, one[1], one[2], 1, 0), (one[0], None, one[2], 1, 0), (one[0], one[1], None, 1, 0),
                                          (*one, 0, 0), (*one, -1, 0), (*one, 1, -1)):
        assert lib.pb_tensors_build(bufs, sizes, kinds, n, device, C.byref(out)) == pb.PB_EINVAL
    assert lib.pb_tensors_build(*one, 1, 0, None) == pb.PB_EINVAL
    for buffers, sizes, kinds, want in (([None], [1], [0], pb.PB_EINVAL), ([P], [-1], [0], pb.PB_EINVAL), ([P], [1], [3], pb.PB_EINVAL),
                                        ([P + 2], [1], [0], pb.PB_EINVAL), ([P + 1], [1], [2], pb.PB_EINVAL), ([P], [1 << 41], [0], pb.PB_EUNSUPPORTED),
                                        ([P, 2 * P], [1 << 39, (1 << 39) + 1], [2, 2], pb.PB_EUNSUPPORTED),
                                        ([], [], [], pb.PB_EINVAL), ([P], [1, 2], [0], pb.PB_EINVAL)):
        with pytest.raises(pb.PbError) as e:
            pb.pb_tensors_build(buffers, sizes, kinds)
        assert e.value.code == want
    assert lib.pb_tensors_free(None) == pb.PB_OK
    assert lib.pb_grad_norm_workspace_bytes(None) == pb.PB_EINVAL
    assert lib.pb_grad_norm(None, P, P, 1 << 20, None) == pb.PB_EINVAL and lib.pb_grad_clip(None, P, 1.0, None, None) == pb.PB_EINVAL


def test_workspaces():
    for kind in (pb.PB_F32, pb.PB_F16, pb.PB_BF16):
        assert pb.pb_verify_draft_workspace_bytes(kind, 0, 4, 1000) == 0
        for sequences in (1, 7, 256):
            for n in (0, 1, 63):
                for V in (1, 100, 131072, 393216):
                    need = pb.pb_verify_draft_workspace_bytes(kind, sequences, n, V)
                    assert 0 <= need <= 64 << 20 or sequences * n > 7 * 63
                    if not need:
                        continue
                    big = dict(VERIFY, dtype=kind, sequences=sequences, n_draft=n, vocab_size=V, target_row_stride=V, target_seq_stride=(n + 1) * V,
                               draft_row_stride=V, draft_seq_stride=n * V, d_draft_logits=P if n else None, d_draft_tokens=P if n else None)
                    for ws in (dict(d_workspace=None, workspace_bytes=need), dict(d_workspace=P, workspace_bytes=need - 1),
                               dict(d_workspace=P + 8, workspace_bytes=need)):
                        assert code(pb.pb_verify_draft, big, **ws) == pb.PB_EINVAL
    for n, V, dim in ((0, 1, 1), (4, 10, 16), (1000, 393216, 7), (131072, 131072, 2048)):
        need = pb.pb_embed_tokens_backward_workspace_bytes(n, V, dim)
        assert 0 < need <= 1 << 30
        call = dict(GRAD, n_tokens=n, vocab_size=V, dim=dim, grad_stride=dim, table_stride=dim)
        for ws in (dict(d_workspace=None, workspace_bytes=need), dict(d_workspace=P, workspace_bytes=need - 1), dict(d_workspace=P + 8, workspace_bytes=need)):
            assert code(pb.pb_embed_tokens_backward, call, **ws) == pb.PB_EINVAL
    for size, bad, want in ((pb.pb_verify_draft_workspace_bytes, (3, 1, 1, 10), pb.PB_EINVAL), (pb.pb_verify_draft_workspace_bytes, (0, 1, 64, 10), pb.PB_EUNSUPPORTED),
                            (pb.pb_verify_draft_workspace_bytes, (0, -1, 1, 10), pb.PB_EINVAL), (pb.pb_verify_draft_workspace_bytes, (0, 1, -1, 10), pb.PB_EINVAL),
                            (pb.pb_embed_tokens_backward_workspace_bytes, (-1, 10, 10), pb.PB_EINVAL), (pb.pb_embed_tokens_backward_workspace_bytes, (1, 10, 1 << 17), pb.PB_EUNSUPPORTED)):
        with pytest.raises(pb.PbError) as e:
            size(*bad)
        assert e.value.code == want


@pytest.mark.parametrize("V", [1, 129, 1025, 6145, 16000, 32001, 65536, 65537, 131072, 393216])
def test_workspaces_for_more_do_for_fewer(V):
    for dim in (1, 64, 2048):
        counts = sorted({*range(0, 200, 7), *range(4000, 4200, 3), *range(40900, 41100, 3), *range(65400, 65700, 5), *range(130900, 131200, 5), 70000, 200000, 1 << 20, 1 << 24})
        sizes = [pb.pb_embed_tokens_backward_workspace_bytes(n, V, dim) for n in counts]
        assert sizes == sorted(sizes), dim
    for kind in (pb.PB_F32, pb.PB_F16, pb.PB_BF16):
        for n in (0, 1, 3, 8, 15, 63):
            sizes = [pb.pb_verify_draft_workspace_bytes(kind, B, n, V) for B in [*range(0, 1400), 5000, 32768, 32769, 40000, 70000]]
            assert sizes == sorted(sizes), (kind, n)



# p: pointer, h: handle, l: 64-bit, i: 32-bit, f: float -- the C declarations, written out a second time
SIGNATURES = dict(pb_embed_tokens="piliifpipil" + "p", pb_embed_tokens_backward="pilpiiifipilpl" + "p", pb_grad_norm="hppl" + "p",
                  pb_grad_clip="hpfh" + "p", pb_verify_draft="ppilllliiiffppppppl" + "p")


class Buffer:
    def __init__(self, address):
        self.address = address

    def data_ptr(self):
        return self.address


@pytest.mark.parametrize("way", ["extension", "ctypes"])
@pytest.mark.parametrize("buffers", [False, True])
def test_every_argument_arrives_as_it_is(way, buffers):
    real, seen, keep = pb.load(), [], []

    class Recorder:
        pass
    lib = Recorder()
    for name in B.STUDENT_CALLS:
        types = getattr(real, name).argtypes
        fn = C.CFUNCTYPE(C.c_int, *types)(lambda *a, name=name: seen.append((name,) + a) or 7)
        fn.argtypes, fn.restype = types, C.c_int
        keep.append(fn)
        setattr(lib, name, fn)
    assert sorted(SIGNATURES) == sorted(B.STUDENT_CALLS)
    try:
        calls = B._bind_student(lib)
        if way == "ctypes":
            calls = type("Calls", (), {name: staticmethod(getattr(B._CtypesCalls(lib, [name], h), name)) for name, h in B.STUDENT_CALLS.items()})
        else:
            from paper_2508_07014_amd import _pbcall
            assert calls is _pbcall
        for name, sig in SIGNATURES.items():
            for none in (False, True):
                given, want = [], []
                for k, t in enumerate(sig):
                    v = {"p": P + 0x10000 * k, "h": P + 0x10000 * k, "l": (1 << 33) + k, "i": -3 - k, "f": 0.375 + k}[t]
                    if t == "p" and none:
                        v = None
                    want.append(v)
                    given.append(Buffer(v) if t == "p" and buffers and v and k + 1 < len(sig) else v)
                seen.clear()
                assert getattr(calls, name)(*given) == 7
                assert seen == [(name,) + tuple(want)]
    finally:
        B._bind_student(real)


# ---- the definitions -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("sure", [False, True])
def test_what_is_emitted_has_the_targets_distribution(sure):
    """One drafted token, all of its values, and numbers on a grid: the first emitted token's distribution is the target's."""
    rng = np.random.default_rng(3)
    V, T, Ty, G = 5, 0.75, 1.25, 400
    x, y = rng.normal(0, 1.5, (2, V)), rng.normal(0, 1.5, (1, V))
    p, q = S.probabilities(x[0], T)[0], S.probabilities(y[0], Ty)[0]
    emitted = np.zeros(V)
    grid = (np.arange(G) + 0.5) / G
    for t in range(V):
        for u in grid[::8] if sure else grid:
            out, k, _ = S.verify(x, None if sure else y, T, Ty, np.array([t]), np.array([u, 0.5]))
            share = (1.0 / V if sure else q[t]) / len(grid[::8] if sure else grid)
            if k == 1:
                emitted[out[0]] += share
            else:  # (the draw behind it, over a grid of its own)
                for w in grid[::20]:
                    emitted[S.verify(x, None if sure else y, T, Ty, np.array([t]), np.array([u, w]))[0][0]] += share / len(grid[::20])
    # (a number on a grid of m is off by at most 1 / m in each of the V tokens' shares)
    assert np.abs(emitted - p).max() <= V * (8.0 if sure else 1.0) / G + 20.0 / G


def test_verification_by_hand():
    ln = np.log
    x = ln(np.array([[0.5, 0.25, 0.25], [0.25, 0.25, 0.5]]))
    y = ln(np.array([[0.25, 0.25, 0.5]]))
    for u, k, w, first in ((0.4, 1, 0.0, 2), (0.6, 0, 0.0, 0), (0.6, 0, 0.99, 0)):
        out, got, logp = S.verify(x, y, 1.0, 1.0, np.array([2]), np.array([u, w]))
        assert got == k and out[0] == first and np.isclose(logp[0], ln(0.25 if k else 0.5))
        if k:  # the token behind it: the first one
            assert out[1] == 0 and np.isclose(logp[1], ln(0.25))
    assert S.verify(x, None, 1.0, 1.0, np.array([0]), np.array([0.5, 0.5]))[1] == 0          # u q < p is false
    assert S.verify(x, None, 1.0, 1.0, np.array([0]), np.array([0.75, 0.5]))[0][0] == 2      # of {1, 2}: the border belongs to the next
    assert list(S.verify(x, y, 1.0, 1.0, np.array([-1]), np.array([0.9, 0.5]))[0]) == [1, -1]
    assert S.drawn(np.zeros(3), 0.5) == -1 and S.drawn(np.array([0.0, 1.0, 0.0]), 0.0) == 1


def test_table_gradient_is_that_of_the_lookup():
    rng = np.random.default_rng(1)
    V, n, dim, scale = 6, 11, 3, 1.5
    tokens = rng.integers(-1, V + 1, n)
    g, table = rng.normal(size=(n, dim)), rng.normal(size=(V, dim))

    def score(w):
        rows = np.where(((tokens >= 0) & (tokens < V))[:, None], w[np.clip(tokens, 0, V - 1)], 0.0)
        return float((g * scale * rows).sum())
    got = S.table_gradient(g, tokens, V, scale)[0]
    h = 0.5  # (linear: differences are exact but for roundings)
    for v in range(V):
        for j in range(dim):
            a, b = table.copy(), table.copy()
            a[v, j] += h
            b[v, j] -= h
            assert abs((score(a) - score(b)) / (2 * h) - got[v, j]) <= 1e-12
