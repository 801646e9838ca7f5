"""Calls on rows of logits without a GPU: what is refused, workspace sizes, the binding, and the 64-bit definitions that the
GPU tests hold the kernels to against difference quotients."""
import ctypes as C

import numpy as np
import pytest

import logit_rows as R
import paper_2508_07014_amd as pb
from paper_2508_07014_amd import binding as B

P = 0x7f0000001000  # an address that no refused call looks at
ODD = 1

LP = dict(d_logits=P, dtype=pb.PB_F32, row_stride=16, rows=2, vocab_size=16, temperature=1.0, d_tokens=P, n_tokens=1, n_top=2,
          d_logp=P, d_entropy=P, d_top_tokens=P, d_top_logp=P, d_stats=P, d_workspace=None, workspace_bytes=0, stream=0)
BACK = dict(d_logits=P, dtype=pb.PB_F32, row_stride=16, rows=2, vocab_size=16, temperature=1.0, d_stats=P, d_tokens=P,
            n_tokens=1, d_grad_logp=P, d_grad_entropy=P, d_grad_logits=P + 4096, grad_stride=16, stream=0)
DIST = dict(d_logits=P, dtype=pb.PB_F32, row_stride=16, rows=2, vocab_size=16, temperature=1.0, d_teacher_tokens=P,
            d_teacher_logp=P, K=2, mode=0, d_row_grads=P, d_loss=P, d_grad_logits=P + 4096, grad_stride=16,
            d_workspace=None, workspace_bytes=0, stream=0)


def code(call, base, **change):
    try:
        call(**{**base, **change})
    except pb.PbError as e:
        return e.code
    return pb.PB_OK


COMMON = [(dict(rows=-1), pb.PB_EINVAL), (dict(vocab_size=0, row_stride=16), pb.PB_EINVAL), (dict(dtype=3), pb.PB_EINVAL),
          (dict(dtype=-1), pb.PB_EINVAL), (dict(row_stride=15), pb.PB_EINVAL), (dict(row_stride=-16), pb.PB_EINVAL),
          (dict(d_logits=None), pb.PB_EINVAL), (dict(d_logits=P + ODD), pb.PB_EINVAL), (dict(d_logits=P + 2), pb.PB_EINVAL),
          (dict(d_logits=P + ODD, dtype=pb.PB_BF16), pb.PB_EINVAL),
          (dict(temperature=0.0), pb.PB_ERANGE), (dict(temperature=-1.0), pb.PB_ERANGE), (dict(temperature=float("nan")), pb.PB_ERANGE),
          (dict(temperature=float("inf")), pb.PB_ERANGE), (dict(temperature=1e-5), pb.PB_ERANGE), (dict(temperature=1e5), pb.PB_ERANGE),
          (dict(vocab_size=393217, row_stride=1 << 20, grad_stride=1 << 20), pb.PB_EUNSUPPORTED), (dict(rows=0), pb.PB_OK)]


@pytest.mark.parametrize("change,want", COMMON + [
    (dict(n_tokens=-1), pb.PB_EINVAL), (dict(n_top=-1), pb.PB_EINVAL), (dict(n_top=17), pb.PB_EINVAL),
    (dict(n_tokens=65), pb.PB_EUNSUPPORTED), (dict(n_top=65, vocab_size=100, row_stride=100), pb.PB_EUNSUPPORTED),
    (dict(d_tokens=None), pb.PB_EINVAL), (dict(d_logp=None), pb.PB_EINVAL), (dict(d_top_tokens=None), pb.PB_EINVAL),
    (dict(d_top_logp=None), pb.PB_EINVAL), (dict(n_tokens=0), pb.PB_EINVAL), (dict(n_top=0), pb.PB_EINVAL),
    (dict(n_tokens=0, n_top=0, d_tokens=None, d_logp=None, d_top_tokens=None, d_top_logp=None, d_entropy=None, d_stats=None), pb.PB_EINVAL),
    (dict(d_logp=P + 2), pb.PB_EINVAL), (dict(d_stats=P + 2), pb.PB_EINVAL), (dict(d_entropy=P + 1), pb.PB_EINVAL),
    (dict(workspace_bytes=-1), pb.PB_EINVAL)])
def test_logprobs_refusals(change, want):
    change = {k: v for k, v in change.items() if k in LP}
    assert code(pb.pb_token_logprobs, LP, **change) == want


@pytest.mark.parametrize("change,want", COMMON + [
    (dict(n_tokens=-1), pb.PB_EINVAL), (dict(n_tokens=65), pb.PB_EUNSUPPORTED), (dict(grad_stride=15), pb.PB_EINVAL),
    (dict(d_stats=None), pb.PB_EINVAL), (dict(d_grad_logits=None), pb.PB_EINVAL), (dict(d_tokens=None), pb.PB_EINVAL),
    (dict(d_grad_logp=None, d_grad_entropy=None), pb.PB_EINVAL), (dict(n_tokens=0, d_tokens=None), pb.PB_EINVAL),
    (dict(d_grad_logits=P, grad_stride=17), pb.PB_EINVAL), (dict(d_grad_logits=P + 4097), pb.PB_EINVAL),
    (dict(d_stats=P + 1), pb.PB_EINVAL)])
def test_backward_refusals(change, want):
    change = {k: v for k, v in change.items() if k in BACK}
    assert code(pb.pb_token_logprobs_backward, BACK, **change) == want


@pytest.mark.parametrize("change,want", COMMON + [
    (dict(K=0), pb.PB_EINVAL), (dict(K=65), pb.PB_EUNSUPPORTED), (dict(mode=2), pb.PB_EINVAL), (dict(mode=-1), pb.PB_EINVAL),
    (dict(d_teacher_tokens=None), pb.PB_EINVAL), (dict(d_teacher_logp=None), pb.PB_EINVAL), (dict(grad_stride=15), pb.PB_EINVAL),
    (dict(d_loss=None, d_grad_logits=None), pb.PB_EINVAL), (dict(d_loss=P + 2), pb.PB_EINVAL), (dict(d_row_grads=P + 2), pb.PB_EINVAL),
    (dict(d_grad_logits=P, grad_stride=17), pb.PB_EINVAL), (dict(workspace_bytes=-1), pb.PB_EINVAL)])
def test_distill_refusals(change, want):
    change = {k: v for k, v in change.items() if k in DIST}
    assert code(pb.pb_distill_topk, DIST, **change) == want


def test_workspaces():
    lp, di = pb.pb_token_logprobs_workspace_bytes, pb.pb_distill_topk_workspace_bytes
    for size, last in ((lp, 5), (di, 5)):
        assert size(pb.PB_BF16, 0, 1000, last) == 0
        for bad, want in (((3, 1, 10, last), pb.PB_EINVAL), ((0, -1, 10, last), pb.PB_EINVAL), ((0, 1, 0, last), pb.PB_EINVAL),
                          ((0, 1, 393217, last), pb.PB_EUNSUPPORTED), ((0, 1, 1000, 65), pb.PB_EUNSUPPORTED)):
            with pytest.raises(pb.PbError) as e:
                size(*bad)
            assert e.value.code == want
    for call, base, size in ((pb.pb_token_logprobs, LP, lp), (pb.pb_distill_topk, DIST, di)):
        for kind in (pb.PB_F32, pb.PB_F16, pb.PB_BF16):
            for rows in (1, 7, 100, 2000):
                for V in (100, 5000, 131072, 393216):
                    need = size(kind, rows, V, base.get("n_top", 2))
                    assert 0 <= need <= 64 << 20
                    if need:  # too little, none, misaligned: refused before anything is launched
                        big = dict(base, dtype=kind, rows=rows, vocab_size=V, row_stride=V, grad_stride=V)
                        big = {k: v for k, v in big.items() if k in base}
                        for ws in (dict(d_workspace=None, workspace_bytes=need), dict(d_workspace=P, workspace_bytes=need - 1),
                                   dict(d_workspace=P + 8, workspace_bytes=need)):
                            assert code(call, big, **ws) == pb.PB_EINVAL


# p: pointer, l: 64-bit, i: 32-bit, f: float -- the C declarations, written out a second time
SIGNATURES = dict(pb_token_logprobs="piliifpiippppppl" + "p", pb_token_logprobs_backward="piliifppipppl" + "p",
                  pb_distill_topk="piliifppiippplpl" + "p")


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
    for name in B.ROW_CALLS:
        types = getattr(real, name).argtypes
        fn = C.CFUNCTYPE(C.c_int, *types)(lambda *a, name=name: seen.append((name,) + a) or 7)
        fn.argtypes, fn.restype = types, C.c_int
        keep.append(fn)
        setattr(lib, name, fn)
    assert sorted(SIGNATURES) == sorted(B.ROW_CALLS)
    try:
        if way == "ctypes":
            calls = B._CtypesCalls(lib, B.ROW_CALLS, 0)
        else:
            from paper_2508_07014_amd import _pbcall
            calls = B._bind_rows(lib)
            assert calls is _pbcall
        for name, sig in SIGNATURES.items():
            for none in (False, True):
                given, want = [], []
                for k, t in enumerate(sig):
                    v = {"p": P + 0x10000 * k, "l": (1 << 33) + k, "i": -3 - k, "f": 0.375 + k}[t]
                    if t == "p" and none:
                        v = None
                    want.append(v)
                    given.append(Buffer(v) if t == "p" and buffers and v and k + 1 < len(sig) else v)
                seen.clear()
                assert getattr(calls, name)(*given) == 7
                assert seen == [(name,) + tuple(want)]
    finally:
        B._bind_rows(real)


# ---- the definitions -------------------------------------------------------------------------------------------------

def _differences(f, x, h=1e-5):
    g = np.zeros_like(x)
    for j in range(len(x)):
        a, b = x.copy(), x.copy()
        a[j] += h
        b[j] -= h
        g[j] = (f(a) - f(b)) / (2 * h)
    return g


@pytest.mark.parametrize("seed", range(6))
def test_gradients_of_the_definitions_are_difference_quotients(seed):
    rng = np.random.default_rng(seed)
    V, M, K, T = 23, 4, 6, float(rng.choice([0.7, 1.0, 2.0]))
    x = rng.normal(0, 2, V)
    tokens = rng.integers(0, V, M)
    tokens[0] = tokens[1]           # twice
    tokens[2] = V                   # absent
    g, h = rng.normal(0, 1, M), float(rng.normal())

    def score(y):
        lp, _ = R.row_log_probs(y, T)
        ok = tokens < V
        return (g[ok] * lp[tokens[ok]]).sum() + h * R.entropy(lp)
    # (central differences: third derivatives of order 1 / T^3, times h^2 / 6; sums of order 10 rounded at 2^-53, over h)
    assert np.allclose(R.logprobs_grad(x, T, tokens, g, h)[0], _differences(score, x), atol=1e-8)
    t = rng.permutation(V)[:K]
    t[1] = -1
    if seed % 2:
        t[2] = t[3]
    l = R.row_log_probs(rng.normal(0, 2, V), T)[0][np.maximum(t, 0)]
    if seed % 2:
        l[3] = l[2] - 1.0
    for tail in (False, True):
        f = lambda y: R.distill(y, T, t, l, tail, 1.0)[0]  # noqa: E731
        assert np.allclose(R.distill(x, T, t, l, tail, 0.5)[1], 0.5 * _differences(f, x), atol=1e-8)


def test_definitions_by_hand():
    x = np.log(np.array([4.0, 2.0, 1.0, 1.0]))
    r = R.logprobs(x, 1.0, np.array([1, 4, -1]), 3)
    assert np.allclose(r["logp"][0], np.log(0.25)) and np.isnan(r["logp"][1:]).all()
    assert list(r["top"]) == [0, 1, 2] and np.allclose(r["entropy"], 1.75 * np.log(2))
    loss, grad, _, _ = R.distill(x, 1.0, np.array([0, 2]), np.log(np.array([0.5, 0.25])), True, 1.0)
    assert np.allclose(loss, 0.25 * np.log(2) + 0.25 * np.log(0.25 / 0.375))
    assert np.allclose(grad, [0.0, 0.25 * (1 - 2 / 3), 0.125 - 0.25, 0.125 * (1 - 2 / 3)])
