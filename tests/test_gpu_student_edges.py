"""More of the calls around a student on the GPU: handles that are gone, log-probs of near-certain tokens, what
is left of rows that differ in two places."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2508_07014_amd as pb  # noqa: E402
import student as S  # noqa: E402
from gpu_helpers import DEV, stream_ptr  # noqa: E402
from test_gpu_logits import KIND  # noqa: E402
from test_gpu_student import block, run_verify  # noqa: E402


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
