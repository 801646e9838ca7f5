"""More of the calls around a student without a GPU: handles that are gone."""
import pytest

import paper_2508_07014_amd as pb
from paper_2508_07014_amd import binding as B

P = 0x7f0000001000  # an address that nobody looks at


def test_a_closed_set_to_write_to_is_not_in_place(monkeypatch):
    """No address means "in place" to the C call; a set that was closed has none, and is refused before it."""
    pb.load()
    seen = []

    class Set:  # (a handle that nothing frees)
        def __init__(self, handle):
            self.handle = handle

    class Calls:
        @staticmethod
        def pb_grad_clip(*args):
            seen.append(args)
            return pb.PB_OK
    monkeypatch.setattr(B, "_student", Calls)
    grads, out = Set(P), Set(None)
    with pytest.raises(pb.PbError) as e:
        pb.pb_grad_clip(grads, P, 1.0, out)
    assert e.value.code == pb.PB_EINVAL and not seen
    pb.pb_grad_clip(grads, P, 1.0)
    out.handle = P + 64
    pb.pb_grad_clip(grads, P, 1.0, out)
    assert [a[3] for a in seen] == [None, P + 64]
