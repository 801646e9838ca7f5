"""More of the calls around a student on the GPU: handles that are gone."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2508_07014_amd as pb  # noqa: E402
from gpu_helpers import DEV, stream_ptr  # noqa: E402


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
