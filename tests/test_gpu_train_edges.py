"""Calls of the training operators at the edges of what they take.  Tolerances as derived in test_gpu_train."""
import pytest

torch = pytest.importorskip("torch")

import paper_2104_05588_amd as daso  # noqa: E402
from tests.test_gpu_train import announce, gen  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]


@pytest.mark.parametrize("d", [1024, 1025, 8192, 8193, 20000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_layer_norm_backward_in_place(d, dtype):
    """dx over dy gives the bits of a call that keeps dy, for rows of every kernel."""
    announce("norm backward in place", d, dtype)
    x, dy = ((torch.randn(37, d, generator=gen(d + k)) + 0.5).to(dtype).cuda() for k in range(2))
    w = torch.randn(d, generator=gen(d + 2)).cuda()
    _, mean, rstd = daso.layer_norm(x, w)
    dx, dw, db = daso.layer_norm_backward(dy, x, w, mean, rstd)
    same = dy.clone()
    dx2, dw2, db2 = daso.layer_norm_backward(same, x, w, mean, rstd, dx=same)
    assert dx2 is same and torch.equal(dx2, dx) and torch.equal(dw2, dw) and torch.equal(db2, db)
