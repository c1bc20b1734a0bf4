"""Calls of the training operators at the edges of what they take: in place at every length, operands of any size.
Tolerances as derived in test_gpu_train."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2104_05588_amd as daso  # noqa: E402
from tests.test_gpu_train import announce, check_loss, gen, loss_case  # noqa: E402

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


# ------------------------------------------------------------------------- the loss
@pytest.mark.parametrize("hs,ws", [(1e-19, 1e-19), (1e-36, 1e-3), (1e-3, 1e-36), (3e-38, 3e-38)])
@pytest.mark.parametrize("v", [200, 256])
def test_loss_of_tiny_operands(hs, ws, v):
    """Logits next to zero, or that underflow: log V, with classes that fill a tile or do not."""
    announce("loss of tiny operands", hs, ws, v)
    h, w, t, s = loss_case(70, v, 96, torch.float32, 0.2, 31)
    h, w = h * hs, w * ws
    check_loss(h, w, t, s, h.cuda(), w.cuda())
    loss, lse = daso.linear_cross_entropy(h.cuda(), w.cuda(), t.cuda())
    assert (lse.cpu().double() - np.log(v)).abs().max() < 2.0 ** -18


def test_loss_of_huge_operands_that_do_not_meet():
    """hidden and weight have no feature in common: every logit is zero, whatever their size."""
    announce("loss of huge operands")
    h, w, t, s = loss_case(70, 200, 96, torch.float32, 0.2, 32)
    h[:, 48:], w[:, :48] = 0, 0
    h, w = h * 1e25, w * 1e25
    check_loss(h, w, t, s * 1e-20, h.cuda(), w.cuda())
