"""The transformer block's operators on the GPU at the ends of what their documentation allows, against the 64-bit oracle.

Tolerances are those of test_gpu_block.py, from the same arithmetic."""
import pytest

torch = pytest.importorskip("torch")

import paper_2104_05588_amd as daso  # noqa: E402
from tests.test_gpu_block import BF16, F32, check_rotary, rotary_case  # noqa: E402
from tests.test_gpu_train import announce  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]


# ------------------------------------------------------- norm and rotation
# heads that leave lanes of a token's last wavefront without one, and heads that do not
@pytest.mark.parametrize("n,heads,kv,dim,rotated", [(1, 1, 1, 8, 8), (70, 4, 2, 64, 64), (61, 6, 3, 80, 80), (4100, 4, 2, 64, 32), (5000, 3, 2, 128, 128),
                                                    (33, 20, 13, 32, 16), (9, 32, 8, 128, 128)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("inter,affine", [(False, True), (True, False)])
def test_head_norm_rotary_without_eps(n, heads, kv, dim, rotated, dtype, inter, affine):
    announce("head_norm_rotary without eps", n, heads, kv, dim, rotated, dtype, inter, affine)
    q, k, dq, dk, at, qw, kw, freq = rotary_case(n, heads, kv, dim, rotated, dtype, 0, n + dim)
    if not affine:
        qw = kw = None
    args = (at.cuda(), freq.cuda(), None if qw is None else qw.cuda(), None if kw is None else kw.cuda())
    yq, yk = daso.head_norm_rotary(q.cuda(), k.cuda(), *args, eps=0.0, interleaved=inter)
    dxq, dxk, dqw, dkw = daso.head_norm_rotary_backward(dq.cuda(), dk.cuda(), q.cuda(), k.cuda(), *args, eps=0.0, interleaved=inter)
    check_rotary(q, dq, at, qw, freq, inter, yq, dxq, dqw, dtype, eps=0.0)
    check_rotary(k, dk, at, kw, freq, inter, yk, dxk, dkw, dtype, eps=0.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,kv,dim,inter", [(5, 2, 64, False), (4, 4, 128, True), (6, 3, 24, False)])
@pytest.mark.parametrize("size,eps", [(1e18, 1e-6), (1e20, 1e-6), (3e37, 1e-6), (3e37, 3e38), (1e-18, 0.0), (1e-25, 0.0), (1e-36, 0.0), (1e-25, 1e-50),
                                      (1e-25, 1e-6)])
def test_heads_of_any_size_have_their_norm(dtype, heads, kv, dim, inter, size, eps):
    """Squares beyond the range of 32 bits, beside heads of ordinary size in the same wavefront.  Gradients are of sizes that
    leave dx in range."""
    announce("heads' sizes", dtype, heads, kv, dim, inter, size, eps)
    q, k, dq, dk, at, qw, kw, freq = rotary_case(37, heads, kv, dim, dim, dtype, 0, dim)
    q, k, dq, dk = (t.float() for t in (q, k, dq, dk))
    large = min(size, 1e15) if size > 1 else max(size, 1e-15)
    q[:, ::2] *= size
    dq[:, ::2] *= large
    k[1::3] *= size
    dk[1::3] *= large
    q, k, dq, dk = (t.to(dtype) for t in (q, k, dq, dk))
    assert torch.isfinite(q).all() and torch.isfinite(k).all()
    args = (at.cuda(), freq.cuda(), qw.cuda(), kw.cuda())
    eps = float(torch.tensor(eps))  # as the call has it
    yq, yk = daso.head_norm_rotary(q.cuda(), k.cuda(), *args, eps=eps, interleaved=inter)
    dxq, dxk, dqw, dkw = daso.head_norm_rotary_backward(dq.cuda(), dk.cuda(), q.cuda(), k.cuda(), *args, eps=eps, interleaved=inter)
    check_rotary(q, dq, at, qw, freq, inter, yq, dxq, dqw, dtype, eps=eps)
    check_rotary(k, dk, at, kw, freq, inter, yk, dxk, dkw, dtype, eps=eps)
