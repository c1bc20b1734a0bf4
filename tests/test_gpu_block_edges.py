"""The transformer block's operators on the GPU at the ends of what their documentation allows, against the 64-bit oracle.

Tolerances are those of test_gpu_block.py, from the same arithmetic."""
import pytest

torch = pytest.importorskip("torch")

import paper_2104_05588_amd as daso  # noqa: E402
from tests.test_gpu_block import BF16, F32, attention_case, check_attention, check_rotary, rotary_case  # noqa: E402
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


# --------------------------------------------------------------- attention
def sequences_of(offsets, n):
    """Pairs that ascend within the tokens and begin behind all such pairs before them."""
    out, end = [], 0
    for a, b in zip(offsets, offsets[1:]):
        if 0 <= a < b <= n:
            if a >= end:
                out.append((a, b))
            end = max(end, b)
    return out


APART = [  # tokens and offsets whose sequences share no token, but leave some out
    (100, [30, 80]), (5, [3]), (5, [-1]), (300, [1 << 50]), (300, [0, 40, 301]), (300, [17, 17, 170, 171, 999]), (200, [-7, 20, 60, 200]),
    (700, [0, 130, 1 << 40, 140, 400, -1, 400, 640]), (13000, [100 + 129 * i for i in range(101)]),
    (1000, [5 * i for i in range(70)] + [-1] + [400 + 2 * i for i in range(130)]), (600, [1, 1, 1]), (4000, [3000, 3300])]
SHARED = [  # offsets that come back into sequences before them
    (150, [0, 100, 50, 150]), (500, [0, 300, 0, 300, 0, 500]), (500, [200, 300, 100, 400, 350, 500, 400, 480]),
    (1000, [7 * i for i in range(80)] + [300 + 7 * i for i in range(100)]), (400, [0, 400, 399, 400, 0, 1]),
    (900, [10, 500] + [400, 600] * 40 + [0, 880, 890, 890, 0, 10])]


def no_sequence(n, offsets, heads, kv, dim, dtype, causal):
    """Rows in no sequence are zeros in tensors made by the call, whatever memory they get, and left alone in given ones; each sequence
    is as by itself."""
    announce("rows in no sequence", n, offsets[:8], heads, kv, dim, dtype, causal)
    seqs = sequences_of(offsets, n)
    host = attention_case(n, heads, kv, dim, dtype, n)
    rest = torch.ones(n, dtype=torch.bool)
    for a, b in seqs:
        rest[a:b] = False
    for t in host:
        t[rest] = float("nan")
    q, k, v, dout = (t.cuda() for t in host)
    off = torch.tensor(offsets, device="cuda")
    spoiled = [torch.full((n, h, dim), 7.0, dtype=dtype, device="cuda") for h in (heads, heads, kv, kv)] + [torch.full((heads, n), 7.0, device="cuda")]
    del spoiled  # what the allocator hands out next
    out, lse = daso.packed_attention(q, k, v, off, causal)
    grads = daso.packed_attention_backward(dout, q, k, v, out, lse, off, causal)
    gone = rest.cuda()
    assert not out[gone].any() and not lse[:, gone].any() and not any(t[gone].any() for t in grads)
    for a, b in seqs[:3] + seqs[3::29] + seqs[-2:]:
        check_attention(*(t[a:b] for t in host), None, causal, None, out[a:b], lse[:, a:b], [t[a:b] for t in grads], dtype)
        alone, lse_alone = daso.packed_attention(q[a:b], k[a:b], v[a:b], None, causal)
        assert torch.equal(alone, out[a:b]) and torch.equal(lse_alone, lse[:, a:b])
    to, stats = torch.full_like(q, 7), torch.full_like(lse, 7)
    daso.packed_attention(q, k, v, off, causal, out=to, lse=stats)
    given = daso.packed_attention_backward(dout, q, k, v, out, lse, off, causal, dq=torch.full_like(q, 7), dk=torch.full_like(k, 7),
                                           dv=torch.full_like(v, 7))
    assert (to[gone] == 7).all() and (stats[:, gone] == 7).all() and all((t[gone] == 7).all() for t in given)
    assert torch.equal(to[~gone], out[~gone]) and torch.equal(stats[:, ~gone], lse[:, ~gone])
    assert all(torch.equal(t[~gone], g[~gone]) for t, g in zip(given, grads))


@pytest.mark.parametrize("n,offsets", APART)
@pytest.mark.parametrize("heads,kv,dim,dtype,causal", [(8, 8, 16, BF16, True), (3, 1, 72, F32, False)])
def test_rows_between_sequences_are_zeros_in_tensors_made_here(n, offsets, heads, kv, dim, dtype, causal):
    no_sequence(n, offsets, heads, kv, dim, dtype, causal)


@pytest.mark.parametrize("n,offsets", SHARED)
@pytest.mark.parametrize("heads,kv,dim,dtype,causal", [(8, 8, 16, BF16, True), (3, 1, 72, F32, False)])
def test_pairs_that_come_back_into_a_sequence_are_none(n, offsets, heads, kv, dim, dtype, causal):
    no_sequence(n, offsets, heads, kv, dim, dtype, causal)
