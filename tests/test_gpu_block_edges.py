"""The transformer block's operators on the GPU at the ends of what their documentation allows, and on the ways that large
launches take, against the 64-bit oracle.

Tolerances are those of test_gpu_block.py, from the same arithmetic."""
import pytest

torch = pytest.importorskip("torch")

import paper_2104_05588_amd as daso  # noqa: E402
from tests.test_gpu_block import (BF16, F32, attention_case, both_ways, check_attention, check_rotary, rotary_case,  # noqa: E402
                                  test_clip_gradients as check_clip)
from tests.test_gpu_train import announce, gen  # noqa: E402

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


@pytest.mark.parametrize("n,heads,kv,dim,dtype,inter", [(9001, 2, 1, 64, BF16, False), (17000, 1, 1, 8, F32, True), (3001, 100, 30, 16, BF16, False),
                                                        (8500, 9, 9, 24, F32, False)])
def test_head_norm_rotary_of_more_tokens_than_wavefronts(n, heads, kv, dim, dtype, inter):
    """More tokens, or shares of their heads, than a launch has wavefronts: each takes several."""
    announce("rotary of many tokens", n, heads, kv, dim, dtype, inter)
    q, k, dq, dk, at, qw, kw, freq = rotary_case(n, heads, kv, dim, dim, dtype, 5, 3)
    args = (at.cuda(), freq.cuda(), qw.cuda(), kw.cuda())
    yq, yk = daso.head_norm_rotary(q.cuda(), k.cuda(), *args, interleaved=inter)
    dxq, dxk, dqw, dkw = daso.head_norm_rotary_backward(dq.cuda(), dk.cuda(), q.cuda(), k.cuda(), *args, interleaved=inter)
    check_rotary(q, dq, at, qw, freq, inter, yq, dxq, dqw, dtype)
    check_rotary(k, dk, at, kw, freq, inter, yk, dxk, dkw, dtype)


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


def ends_of(lengths):
    ends = [0]
    for k in lengths:
        ends.append(ends[-1] + k)
    return ends


# Launches by keys of 512 workgroups and more without parts, or with fewer parts than query heads: a workgroup walks over several
# heads.  (What a launch counts on: tokens / 128 + sequences + 1 tiles of each key head.)
@pytest.mark.parametrize("heads,kv,lengths,dim,parts", [
    (32, 8, [1 + i * 7 % 13 for i in range(68)] + [131, 260], 64, 1), (32, 8, [3 + i % 5 for i in range(38)] + [200, 1, 290], 80, 2),
    (48, 8, [129, 0, 40, 64, 65, 1, 2, 33] * 2 + [31, 5, 17], 128, 3), (24, 12, [1, 3] * 20 + [150], 16, 1)])
@pytest.mark.parametrize("dtype,causal", [(BF16, True), (BF16, False), (F32, True), (F32, False)])
def test_keys_of_several_query_heads_in_a_workgroup(heads, kv, lengths, dim, parts, dtype, causal):
    announce("several query heads", heads, kv, len(lengths), dim, parts, dtype, causal)
    ends, share = ends_of(lengths), heads // kv
    n = ends[-1]
    tiles, found = (n // 128 + len(lengths) + 1) * kv, 1
    while found < share and (share % found or tiles * found < 512):
        found += 1
    assert found == parts < share
    q, k, v, dout = attention_case(n, heads, kv, dim, dtype, dim)
    out, lse, grads = both_ways(q, k, v, dout, ends, causal, dtype=dtype)
    check_attention(q, k, v, dout, ends, causal, None, out, lse, grads, dtype)


# More than 2048 tiles of all heads, which are not taken in the order of their work: with and without offsets, heads by eights and not
@pytest.mark.parametrize("heads,ends", [(32, None), (33, None), (16, ends_of([1 + i * 5 % 17 for i in range(160)])), (40, [0, 4000, 4001, 7100]),
                                        (20, [0, 130, 9000, 13300]), (8, ends_of([40 * (i % 9) for i in range(300)]))])
@pytest.mark.parametrize("causal", [True, False])
def test_attention_of_launches_of_many_tiles(heads, ends, causal):
    announce("many tiles", heads, None if ends is None else len(ends), causal)
    n, dim = 8300 if ends is None else ends[-1], 16
    assert (n // 128 + (1 if ends is None else len(ends))) * heads > 2048
    host = attention_case(n, heads, heads, dim, BF16, heads)
    q, k, v, dout = (t.cuda() for t in host)
    off = None if ends is None else torch.tensor(ends, device="cuda")
    out, lse = daso.packed_attention(q, k, v, off, causal)
    grads = daso.packed_attention_backward(dout, q, k, v, out, lse, off, causal)
    # one head at a time, or a sequence at a time: the same bits
    seqs = [(0, n)] if ends is None else [p for p in zip(ends, ends[1:]) if p[0] < p[1]]
    assert not out.isnan().any() and len(seqs) >= 1
    for h in range(heads):
        h = slice(h, h + 1)
        alone, lse_alone = daso.packed_attention(q[:, h], k[:, h], v[:, h], off, causal)
        assert torch.equal(alone, out[:, h]) and torch.equal(lse_alone, lse[h])
        for got, one in zip(grads, daso.packed_attention_backward(dout[:, h], q[:, h], k[:, h], v[:, h], alone, lse_alone, off, causal)):
            assert torch.equal(one, got[:, h])
    for a, b in seqs[:2] + seqs[2:-1:37] + seqs[-1:]:
        alone, lse_alone = daso.packed_attention(q[a:b], k[a:b], v[a:b], None, causal)
        assert torch.equal(alone, out[a:b]) and torch.equal(lse_alone, lse[:, a:b])
        for got, one in zip(grads, daso.packed_attention_backward(dout[a:b], q[a:b], k[a:b], v[a:b], alone, lse_alone, None, causal)):
            assert torch.equal(one, got[a:b])
    # and the last head of a short one against the oracle
    a, b = min(seqs, key=lambda p: abs(p[1] - p[0] - 1000))
    if b - a <= 4000:
        check_attention(*(t[a:b, -1:] for t in host), None, causal, None, out[a:b, -1:], lse[-1:, a:b], [t[a:b, -1:] for t in grads], BF16)


@pytest.mark.parametrize("dtype,dim", [(BF16, 64), (BF16, 128), (F32, 32)])
def test_attention_of_a_long_sequence(dtype, dim):
    """Keys far behind, which a running maximum and sum go through, against the oracle."""
    announce("long sequence", dtype, dim)
    q, k, v, dout = attention_case(4133, 1, 1, dim, dtype, 41)
    out, lse, grads = both_ways(q, k, v, dout, dtype=dtype)
    check_attention(q, k, v, dout, None, True, None, out, lse, grads, dtype)


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


# ---------------------------------------------------------------- clipping
def tensors_of(n, count, seed):
    """Tensors of all lengths from none, some behind a gap, which begin anywhere."""
    cuts = (torch.rand(count - 1, generator=gen(seed)) ** 3 * n).long().sort().values.tolist()
    cuts[5:9] = cuts[5:6] * len(cuts[5:9])  # of no elements
    out = []
    for i, (a, b) in enumerate(zip([0] + cuts, cuts + [n])):
        a += min(b - a, (0, 1, 777)[i % 3] if i % 2 else 0)
        out.append((a, b - a))
    return out


# More than 4096 pieces of 1024 elements, whose sums kernels of their own add, of more tensors than a launch's table holds
@pytest.mark.parametrize("n,count,g", [(5_000_011, 300, 1), (5_000_011, 300, 4), (4_400_000, 650, 5), (4_300_000, 2, 2), (4_480_000, 70_000, 2),
                                       (4_194_304, 1, 1), (4_194_305, 209, 8)])
@pytest.mark.parametrize("size,part", [(1.0, 0.25), (1e-3, 2.0)])
def test_clipping_of_many_tensors_of_many_pieces(n, count, g, size, part):
    spans = [(64 * i, 64) for i in range(count)] if count == 70_000 else [(0, n)] if count == 1 else tensors_of(n, count, g)
    check_clip(n, spans, g, size, part)
