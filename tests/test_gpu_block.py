"""The transformer block's operators on the GPU against the 64-bit oracle.

Tolerances follow from the arithmetic.  u = 2^-24 is the rounding of one 32-bit operation, h that of a result to its type:
2^-8 of itself for bf16 and u for fp32.  A sum of k terms in any order is off by at most k u times the sum of their
magnitudes.  Hardware's exp2 and the library's log are off by 2 u of their result, sine and cosine by 4 u absolutely."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2104_05588_amd as daso  # noqa: E402
from oracle import block_oracle as O  # noqa: E402
from tests.test_gpu_train import U, announce, close, gen, np64  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]

BF16, F32 = torch.bfloat16, torch.float32


def half_step(dtype):
    return 2.0 ** -8 if dtype == BF16 else U


def parts(n, widths, dim, dtype, pad=0, shift=0, fill=7.0):
    """[n, heads, dim] tensors beside one another in rows of one wider buffer, as a projection leaves them."""
    width = sum(widths) * dim + pad
    store = torch.full((n * width + shift + 8,), fill, dtype=dtype, device="cuda")
    wide = store[shift:shift + n * width].view(n, width)
    out, at = [], 0
    for w in widths:
        out.append(wide[:, at * dim:(at + w) * dim].unflatten(1, (w, dim)))
        at += w
    return out


# ------------------------------------------------------- norm and rotation
ROTARY = [  # tokens, heads, kv heads, dim, rotated
    (1, 1, 1, 8, 8), (3, 2, 1, 16, 16), (61, 6, 3, 80, 80), (7, 5, 2, 40, 24), (130, 16, 16, 64, 64), (33, 3, 1, 128, 128),
    (5, 1, 1, 128, 0), (9, 40, 8, 32, 32), (4100, 2, 2, 64, 32), (5001, 3, 1, 24, 24), (257, 12, 4, 96, 96), (12, 7, 3, 104, 56)]


def rotary_case(n, heads, kv, dim, rotated, dtype, first, seed):
    g = gen(seed)
    q, k, dq, dk = ((torch.randn(n, h, dim, generator=g) * s).to(dtype) for h, s in ((heads, 2), (kv, 0.5), (heads, 0.1), (kv, 0.1)))
    at = torch.randint(0, 50, (n,), generator=g) + first
    return q, k, dq, dk, at, torch.randn(dim, generator=g), torch.randn(dim, generator=g), daso.rotary_frequencies(rotated, device="cpu")


def check_rotary(x, dy, at, w, freq, inter, y, dx, dw, dtype, eps=1e-6):
    """One of the two, with the bound of each result."""
    dim, rows = x.shape[2], x.shape[0] * x.shape[1]
    xh, wh = np64(x), np.ones(dim) if w is None else np64(w)
    args = (np64(at), np64(freq))
    want = O.head_norm_rotary(xh, *args, wh, eps, inter)
    # the sum of squares is off by dim / 8 + 10 roundings, rstd by half of that and 4 more; a turned element is two products,
    # each with the table's error, the norm's and 4 roundings
    rstd = 1 / np.sqrt((xh * xh).mean(axis=2, keepdims=True) + eps)
    rel = (dim / 16 + 10) * U
    size = np.abs(xh * rstd * wh)
    pairs = O._pair_indexes(2 * len(freq), inter)
    both = size.copy()
    both[..., pairs[0]] = both[..., pairs[1]] = size[..., pairs[0]] + size[..., pairs[1]]
    close(y, want, both * (rel + 10 * U) + np.abs(want) * half_step(dtype) + 1e-37, "y")
    want_dx, want_dw = O.head_norm_rotary_backward(np64(dy), xh, *args, wh, eps, inter)
    d = np.abs(np64(dy))
    turned = d.copy()
    turned[..., pairs[0]] = turned[..., pairs[1]] = d[..., pairs[0]] + d[..., pairs[1]]
    gm, xhat = turned * np.abs(wh), np.abs(xh * rstd)
    mean = (gm * xhat).mean(axis=2, keepdims=True)
    tol = rstd * (gm * (rel + 12 * U) + xhat * mean * (3 * rel + (dim / 8 + 20) * U))
    close(dx, want_dx, tol + np.abs(want_dx) * half_step(dtype) + 1e-37, "dx")
    # a column's sum: at most rows / 64 terms a lane one after the other, then some 40 by trees
    close(dw, want_dw, (turned * xhat).sum(axis=(0, 1)) * (rel + 12 * U + (rows / 64 + 40) * U) + 1e-37, "dweight")


@pytest.mark.parametrize("n,heads,kv,dim,rotated", ROTARY)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("inter,pad,shift,affine,first", [(False, 0, 0, True, 0), (True, 5, 1, True, 1_000_003), (False, 8, 3, False, 77)])
def test_head_norm_rotary(n, heads, kv, dim, rotated, dtype, inter, pad, shift, affine, first):
    announce("head_norm_rotary", n, heads, kv, dim, rotated, dtype, inter, pad, shift, affine, first)
    q, k, dq, dk, at, qw, kw, freq = rotary_case(n, heads, kv, dim, rotated, dtype, first, n + dim)
    if not affine:
        qw = kw = None
    qd, kd, _ = parts(n, (heads, kv, kv), dim, dtype, pad, shift)
    qd.copy_(q), kd.copy_(k)
    args = (at.cuda(), freq.cuda(), None if qw is None else qw.cuda(), None if kw is None else kw.cuda())
    yq, yk = daso.head_norm_rotary(qd, kd, *args, interleaved=inter)
    gq, gk = parts(n, (heads, kv), dim, dtype, pad + 3, shift)
    gq.copy_(dq), gk.copy_(dk)
    dxq, dxk, dqw, dkw = daso.head_norm_rotary_backward(gq, gk, qd, kd, *args, interleaved=inter)
    check_rotary(q, dq, at, qw, freq, inter, yq, dxq, dqw, dtype)
    check_rotary(k, dk, at, kw, freq, inter, yk, dxk, dkw, dtype)


def test_head_norm_rotary_in_place_and_parts():
    announce("head_norm_rotary in place")
    q, k, dq, dk, at, qw, kw, freq = rotary_case(77, 6, 2, 64, 64, BF16, 0, 5)
    args = (at.cuda(), freq.cuda(), qw.cuda(), kw.cuda())
    qd, kd, vd = parts(77, (6, 2, 2), 64, BF16)
    qd.copy_(q), kd.copy_(k)
    yq, yk = daso.head_norm_rotary(qd, kd, *args)
    want = daso.head_norm_rotary_backward(dq.cuda(), dk.cuda(), qd, kd, *args)
    iq, ik, iv = parts(77, (6, 2, 2), 64, BF16)
    iq.copy_(q), ik.copy_(k)
    out = daso.head_norm_rotary(iq, ik, *args, out_q=iq, out_k=ik)
    assert out[0] is iq and torch.equal(iq, yq) and torch.equal(ik, yk) and (iv == 7).all()
    gq, gk, gv = parts(77, (6, 2, 2), 64, BF16)
    gq.copy_(dq), gk.copy_(dk)
    flat = torch.full((300,), 3.0, device="cuda")
    got = daso.head_norm_rotary_backward(gq, gk, qd, kd, *args, dq=gq, dk=gk, dq_weight=flat[5:69], dk_weight=flat[100:164])
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and (gv == 7).all() and (vd == 7).all()
    assert (flat[:5] == 3).all() and (flat[69:100] == 3).all() and (flat[164:] == 3).all()
    # heads as blocks of tokens: [heads, tokens, dim] seen as [tokens, heads, dim]
    hq, hk = q.cuda().transpose(0, 1).contiguous().transpose(0, 1), k.cuda().transpose(0, 1).contiguous().transpose(0, 1)
    again = daso.head_norm_rotary(hq, hk, *args, out_q=torch.empty_like(hq), out_k=torch.empty_like(hk))
    assert torch.equal(again[0], yq) and torch.equal(again[1], yk)


def test_head_norm_rotary_of_nothing_and_of_zeros():
    announce("head_norm_rotary of nothing")
    freq, none = daso.rotary_frequencies(64), torch.empty(0, 2, 64, device="cuda")
    at = torch.empty(0, dtype=torch.int64, device="cuda")
    yq, yk = daso.head_norm_rotary(none, none, at, freq)
    assert yq.shape == (0, 2, 64) == yk.shape
    dq, _, dqw, dkw = daso.head_norm_rotary_backward(none, none, none, none, at, freq)
    assert dq.shape == (0, 2, 64) and not dqw.any() and not dkw.any()
    zero, at = torch.zeros(3, 2, 64, device="cuda"), torch.arange(3, device="cuda")
    assert not daso.head_norm_rotary(zero, zero, at, freq)[0].any()
    dq, _, dqw, _ = daso.head_norm_rotary_backward(zero + 1, zero, zero, zero, at, freq)
    assert torch.isfinite(dq).all() and not dqw.any()


@pytest.mark.parametrize("first", [0, 10 ** 6, 2 ** 31 + 5, 10 ** 9 * 7])
def test_rotation_of_far_positions(first):
    """A turn by the difference of two positions, wherever they are: angles of 64 bits are off by 2^-52 of their turns."""
    announce("far positions", first)
    n, dim = 70, 64
    x = torch.randn(1, 1, dim, generator=gen(1)).expand(n, 1, dim).contiguous()
    at, freq = torch.arange(n) + first, daso.rotary_frequencies(dim, device="cpu")
    y, _ = daso.head_norm_rotary(x.cuda(), x.cuda(), at.cuda(), freq.cuda())
    want = O.head_norm_rotary(np64(x), np64(at), np64(freq))
    # (the oracle's own angle is off by 2^-53 of itself)
    close(y, want, 4.0 * (20 * U + (first + n) * 2.0 ** -51), "y")


# --------------------------------------------------------------- attention
def attention_case(n, heads, kv, dim, dtype, seed, peak=1.0):
    g = gen(seed)
    return [(torch.randn(n, h, dim, generator=g) * s).to(dtype) for h, s in ((heads, peak), (kv, 1), (kv, 1), (heads, 0.1))]


def check_attention(q, k, v, dout, offsets, causal, scale, out, lse, grads, dtype):
    n, heads, dim = q.shape
    share, c = heads // k.shape[1], 1 / np.sqrt(dim) if scale is None else scale
    qh, kh, vh, gh = (np64(t) for t in (q, k, v, dout))
    ends = None if offsets is None else [int(e) for e in offsets]
    want, want_lse, probs = O.attention(qh, kh, vh, ends, causal, scale)
    want_grads = O.attention_backward(gh, qh, kh, vh, ends, causal, scale)
    tol_out, tol_lse = np.zeros_like(want), np.zeros_like(want_lse)
    tol = [np.zeros_like(t) for t in want_grads]
    low = 2.0 ** -8 if dtype == BF16 else 0.0  # of p and ds where they are operands
    h2 = half_step(dtype)
    for (h, s), p in probs.items():
        rows = slice(0, n) if ends is None else slice(ends[s], ends[s + 1])
        of, m = h // share, p.shape[0]
        qq, kk, vv, gg = qh[rows, h], kh[rows, of], vh[rows, of], gh[rows, h]
        # z: dim products, and the roundings of its scaling; the exponent's base is off as the largest z is
        ze = np.where(p > 0, c * (np.abs(qq) @ np.abs(kk).T) * (dim + 8) * U, 0.0)
        ze = ze + 4 * U * np.abs(want_lse[h, rows])[:, None] + 4 * U
        zmax = ze.max(axis=1, keepdims=True)
        pe = ze + zmax  # of p, relative
        tol_lse[h, rows] = zmax[:, 0] + (m + 8) * U + 4 * U * np.abs(want_lse[h, rows])
        fwd = (p * (2 * pe + low + 2 * m * U)) @ np.abs(vv) + 4 * U * np.abs(want[rows, h]) + 1e-37
        tol_out[rows, h] = fwd + np.abs(want[rows, h]) * h2
        # backward: p from the stored lse
        pb = 2 * pe + 8 * U * np.abs(want_lse[h, rows])[:, None] + 8 * U
        tol[2][rows, of] += (p * (pb + low + share * m * U)).T @ np.abs(gg)
        dp, delta = np.abs(gg) @ np.abs(vv).T, (np.abs(gg) * np.abs(want[rows, h])).sum(axis=1, keepdims=True)
        ds = p * np.abs(gg @ vv.T - (gg * want[rows, h]).sum(axis=1, keepdims=True))
        # delta is of the rounded out
        de = (np.abs(gg) * tol_out[rows, h]).sum(axis=1, keepdims=True) + (dim + 4) * U * delta
        dse = ds * (pb + low + share * m * U) + p * (dp * (dim + 4) * U + de + 4 * U * (dp + delta))
        tol[0][rows, h] += c * (dse @ np.abs(kk))
        tol[1][rows, of] += c * (dse.T @ np.abs(qq))
    live = ~np.isnan(want)
    close(out[torch.from_numpy(live)], want[live], tol_out[live], "out")
    live = ~np.isnan(want_lse)
    close(lse[torch.from_numpy(live)], want_lse[live], tol_lse[live], "lse")
    if grads is None:
        return
    for what, got, exact, bound in zip(("dq", "dk", "dv"), grads, want_grads, tol):
        seen = np.ones(len(exact), bool) if ends is None else np.arange(len(exact)) < ends[-1]
        close(got[torch.from_numpy(seen)], exact[seen], (bound + np.abs(exact) * (h2 + 4 * U) + 1e-37)[seen], what)


def both_ways(q, k, v, dout, offsets=None, causal=True, scale=None, pad=0, shift=0, dtype=BF16):
    n, heads, dim = q.shape
    kv = k.shape[1]
    qd, kd, vd = parts(n, (heads, kv, kv), dim, dtype, pad, shift)
    for to, t in ((qd, q), (kd, k), (vd, v)):
        to.copy_(t)
    gd, = parts(n, (heads,), dim, dtype, pad, shift)
    gd.copy_(dout)
    off = None if offsets is None else torch.tensor(offsets, device="cuda")
    out, lse = daso.packed_attention(qd, kd, vd, off, causal, scale)
    dq, dk, dv = parts(n, (heads, kv, kv), dim, dtype, pad, shift)
    grads = daso.packed_attention_backward(gd, qd, kd, vd, out, lse, off, causal, scale, dq=dq, dk=dk, dv=dv)
    return out, lse, grads


ATTENTION = [  # tokens, offsets, heads, kv heads, dim
    (1, None, 1, 1, 8), (2, None, 2, 1, 16), (31, None, 2, 2, 32), (32, None, 1, 1, 64), (33, None, 3, 1, 40), (64, None, 2, 2, 64),
    (65, None, 2, 1, 72), (127, None, 1, 1, 128), (128, None, 8, 2, 64), (129, None, 4, 4, 96), (300, None, 8, 1, 64), (511, None, 2, 1, 128),
    (40, [0, 1, 1, 2, 5, 40], 2, 1, 64), (200, [0, 0, 63, 64, 129, 200, 200], 4, 2, 80), (257, [0, 128, 256, 257], 8, 8, 64),
    (100, [0, 37], 2, 2, 24), (70, [0, 0], 1, 1, 64), (90, list(range(0, 91)), 2, 1, 48), (600, [0, 33, 290, 545, 546, 600], 16, 4, 128)]


@pytest.mark.parametrize("n,offsets,heads,kv,dim", ATTENTION)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal,scale,pad,shift", [(True, None, 0, 0), (False, 0.3, 5, 1)])
def test_attention(n, offsets, heads, kv, dim, dtype, causal, scale, pad, shift):
    announce("attention", n, offsets, heads, kv, dim, dtype, causal, scale, pad, shift)
    q, k, v, dout = attention_case(n, heads, kv, dim, dtype, n + dim)
    out, lse, grads = both_ways(q, k, v, dout, offsets, causal, scale, pad, shift, dtype)
    check_attention(q, k, v, dout, offsets, causal, scale, out, lse, grads, dtype)
    if offsets is not None and offsets[-1] < n:  # rows of no sequence are left as they were
        assert all((t[offsets[-1]:] == 7).all() for t in grads)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim,n", [(64, 200), (128, 150), (80, 300)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_a_token_does_not_see_changes_nothing(dtype, dim, n, bad):
    """What is no number in later tokens, in another sequence and behind the last one: the same bits where they are not
    seen, and none where they are."""
    announce("unseen values", dtype, dim, n, bad)
    q, k, v, dout = attention_case(n, 4, 2, dim, dtype, 11)
    ends, token = [0, 70, n - 20], n - 45
    out, lse, (dq, dk, dv) = both_ways(q, k, v, dout, ends, dtype=dtype)
    before = torch.ones(n, dtype=torch.bool)
    before[token:] = False
    for which in range(4):
        t = [x.clone() for x in (q, k, v, dout)]
        t[which][token, -1, 3] = bad
        t[which][n - 20:] = bad
        out2, lse2, (dq2, dk2, dv2) = both_ways(*t, ends, dtype=dtype)
        same = before.cuda()
        assert torch.equal(out2[same], out[same]) and torch.equal(lse2[:, same], lse[:, same]), which
        assert torch.equal(dq2[same], dq[same]), which
        assert torch.equal(dk2[:70], dk[:70]) and torch.equal(dv2[:70], dv[:70]), which
        after = slice(token + 1, n - 20)  # tokens that see it, or that it does not see
        if which == 0:  # a query alone: its own row, and what it sees
            assert torch.equal(out2[after], out[after]) and torch.equal(dk2[after], dk[after]) and torch.equal(dv2[after], dv[after])
            assert torch.isnan(out2[token, -1]).all()
        elif which == 3:  # its own dq and the keys that it sees
            assert torch.equal(dv2[after], dv[after]) and torch.equal(dk2[after], dk[after]) and torch.equal(dq2[after], dq[after])
            assert not torch.isfinite(dv2[70:token + 1, -1, 3]).any() and not torch.isfinite(dq2[token, -1]).any()
        elif which == 2:
            gone = out2[after, 2:, 3]
            assert not torch.isfinite(gone).any() and not torch.isfinite(dq2[after, 2:]).any()
            rest = [c for c in range(dim) if c != 3]
            assert torch.equal(out2[after][:, :, rest], out[after][:, :, rest])
        else:
            assert not torch.isfinite(lse2[2:, after]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [100, 130])
def test_what_all_tokens_see_reaches_all(dtype, n):
    """Not causal: a value that is no number reaches each token of its sequence, in the last part of a tile too."""
    announce("seen by all", dtype, n)
    for which, token in ((2, n - 1), (3, n - 1), (1, 3), (0, n - 2)):
        t = attention_case(n, 2, 2, 64, dtype, 13)
        t[which][token, 1, 5] = float("nan")
        out, lse, (dq, dk, dv) = both_ways(*t, causal=False, dtype=dtype)
        assert torch.isfinite(out[:, 0]).all() and torch.isfinite(dk[:, 0]).all() and torch.isfinite(dv[:, 0]).all()
        if which == 2:
            assert out[:, 1, 5].isnan().all() and torch.isfinite(out[:, 1, 6]).all() and dq[:, 1].isnan().all()
        elif which == 3:
            assert dv[:, 1, 5].isnan().all() and torch.isfinite(dv[:, 1, 6]).all() and dk[:, 1].isnan().all()
        elif which == 1:
            assert lse[1].isnan().all() and dv[:, 1].isnan().all()
        else:
            assert dk[:, 1].isnan().all() and dv[:, 1].isnan().all() and out[token, 1].isnan().all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("size", [1e-3, 30.0, 1e4])
def test_attention_of_small_and_huge_scores(dtype, size):
    """From weights that are all alike to one that decides: nothing overflows, and p is as exact as its score is."""
    announce("scores", dtype, size)
    n, dim = 150, 64
    q, k, v, dout = attention_case(n, 2, 2, dim, dtype, 3, peak=size)
    k[:, :, 0] -= 4  # scores far below zero, too
    out, lse, grads = both_ways(q, k, v, dout, dtype=dtype)
    assert all(torch.isfinite(t).all() for t in (out, lse, *grads))
    if size < 1e4:
        check_attention(q, k, v, dout, None, True, None, out, lse, grads, dtype)
    else:  # the rows where one key decides by far
        z = np.einsum("ihd,jhd->hij", np64(q), np64(k)) / 8
        z[:, np.triu(np.ones((n, n), bool), 1)] = -np.inf
        two = np.sort(z, axis=2)[:, 1:, -2:]
        sure = two[:, :, 1] - two[:, :, 0] > 100
        assert sure.mean() > 0.8
        want = np.stack([np64(v)[z[h].argmax(axis=1)[1:], h] for h in range(2)])
        off = np.abs(np64(out).transpose(1, 0, 2)[:, 1:] - want)
        assert (off <= np.abs(want) * 2.0 ** -7)[sure].all()


def test_keys_of_minus_infinity_weigh_nothing():
    announce("keys of minus infinity")
    n, dim = 100, 64
    q, k, v, dout = (t.abs() + 0.1 for t in attention_case(n, 1, 1, dim, F32, 4))
    k[5:40] = -float("inf")
    out, lse, _ = both_ways(q, k, v, dout, dtype=F32)
    keep = [i for i in range(n) if not 5 <= i < 40]
    want, want_lse, _ = O.attention(np64(q)[keep], np64(k)[keep], np64(v)[keep])
    close(out[keep], want, np.abs(want) * 1e-5, "out")
    close(lse[:, keep], want_lse, np.abs(want_lse) * 1e-5 + 1e-5, "lse")


def test_attention_of_odd_offsets_reads_and_writes_nothing_outside():
    """Pairs of offsets that fall or pass the last token are empty sequences."""
    announce("odd offsets")
    n = 100
    q, k, v, dout = attention_case(n, 2, 1, 64, BF16, 8)
    out, lse, grads = both_ways(q, k, v, dout, [0, 40, 90])
    odd = torch.tensor([-5, 0, 40, 90, 101, 1 << 40, -(1 << 40), 3, 2], device="cuda")
    to = torch.full_like(out, 7)
    stats = torch.full_like(lse, 7)
    qd, kd, vd = q.cuda(), k.cuda(), v.cuda()
    daso.packed_attention(qd, kd, vd, odd, out=to, lse=stats)
    assert torch.equal(to[:90], out[:90]) and (to[90:] == 7).all() and torch.equal(stats[:, :90], lse[:, :90]) and (stats[:, 90:] == 7).all()
    got = daso.packed_attention_backward(dout.cuda(), qd, kd, vd, to, stats, odd, dq=torch.full_like(qd, 7), dk=torch.full_like(kd, 7),
                                         dv=torch.full_like(vd, 7))
    for a, b in zip(got, grads):
        assert torch.equal(a[:90], b[:90]) and (a[90:] == 7).all()


@pytest.mark.parametrize("n,offsets", [(100, [0, 37]), (300, [0, 130, 131]), (5, [0]), (700, [0, 0])])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_behind_the_last_sequence_are_zeros_in_tensors_made_here(n, offsets, dtype):
    announce("rest", n, offsets, dtype)
    q, k, v, dout = (t.cuda() for t in attention_case(n, 4, 2, 72, dtype, 12))
    off, end = torch.tensor(offsets, device="cuda"), offsets[-1]
    q[end:], k[end:], v[end:], dout[end:] = (float("nan"),) * 4
    torch.full((n * 4 * 72 * 4,), 7.0, device="cuda")  # what the allocator may hand out again
    out, lse = daso.packed_attention(q, k, v, off)
    grads = daso.packed_attention_backward(dout, q, k, v, out, lse, off)
    assert not out[end:].any() and not lse[:, end:].any() and not any(t[end:].any() for t in grads)
    assert all(torch.isfinite(t).all() for t in (out, lse, *grads))


def test_attention_of_many_sequences_and_other_layouts():
    announce("many sequences")
    g = gen(9)
    lengths = torch.randint(0, 9, (700,), generator=g)
    lengths[350] = 260
    ends = [0] + lengths.cumsum(0).tolist()
    n = ends[-1]
    q, k, v, dout = attention_case(n, 2, 2, 32, BF16, 10)
    out, lse, grads = both_ways(q, k, v, dout, ends)
    check_attention(q, k, v, dout, ends, True, None, out, lse, grads, BF16)
    heads_first = [t.cuda().transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v, dout)]
    off = torch.tensor(ends, device="cuda")
    to = torch.empty_like(heads_first[0])
    again, lse2 = daso.packed_attention(*heads_first[:3], off, out=to)
    assert again is to and torch.equal(again, out) and torch.equal(lse2, lse)
    # heads interleaved as [tokens, heads, (q, k, v), dim], and their gradients likewise
    joint, grad = (torch.empty(n, 2, 3, 32, dtype=BF16, device="cuda") for _ in range(2))
    for i, t in enumerate((q, k, v)):
        joint[:, :, i] = t.cuda()
    out3, lse3 = daso.packed_attention(joint[:, :, 0], joint[:, :, 1], joint[:, :, 2], off)
    got = daso.packed_attention_backward(dout.cuda(), joint[:, :, 0], joint[:, :, 1], joint[:, :, 2], out3, lse3, off, dq=grad[:, :, 0],
                                         dk=grad[:, :, 1], dv=grad[:, :, 2])
    assert torch.equal(out3, out) and all(torch.equal(a, b) for a, b in zip(got, grads))


@pytest.mark.parametrize("ends", [[0, 100, 40000, 40001, 40100], [0, 3000, 3000, 17000, 41000], [0] + [1000 * (i + 1) for i in range(40)]])
def test_long_sequences_of_one_head_are_each_by_itself(ends):
    """More tiles of a sequence than the order of their work is kept for, more sequences, and few of them: the same bits as by themselves."""
    announce("long sequences", ends)
    n, dim = ends[-1], 16
    q, k, v, dout = (t.cuda() for t in attention_case(n, 1, 1, dim, BF16, 5))
    off = torch.tensor(ends, device="cuda")
    out, lse = daso.packed_attention(q, k, v, off)
    grads = daso.packed_attention_backward(dout, q, k, v, out, lse, off)
    for a, b in zip(ends, ends[1:]):
        o, l = daso.packed_attention(q[a:b], k[a:b], v[a:b])
        assert torch.equal(o, out[a:b]) and torch.equal(l, lse[:, a:b]), (a, b)
        for got, one in zip(grads, daso.packed_attention_backward(dout[a:b], q[a:b], k[a:b], v[a:b], o, l)):
            assert torch.equal(one, got[a:b]), (a, b)


@pytest.mark.parametrize("dim", [32, 64, 96, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_attention_gradients_of_bf16_are_off_by_their_own_roundings(dim, causal):
    """A rounding to bf16 is off by at most 2^-8 of a value in [1, 2) times its power of two, evenly: by 2^-8 / sqrt(3) times
    sqrt(E m^-2) = 0.74 of the norm, where the logarithm of m is spread evenly; that is 0.00166.  dq and dk have two of them, of ds
    and their own (0.0024), dv of p and its own, out the same; a tenth more for the sample.  A delta of the rounded out, which is a
    third one of dq and dk, makes 0.0031 and is not allowed here."""
    n, heads = 512, 2
    q, k, v, dout = attention_case(n, heads, heads, dim, BF16, 77 + dim)
    out, lse, grads = both_ways(q, k, v, dout, None, causal)
    qh, kh, vh, gh = (np64(t) for t in (q, k, v, dout))
    c = 1 / np.sqrt(dim)
    want = [O.attention(qh, kh, vh, None, causal, c)[0], *O.attention_backward(gh, qh, kh, vh, None, causal, c)]
    for what, got, exact in zip(("out", "dq", "dk", "dv"), (out, *grads), want):
        off = np.linalg.norm(np64(got.cpu()) - exact) / np.linalg.norm(exact)
        assert off < 1.1 * np.sqrt(2) * 0.00166, (what, off)


def test_attention_gradients_against_differences():
    """fp32, along random directions: (f(x + e d) - f(x - e d)) / 2e is off by e^2 f''' and rounding / e."""
    announce("differences")
    n, dim, ends = 70, 32, [0, 25, 70]
    q, k, v, dout = attention_case(n, 2, 1, dim, F32, 21)
    _, _, grads = both_ways(q, k, v, dout, ends, dtype=F32)
    e = 2.0 ** -12
    for which, grad in enumerate(grads):
        d = torch.randn((q, k, v)[which].shape, generator=gen(which))
        value = []
        for sign in (1, -1):
            t = [q, k, v]
            t[which] = t[which] + sign * e * d
            out, _, _ = O.attention(*(np64(x) for x in t), ends)
            value.append((out * np64(dout)).sum())
        want = (value[0] - value[1]) / (2 * e)
        terms = np.abs(np64(grad) * np64(d))
        # the kernel's own error is some hundreds of roundings of its terms; a third derivative is below |d|^3 of the logits' size, 100
        assert abs((np64(grad) * np64(d)).sum() - want) <= terms.sum() * 500 * U + e * e * 100 * np.abs(np64(dout)).sum()


# ---------------------------------------------------------------- clipping
CLIPS = [  # n, tensors, g
    (1, [(0, 1)], 1), (3, [(0, 3)], 2), (7, [(1, 3), (5, 1)], 3), (4096, None, 4), (4097, [(0, 4097)], 8), (65536, None, 4),
    (70001, [(0, 5), (5, 0), (6, 2), (9, 60000), (60010, 9990)], 5), (300_000, [(i * 1000 + i % 3, 990 - i) for i in range(300)], 2),
    (5_000_003, [(3, 4_999_999)], 1), (9000, [(0, 4100), (4101, 1), (4103, 4500)], 64), (2000, [(i, 1) for i in range(0, 2000, 2)], 7)]


@pytest.mark.parametrize("n,tensors,g", CLIPS)
@pytest.mark.parametrize("size,part", [(1e-3, 0.5), (1e30, 0.01), (1e-30, 0.3), (1.0, 3.0)])
def test_clip_gradients(n, tensors, g, size, part):
    announce("clip", n, None if tensors is None else len(tensors), g, size, part)
    gn = gen(n + g)
    grads = [torch.randn(n, generator=gn) * size for _ in range(g)]
    spans = [(0, n)] if tensors is None else tensors
    most = part * float(O.clip_gradients([np64(x) for x in grads], 1.0, spans)[1])
    most = float(np.float32(most))
    eps = 1e-6 * most
    want, want_norm, want_norms = O.clip_gradients([np64(x) for x in grads], most, spans, float(np.float32(eps)))
    dev = [x.cuda() for x in grads]
    out = torch.full((n,), 7.0, device="cuda")
    norm, norms = daso.clip_gradients(dev, most, tensors, out=out, eps=eps)
    # the mean of g terms: g roundings of their magnitudes; norms as exact as that (in the root of the squares' sum), and one more
    mags = np.mean([np.abs(np64(x)) for x in grads], axis=0) * g * U
    off = np.array([np.sqrt((mags[a:a + k] ** 2).sum()) for a, k in spans])
    close(norms, want_norms, off + 2 * U * want_norms + 2.0 ** -149, "norms")
    close(norm, np.array(want_norm), np.sqrt((off ** 2).sum()) + 2 * U * want_norm + 2.0 ** -149, "norm")
    inside = np.zeros(n, bool)
    for a, k in spans:
        inside[a:a + k] = True
    factor = 1 if part > 1 else part
    tol = (mags + np.abs(want) / factor * (np.sqrt((off ** 2).sum()) / max(want_norm, 1e-300) + 4 * U)) * factor + 2.0 ** -149
    close(out[torch.from_numpy(inside)], want[inside], tol[inside], "out")
    assert (np64(out)[~inside] == 7).all()
    same_norm, same_norms = daso.gradient_norm(dev, tensors)
    assert torch.equal(same_norm, norm) and torch.equal(same_norms, norms)
    # in place, over the first replica and the last
    for at in {0, g - 1}:
        copies = [x.clone() for x in dev]
        again, _ = daso.clip_gradients(copies, most, tensors, out=copies[at], eps=eps)
        assert torch.equal(again, norm) and torch.equal(copies[at].cpu()[torch.from_numpy(inside)], out.cpu()[torch.from_numpy(inside)])
        assert torch.equal(copies[at].cpu()[torch.from_numpy(~inside)], grads[at][torch.from_numpy(~inside)])


@pytest.mark.parametrize("g", [1, 2, 3, 4, 8, 11])
def test_clipping_nothing_gives_the_averages_bits(g):
    """Where the norm is small, out is the mean as local_avg has it."""
    announce("clip nothing", g)
    dev = [torch.randn(100_003, generator=gen(i)).cuda() for i in range(g)]
    want, out = torch.empty_like(dev[0]), torch.empty_like(dev[0])
    daso.local_avg(dev, want)
    daso.clip_gradients(dev, 1e9, out=out)
    assert torch.equal(out, want)
    daso.clip_gradients(dev, 1e9)
    assert torch.equal(dev[0], want)


def test_clipping_of_what_is_no_number():
    announce("clip nan")
    for bad in (float("nan"), float("inf")):
        x = torch.ones(10_000, device="cuda")
        x[777] = bad
        out = torch.empty_like(x)
        norm, norms = daso.clip_gradients([x], 1.0, [(0, 700), (700, 100), (5000, 10)], out=out)
        want = torch.tensor([700.0, bad * bad, 10.0]).sqrt()
        assert torch.equal(norm.isnan().cpu(), torch.tensor(bad != bad)) and torch.allclose(norms.cpu(), want, equal_nan=True)
        assert out[:777].isnan().all() if bad != bad else not out[:777].any()
        assert out[777].isnan()
    norm, norms = daso.clip_gradients([torch.ones(8, device="cuda")], 0.0, [], out=torch.empty(8, device="cuda"))
    assert float(norm) == 0 and norms.numel() == 0
    norm, norms = daso.gradient_norm([torch.empty(0, device="cuda")])
    assert float(norm) == 0 and float(norms) == 0


# ------------------------------------------------ streams, graphs, all together
def block_step(q, k, v, dy, at, freq, qw, kw, off, flat, clipped):
    """What a training step does with them, the norms' weight gradients in a flat buffer that is then clipped."""
    dim = q.shape[2]
    yq, yk = daso.head_norm_rotary(q, k, at, freq, qw, kw)
    out, lse = daso.packed_attention(yq, yk, v, off)
    dq, dk, dv = daso.packed_attention_backward(dy, yq, yk, v, out, lse, off)
    dxq, dxk, _, _ = daso.head_norm_rotary_backward(dq, dk, q, k, at, freq, qw, kw, dq=dq, dk=dk, dq_weight=flat[:dim],
                                                    dk_weight=flat[dim:2 * dim])
    norm, norms = daso.clip_gradients([flat], 0.01, [(0, dim), (dim, dim)], out=clipped)
    return out, lse, dxq, dxk, dv, norm, norms, clipped


def step_inputs(seed, n=300, dim=64):
    q, k, v, dy = (t.cuda() for t in attention_case(n, 4, 2, dim, BF16, seed))
    g = gen(seed + 1)
    return [q, k, v, dy, torch.arange(n).cuda(), daso.rotary_frequencies(dim), torch.randn(dim, generator=g).cuda(),
            torch.randn(dim, generator=g).cuda(), torch.tensor([0, 120, 121, n], device="cuda")]


def test_a_block_step_captured_and_replayed():
    """Replays between eager work, on inputs and offsets that change: the eager call's bits."""
    announce("capture")
    flat, clipped = torch.zeros(128, device="cuda"), torch.zeros(128, device="cuda")
    inputs = step_inputs(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block_step(*inputs, flat, clipped)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = block_step(*inputs, flat, clipped)
    torch.cuda.current_stream().wait_stream(side)
    for seed in (2, 3, 2):
        new = step_inputs(seed)
        new[8] = torch.tensor([0, 50 * seed, 200, 290], device="cuda")
        want = [t.clone() for t in block_step(*new, torch.zeros(128, device="cuda"), torch.zeros(128, device="cuda"))]
        for t, s in zip(inputs, new):
            t.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), seed


def test_calls_on_two_streams_at_once():
    announce("two streams")
    streams = [torch.cuda.Stream() for _ in range(2)]
    inputs = [step_inputs(s) for s in (5, 6)]
    want = [[t.clone() for t in block_step(*i, torch.zeros(128, device="cuda"), torch.zeros(128, device="cuda"))] for i in inputs]
    spare = [(torch.zeros(128, device="cuda"), torch.zeros(128, device="cuda")) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for s, i, sp in zip(streams, inputs, spare):
            with torch.cuda.stream(s):
                got.append(block_step(*i, *sp))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))


def test_heads_in_a_far_part_of_a_long_buffer():
    """Rows whose distance from the first passes 32 bits, in elements and in bytes."""
    announce("far rows")
    n, dim, apart = 2100, 64, 2 << 20
    store = torch.empty(n * apart, dtype=BF16, device="cuda")
    far = [store[i * 128:].as_strided((n, 2, dim), (apart, dim, 1)) for i in range(3)]
    q, k, v, dout = attention_case(n, 2, 2, dim, BF16, 31)
    for to, t in zip(far, (q, k, v)):
        to.copy_(t)
    out, lse = daso.packed_attention(*far)
    grads = daso.packed_attention_backward(dout.cuda(), *far, out, lse)
    check_attention(q, k, v, dout, None, True, None, out, lse, grads, BF16)
    at, freq = torch.arange(n, device="cuda"), daso.rotary_frequencies(dim)
    a, _ = daso.head_norm_rotary(far[0], far[1], at, freq)
    b, _ = daso.head_norm_rotary(q.cuda(), k.cuda(), at, freq)
    assert torch.equal(a, b)
