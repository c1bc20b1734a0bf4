"""Calls of the training operators at the edges of what they take: in place at every length, operands of any size,
whatever lies in ignored places.  Tolerances as derived in test_gpu_train."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2104_05588_amd as daso  # noqa: E402
from oracle import train_oracle as O  # noqa: E402
from tests.test_gpu_train import U, announce, check_loss, close, gen, loss_case, np64  # noqa: E402

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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("size", [1e3, 1e5, 1e6, 1e9])
def test_loss_of_huge_logits(dtype, size):
    """Logits up to 1e18: of each token the largest one decides, and nothing overflows."""
    announce("loss of huge logits", dtype, size)
    n, v, d = 130, 300, 96
    h, w, t, s = loss_case(n, v, d, dtype, 0.1, 47)
    h, w = (h.double() * size).to(dtype), (w.double() * size).to(dtype)
    hd, wd, td = h.cuda(), w.cuda(), t.cuda()
    loss, lse = daso.linear_cross_entropy(hd, wd, td)
    h64, w64, s64 = np64(h), np64(w), np.where(t.numpy() == -100, 0, np64(s))
    want_loss, want_lse = O.linear_cross_entropy(h64, w64, t.numpy())
    mag = (np.abs(h64) @ np.abs(w64).T).max(axis=1)
    tol = 2 * (d * U + 2.0 ** -20) * mag + 8 * U * (np.abs(want_lse) + mag)
    close(lse, want_lse, tol, "lse")
    close(loss, want_loss, tol, "loss")
    # p may be anything where two logits are nearer to each other than they are off; else it is zero or one
    dh, dw = daso.linear_cross_entropy_backward(s.cuda(), hd, wd, td, lse, dweight=torch.empty(v, d, device="cuda"))
    a = np.abs(s64)[:, None]
    assert torch.isfinite(dh).all() and torch.isfinite(dw).all()
    assert (np.abs(np64(dh)) <= (a * 2.01) * np.abs(w64).sum(axis=0)).all()
    z = h64 @ w64.T
    two = np.sort(z, axis=1)[:, -2:]
    sure = two[:, 1] - two[:, 0] > 2 * tol + 100
    assert sure.sum() > n // 4
    want_dh, _, _ = O.linear_cross_entropy_backward(s64, h64, w64, t.numpy())
    # where one class is sure its p is off by what the logit and the log-sum-exp are, of which 1e5 is all of it; the others' are zero
    off = np.abs(np64(dh) - want_dh)
    plane = np.abs(want_dh) * 2.0 ** -8 + a * np.abs(w64).max() * (2.0 ** -10 + v * 2.0 ** -37)
    assert (off <= a * np.abs(w64[z.argmax(axis=1)]) * 1.01 + plane)[sure].all()


@pytest.mark.parametrize("dtype,grad", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)])
@pytest.mark.parametrize("h_junk,s_junk", [(1e20, 1e9), (1.0, 3e38), (1e30, 0.0), (1e-30, 1e-30)])
@pytest.mark.parametrize("n,v,d", [(150, 300, 96), (70, 129, 65)])
def test_what_lies_in_ignored_rows_changes_nothing(dtype, grad, h_junk, s_junk, n, v, d):
    """hidden and dloss of ignored tokens may hold any value: the same bits for all others."""
    announce("ignored rows", dtype, grad, h_junk, s_junk, n, v, d)
    h, w, t, s = loss_case(n, v, d, dtype, 0.3, n + v)
    s *= 1e-4
    gone = t == -100
    h[gone], s[gone] = 0, 0
    loss, lse, dh, dw = check_loss(h, w, t, s, h.cuda(), w.cuda(), grad)
    h2, s2 = h.clone(), s.clone()
    h2[gone] = (torch.randn(int(gone.sum()), d, generator=gen(1)) * h_junk).to(dtype)
    s2[gone] = s_junk
    td, wd = t.cuda(), w.cuda()
    loss2, lse2 = daso.linear_cross_entropy(h2.cuda(), wd, td)
    dh2, dw2 = daso.linear_cross_entropy_backward(s2.cuda(), h2.cuda(), wd, td, lse2, dweight=torch.empty(v, d, dtype=grad, device="cuda"))
    live = ~gone.cuda()
    assert torch.equal(lse2[live], lse[live]) and torch.equal(loss2, loss)
    _, want = O.linear_cross_entropy(np64(h2), np64(w), t.numpy())
    mag = (np.abs(np64(h2)) @ np.abs(np64(w)).T).max(axis=1)
    close(lse2, want, (d * U + 2.0 ** -20) * 2 * mag + 2.0 ** -19 + 8 * U * np.abs(want), "lse")
    assert torch.equal(dh2, dh) and not dh2[~live].any() and torch.equal(dw2, dw)


@pytest.mark.parametrize("dtype,grad", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)])
@pytest.mark.parametrize("low,high", [(-60, 0), (-100, -40), (0, 60)])
def test_gradients_of_tokens_of_any_weight(dtype, grad, low, high):
    """dloss over many binades: each token's dhidden has its own bits, and dweight those of its largest terms."""
    announce("dloss over binades", dtype, grad, low, high)
    n, v, d = 130, 300, 96
    h, w, t, _ = loss_case(n, v, d, dtype, 0.1, 41)
    s = torch.exp2(torch.linspace(low, high, n, dtype=torch.float64)).float() * (torch.rand(n, generator=gen(2)) + 1)
    s[::3] *= -1
    hd, wd, td, sd = h.cuda(), w.cuda(), t.cuda(), s.cuda()
    _, lse = daso.linear_cross_entropy(hd, wd, td)
    dh, dw = daso.linear_cross_entropy_backward(sd, hd, wd, td, lse, dweight=torch.empty(v, d, dtype=grad, device="cuda"))
    h64, w64, s64 = np64(h), np64(w), np.where(t.numpy() == -100, 0, np64(s))
    want_dh, want_dw, dz = O.linear_cross_entropy_backward(s64, h64, w64, t.numpy())
    # p is off by its logit's and the log-sum-exp's error, 2^-14 with room; dz by its planes, or by 2^-38 of its token's dloss
    a, bf16 = np.abs(s64)[:, None], dtype == torch.bfloat16
    p = np.abs(dz) + (np.arange(v)[None] == t.numpy()[:, None]) * a
    ze = (d * U + 2.0 ** -20) * (np.abs(h64) @ np.abs(w64).T).max(axis=1) + 2.0 ** -16
    off = (2.0 ** -11 if bf16 else 2.0 ** -20) * np.abs(dz) + p * 2 * ze[:, None] + 2.0 ** -37 * a
    close(dh, want_dh, off @ np.abs(w64) + v * U * (np.abs(dz) @ np.abs(w64)) + np.abs(want_dh) * (2.0 ** -8 if bf16 else U), "dhidden")
    # a term of dweight is also off by 2^-37 of the largest dloss_i * hidden_i
    narrow = grad == torch.bfloat16
    off = (2.0 ** -11 if narrow else 2.0 ** -19) * np.abs(dz) + p * 2 * ze[:, None] + 2.0 ** -37 * a
    most = (a * np.abs(h64).max(axis=1, keepdims=True)).max()
    share = (np.abs(dz) / np.maximum(a, 1e-300)).T.sum(axis=1, keepdims=True)
    tol = off.T @ np.abs(h64) + n * U * (np.abs(dz).T @ np.abs(h64)) + 2.0 ** -37 * most * share
    close(dw, want_dw, tol + np.abs(want_dw) * (2.0 ** -8 if narrow else U), "dweight")


@pytest.mark.parametrize("big", [1e6, 1e12, 1e18])
def test_loss_of_tokens_of_any_size(big):
    """fp32 rows of hidden from tiny to huge side by side: each token's loss and dhidden are its own."""
    announce("hidden over binades", big)
    n, v, d = 130, 300, 96
    h, w, t, s = loss_case(n, v, d, torch.float32, 0.1, 43)
    size = torch.ones(n)
    size[::5], size[1::5] = big, 1.0 / big
    h = h * size[:, None]
    hd, wd, td = h.cuda(), w.cuda(), t.cuda()
    loss, lse = daso.linear_cross_entropy(hd, wd, td)
    dh, _ = daso.linear_cross_entropy_backward(s.cuda(), hd, wd, td, lse)
    h64, w64, s64 = np64(h), np64(w), np.where(t.numpy() == -100, 0, np64(s))
    want_loss, want_lse = O.linear_cross_entropy(h64, w64, t.numpy())
    mag = (np.abs(h64) @ np.abs(w64).T).max(axis=1)
    ze = (d * U + 2.0 ** -20) * mag
    tol = 2 * ze + 2.0 ** -20 + 8 * U * (np.abs(want_lse) + mag)
    close(lse, want_lse, tol, "lse")
    close(loss, want_loss, tol, "loss")
    want_dh, _, dz = O.linear_cross_entropy_backward(s64, h64, w64, t.numpy())
    # (of a huge token p is one or zero where the logits lie further apart than they are off, and anything between them else)
    a = np.abs(s64)[:, None]
    p = np.abs(dz) + (np.arange(v)[None] == t.numpy()[:, None]) * a
    off = np.where((size > 1).numpy()[:, None], a, p * np.minimum(2 * (ze + tol), 1)[:, None]) + 2.0 ** -19 * np.abs(dz) + 2.0 ** -37 * a
    close(dh, want_dh, off @ np.abs(w64) + np.abs(want_dh) * U, "dhidden")


@pytest.mark.parametrize("dtype,grad", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)])
@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -float("inf")])
def test_ignored_rows_without_numbers(dtype, grad, junk):
    """NaN and infinities in hidden and dloss of ignored tokens reach no gradient."""
    announce("ignored rows without numbers", dtype, grad, junk)
    h, w, t, s = loss_case(150, 300, 96, dtype, 0.3, 51)
    gone = t == -100
    h[gone], s[gone] = 0, 0
    _, _, dh, dw = check_loss(h, w, t, s, h.cuda(), w.cuda(), grad)
    h[gone, 5:9], s[gone] = junk, junk
    loss, lse = daso.linear_cross_entropy(h.cuda(), w.cuda(), t.cuda())
    assert torch.isfinite(loss).all()
    dh2, dw2 = daso.linear_cross_entropy_backward(s.cuda(), h.cuda(), w.cuda(), t.cuda(), lse,
                                                  dweight=torch.empty(300, 96, dtype=grad, device="cuda"))
    assert torch.equal(dh2, dh) and torch.equal(dw2, dw)


@pytest.mark.parametrize("dtype,grad", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)])
@pytest.mark.parametrize("junk", [float("nan"), float("inf"), 1e38, 1.0])
def test_tokens_without_weight(dtype, grad, junk):
    """A token whose dloss is zero counts in no gradient, whatever it holds, as with a loss that is masked by weights."""
    announce("tokens without weight", dtype, grad, junk)
    h, w, t, s = loss_case(150, 300, 96, dtype, 0.0, 53)
    gone = torch.rand(150, generator=gen(54)) < 0.3
    h[gone], s[gone] = 0, 0
    s[~gone] += 0.1
    _, _, dh, dw = check_loss(h, w, t, s, h.cuda(), w.cuda(), grad)
    h[gone, 5:9] = junk
    s[gone] *= -1  # (and the other zero)
    _, lse = daso.linear_cross_entropy(h.cuda(), w.cuda(), t.cuda())
    dh2, dw2 = daso.linear_cross_entropy_backward(s.cuda(), h.cuda(), w.cuda(), t.cuda(), lse,
                                                  dweight=torch.empty(300, 96, dtype=grad, device="cuda"))
    assert torch.equal(dh2, dh) and torch.equal(dw2, dw)


# ------------------------------------------------------------------------- layer norm of nothing
@pytest.mark.parametrize("rows", [0, 1, 700])
def test_layer_norm_of_empty_rows(rows):
    """A row of no elements has no mean: 0 / 0."""
    announce("layer norm of empty rows", rows)
    torch.full((4096,), 5.0, device="cuda")  # (what the allocator hands out next has been written)
    y, mean, rstd = daso.layer_norm(torch.empty(rows, 0, device="cuda"))
    assert y.shape == (rows, 0) and mean.shape == rstd.shape == (rows,)
    assert torch.isnan(mean).all() and torch.isnan(rstd).all()
    dx, dw, db = daso.layer_norm_backward(y, y, None, mean, rstd)
    assert dx.shape == (rows, 0) and dw.numel() == 0 and db.numel() == 0


# ------------------------------------------------------------------------- Newton-Schulz
@pytest.mark.parametrize("rows,cols", [(24, 40), (130, 200)])
@pytest.mark.parametrize("size", [3e-38, 1e-36])
def test_orthogonalize_of_tiny_matrices(rows, cols, size):
    """With eps = 0 the scale of a matrix does not matter, down to the smallest normal numbers."""
    announce("orthogonalize tiny", rows, cols, size)
    u = torch.randint(1, 4, (rows, cols), generator=gen(3)).float() * torch.sign(torch.randn(rows, cols, generator=gen(4)))
    got = daso.orthogonalize((u * size).cuda(), eps=0.0)
    want = O.newton_schulz(np64(u * size), [(3.4445, -4.7750, 2.0315)] * 5, 0.0)
    # as the tolerance of test_gpu_train for fp32: 4 roundings of 2^-21 a step, and what the weak directions add
    tol = 4 * 5 * 2.0 ** -21 + 2.0 ** -22 * 3.5 ** 5 / np.linalg.norm(want) + U
    assert np.linalg.norm(np64(got) - want) <= tol * np.linalg.norm(want)


# ------------------------------------------------------------------------- the step on other streams
def test_muon_step_on_streams_it_was_not_made_on():
    """The same bits, with the workspace's memory in use on the stream of construction before and after."""
    announce("muon step on other streams")
    mats, n = [(0, 192, 256), (49152, 256, 192)], 98304
    r = gen(61)
    grads, p0, m0 = [torch.randn(n, generator=r).cuda() for _ in range(4)], torch.randn(n, generator=r).cuda(), torch.randn(n, generator=r).cuda()
    want_p, want_m = p0.clone(), m0.clone()
    daso.muon_step(grads, want_p, want_m, mats, 0.1, 0.9)
    torch.cuda.synchronize()
    for _ in range(3):
        p, m = p0.clone(), m0.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        size = daso.MuonStep(grads, p, m, mats, 0.1, 0.9).args.workspace_bytes
        for _ in range(20):
            torch.empty(size, dtype=torch.uint8, device="cuda").fill_(255)  # (memory that the step is given next)
        step = daso.MuonStep(grads, p, m, mats, 0.1, 0.9)
        step(side)
        del step
        for _ in range(20):
            torch.empty(size, dtype=torch.uint8, device="cuda").fill_(255)
        side.synchronize()
        assert torch.equal(p, want_p) and torch.equal(m, want_m)


def test_muon_step_captured_on_another_stream():
    announce("muon step captured")
    mats, n = [(0, 192, 256), (49152, 256, 192)], 98304
    r = gen(62)
    grads, p0, m0 = [torch.randn(n, generator=r).cuda() for _ in range(2)], torch.randn(n, generator=r).cuda(), torch.randn(n, generator=r).cuda()
    p, m, want_p, want_m = p0.clone(), m0.clone(), p0.clone(), m0.clone()
    step, eager = daso.MuonStep(grads, p, m, mats, 0.1, 0.9), daso.MuonStep(grads, want_p, want_m, mats, 0.1, 0.9)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        graph.replay()
        eager()
        torch.cuda.synchronize()
        assert torch.equal(p, want_p) and torch.equal(m, want_m), k


@pytest.mark.parametrize("rows,cols", [(24, 40), (72, 100), (100, 72)])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_orthogonalize_in_several_rounds(rows, cols, out):
    """More matrices than are taken at a time, the last round with fewer; and in place."""
    announce("orthogonalize in rounds", rows, cols, out)
    u = torch.randn(300, rows, cols, generator=gen(71)).cuda()
    got = daso.orthogonalize(u, out=torch.full(u.shape, float("nan"), dtype=out, device="cuda"))
    for i in (0, 127, 128, 255, 256, 299):
        want = O.newton_schulz(np64(u[i]), [(3.4445, -4.7750, 2.0315)] * 5)
        plane = 2.0 ** -11 if out == torch.bfloat16 else 2.0 ** -21  # (the tolerance of test_gpu_train)
        tol = 4 * 5 * plane + 2.0 ** -22 * 3.5 ** 5 / np.linalg.norm(want) + (2.0 ** -8 if out == torch.bfloat16 else U)
        assert np.linalg.norm(np64(got[i]) - want) <= tol * np.linalg.norm(want), i
    if out == torch.float32:
        assert torch.equal(daso.orthogonalize(u, out=u), got)


# ------------------------------------------------------------------------- columns of one buffer
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 129, 9000])
def test_operands_that_are_columns_of_one_buffer(dtype, d):
    """Outputs beside the inputs of their rows: the bits of separate buffers, and nothing written between."""
    announce("columns of one buffer", dtype, d)
    n, v = 70, 90
    store = torch.full((n, 3 * d + 10), 3.0, dtype=dtype, device="cuda")
    x, y, z = store[:, 1:d + 1], store[:, d + 2:2 * d + 2], store[:, 2 * d + 7:3 * d + 7]
    x.copy_(torch.randn(n, d, generator=gen(d)))
    kept = store.clone()
    want, mean, rstd = daso.layer_norm(x.contiguous())
    got, mean2, rstd2 = daso.layer_norm(x, out=y)
    assert got is y and torch.equal(y, want) and torch.equal(mean, mean2) and torch.equal(rstd, rstd2)
    want = daso.layer_norm_backward(y.contiguous(), x.contiguous(), None, mean, rstd)
    got = daso.layer_norm_backward(y, x, None, mean, rstd, dx=z)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    z.copy_(kept[:, 2 * d + 7:3 * d + 7]), y.copy_(kept[:, d + 2:2 * d + 2])
    assert torch.equal(store, kept)
    w = (torch.randn(v, d, generator=gen(d + 1)) * 0.05).to(dtype).cuda()
    t, s = torch.randint(0, v, (n,), generator=gen(3)).cuda(), torch.rand(n, generator=gen(4)).cuda()
    want_loss, want_lse = daso.linear_cross_entropy(x.contiguous(), w, t)
    loss, lse = daso.linear_cross_entropy(x, w, t)
    assert torch.equal(loss, want_loss) and torch.equal(lse, want_lse)
    want, want_dw = daso.linear_cross_entropy_backward(s, x.contiguous(), w, t, lse)
    got, dw = daso.linear_cross_entropy_backward(s, x, w, t, lse, dhidden=y)
    assert torch.equal(y, want) and torch.equal(dw, want_dw)
    y.copy_(kept[:, d + 2:2 * d + 2])
    assert torch.equal(store, kept)
