"""Pins of the transformer block's oracle: properties that its formulas do not spell out, and gradients against differences."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as O

RNG = np.random.default_rng


def differences(f, x, dy, eps=1e-6):
    """The gradient of sum(f(x) * dy), element by element."""
    grad = np.zeros_like(x)
    it = np.nditer(x, flags=["multi_index"])
    for _ in it:
        i = it.multi_index
        keep = x[i]
        x[i] = keep + eps
        up = (f(x) * dy).sum()
        x[i] = keep - eps
        grad[i] = (up - (f(x) * dy).sum()) / (2 * eps)
        x[i] = keep
    return grad


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dim,rotated", [(16, 16), (16, 8), (8, 0)])
def test_rotary_gradients_against_differences(inter, dim, rotated):
    r = RNG(1)
    x, dy, w = r.normal(size=(3, 2, dim)), r.normal(size=(3, 2, dim)), r.normal(size=dim)
    at, freq = np.array([0, 5, 11]), 10.0 ** -np.arange(rotated // 2)
    dx, dw = O.head_norm_rotary_backward(dy, x, at, freq, w, 1e-3, inter)
    assert np.allclose(dx, differences(lambda t: O.head_norm_rotary(t, at, freq, w, 1e-3, inter), x, dy), atol=1e-7)
    assert np.allclose(dw, differences(lambda t: O.head_norm_rotary(x, at, freq, t, 1e-3, inter), w, dy), atol=1e-7)


@pytest.mark.parametrize("inter", [False, True])
def test_rotation_keeps_norms_and_products_depend_on_distance(inter):
    r, dim = RNG(2), 32
    freq = 100.0 ** -(np.arange(16) / 16)
    a, b = (np.repeat(r.normal(size=(1, 1, dim)), 9, axis=0) for _ in range(2))
    ya, yb = (O.head_norm_rotary(t, np.arange(9), freq, None, 0.0, inter)[:, 0] for t in (a, b))
    assert np.allclose((ya ** 2).sum(axis=1), dim)
    dots = ya @ yb.T
    for shift in range(1, 5):
        assert np.allclose(np.diag(dots, shift), np.diag(dots, shift)[0])
    assert not np.isclose(dots[0, 1], dots[0, 4])
    # a quarter turn takes the first element of the pair to the second
    one = np.zeros((1, 1, 4))
    one[..., 0] = 2.0
    y = O.head_norm_rotary(one, np.array([1]), np.array([np.pi / 2, 1.0]), None, 0.0, inter)[0, 0]
    assert np.allclose(y, [0, 2, 0, 0] if inter else [0, 0, 2, 0])


@pytest.mark.parametrize("causal", [True, False])
def test_attention_against_torch_sequence_by_sequence(causal):
    r, ends = RNG(3), [0, 4, 4, 5, 12]
    q, k, v = r.normal(size=(12, 6, 8)), r.normal(size=(12, 2, 8)), r.normal(size=(12, 2, 8))
    out, lse, _ = O.attention(q, k, v, ends, causal)
    for a, b in zip(ends[:-1], ends[1:]):
        for h in range(6) if b > a else ():
            tq, tk, tv = (torch.from_numpy(t[a:b, i]) for t, i in ((q, h), (k, h // 3), (v, h // 3)))
            z = tq @ tk.T / 8 ** 0.5
            if causal:
                z = z.masked_fill(torch.ones(b - a, b - a).triu(1).bool(), -float("inf"))
            assert np.allclose(out[a:b, h], z.softmax(1) @ tv) and np.allclose(lse[h, a:b], z.logsumexp(1))


@pytest.mark.parametrize("causal", [True, False])
def test_attention_gradients_against_differences(causal):
    r, ends = RNG(4), [0, 3, 7]
    q, k, v, dout = (r.normal(size=(8, h, 4)) for h in (4, 2, 2, 4))
    dout[7] = 0  # the last token is in no sequence
    got = O.attention_backward(dout, q, k, v, ends, causal, 0.7)
    f = lambda q, k, v: np.nan_to_num(O.attention(q, k, v, ends, causal, 0.7)[0])  # noqa: E731
    assert np.allclose(got[0], differences(lambda t: f(t, k, v), q, dout), atol=1e-7)
    assert np.allclose(got[1], differences(lambda t: f(q, t, v), k, dout), atol=1e-7)
    assert np.allclose(got[2], differences(lambda t: f(q, k, t), v, dout), atol=1e-7)


def test_clipping_against_torch():
    r = RNG(5)
    x = [r.normal(size=100) for _ in range(3)]
    mean = torch.from_numpy(np.mean(x, axis=0))
    pieces = [torch.nn.Parameter(mean[a:a + k].clone()) for a, k in ((0, 10), (10, 90))]
    for p in pieces:
        p.grad = p.detach().clone()
    norm = torch.nn.utils.clip_grad_norm_(pieces, 0.5)
    out, got, norms = O.clip_gradients(x, 0.5, [(0, 10), (10, 90)])
    assert np.allclose(got, float(norm)) and np.allclose(out, np.concatenate([p.grad.numpy() for p in pieces]))
    assert np.allclose(norms, [float(mean[:10].norm()), float(mean[10:].norm())])
    assert np.allclose(O.clip_gradients(x, 1e3, [(0, 100)])[0], mean)
