"""Pins of the 64-bit oracle of the training operators, and mistakes planted in it that the pins catch."""
import numpy as np
import pytest

from oracle import train_oracle as O

QUINTIC = (3.4445, -4.7750, 2.0315)


def rng():
    return np.random.default_rng(20)


def differences(f, x, step=1e-6):
    """The gradient of the scalar f by central differences."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        hi, lo = x.copy(), x.copy()
        hi[i] += step
        lo[i] -= step
        g[i] = (f(hi) - f(lo)) / (2 * step)
    return g


# Central differences of step h are off by h^2 f'''/6 + 2^-52 |f| / h: below 1e-8 here.
CLOSE = dict(rtol=1e-6, atol=1e-7)


def pin_norm(mod):
    r = rng()
    x, w, b, dy = r.normal(size=(3, 7)), r.normal(size=7), r.normal(size=7), r.normal(size=(3, 7))
    y, mean, rstd = mod.layer_norm(x, w, b, 1e-3)
    np.testing.assert_allclose(((y - b) / w).mean(axis=1), 0, atol=1e-12)
    np.testing.assert_allclose((((y - b) / w) ** 2).mean(axis=1), x.var(axis=1) / (x.var(axis=1) + 1e-3), rtol=1e-12)
    dx, dw, db = mod.layer_norm_backward(dy, x, w, mean, rstd)
    np.testing.assert_allclose(dx, differences(lambda v: (O.layer_norm(v, w, b, 1e-3)[0] * dy).sum(), x), **CLOSE)
    np.testing.assert_allclose(dw, differences(lambda v: (O.layer_norm(x, v, b, 1e-3)[0] * dy).sum(), w), **CLOSE)
    np.testing.assert_allclose(db, differences(lambda v: (O.layer_norm(x, w, v, 1e-3)[0] * dy).sum(), b), **CLOSE)


def pin_loss(mod):
    r = rng()
    h, w, s = r.normal(size=(4, 5)), r.normal(size=(6, 5)), r.normal(size=4)
    t = np.array([2, -100, 0, 5])
    loss, lse = mod.linear_cross_entropy(h, w, t)
    z = h @ w.T
    np.testing.assert_allclose(np.exp(z - lse[:, None]).sum(axis=1), 1, rtol=1e-12)
    np.testing.assert_allclose(loss[[0, 2, 3]], [-np.log(np.exp(z[i, t[i]]) / np.exp(z[i]).sum()) for i in (0, 2, 3)], rtol=1e-12)
    assert loss[1] == 0
    dh, dw, _ = mod.linear_cross_entropy_backward(s, h, w, t)
    np.testing.assert_allclose(dh, differences(lambda v: (O.linear_cross_entropy(v, w, t)[0] * s).sum(), h), **CLOSE)
    np.testing.assert_allclose(dw, differences(lambda v: (O.linear_cross_entropy(h, v, t)[0] * s).sum(), w), **CLOSE)


def pin_schulz(mod):
    for shape in ((5, 8), (8, 5), (6, 6)):
        u = rng().normal(size=shape)
        left, sigma, right = np.linalg.svd(u, full_matrices=False)
        sigma = sigma / (np.sqrt((sigma ** 2).sum()) + 1e-7)
        for a, b, c in [QUINTIC] * 4 + [(1.5, -0.5, 0.0)]:
            sigma = a * sigma + b * sigma ** 3 + c * sigma ** 5
        np.testing.assert_allclose(mod.newton_schulz(u, [QUINTIC] * 4 + [(1.5, -0.5, 0.0)]), (left * sigma) @ right, rtol=1e-9, atol=1e-12)


def pin_muon(mod):
    r = rng()
    grads, x, m = [r.normal(size=40) for _ in range(3)], r.normal(size=40), r.normal(size=40)
    mats = [(2, 3, 4, 1.0), (20, 5, 2, 1.5)]
    for nesterov in (False, True):
        got_x, got_m = mod.muon_step(grads, x, m, mats, 0.1, 0.9, 0.01, nesterov, [QUINTIC] * 5)
        mean = (grads[0] + grads[1] + grads[2]) / 3
        inside = np.zeros(40, bool)
        for start, rows, cols, scale in mats:
            cut = slice(start, start + rows * cols)
            inside[cut] = True
            want_m = 0.9 * m[cut] + mean[cut]
            np.testing.assert_allclose(got_m[cut], want_m, rtol=1e-12)
            u = (mean[cut] + 0.9 * want_m if nesterov else want_m).reshape(rows, cols)
            step = (x[cut] * (1 - 0.1 * 0.01) - got_x[cut]).reshape(rows, cols) / (0.1 * scale)
            # the update has u's singular vectors: step^T u and step u^T are symmetric
            np.testing.assert_allclose(step.T @ u, (step.T @ u).T, atol=1e-9)
            np.testing.assert_allclose(step @ u.T, (step @ u.T).T, atol=1e-9)
            assert (step * u).sum() > 0 and 0.6 < np.linalg.svd(step)[1].min() and np.linalg.svd(step)[1].max() < 1.3
        np.testing.assert_array_equal(got_x[~inside], x[~inside])
        np.testing.assert_array_equal(got_m[~inside], m[~inside])


PINS = {"norm": pin_norm, "loss": pin_loss, "schulz": pin_schulz, "muon": pin_muon}


@pytest.mark.parametrize("name", PINS)
def test_pin(name):
    PINS[name](O)


MUTANTS = [
    ("norm", "np.mean((x - mean) ** 2, axis=1, keepdims=True)", "np.mean(x ** 2, axis=1, keepdims=True)"),
    ("norm", "+ eps)\n    y", ")\n    y"),
    ("norm", "- g.sum(axis=1, keepdims=True) / d", ""),
    ("norm", "- xhat * (g * xhat)", "- xhat * g"),
    ("norm", "(dy * xhat).sum(axis=0)", "(dy * x).sum(axis=0)"),
    ("norm", "dy * np.asarray(weight, np.float64)", "dy"),
    ("loss", "lse[i] - z[i, t]", "top[i] - z[i, t]"),
    ("loss", "if t == ignore_index:\n            continue", "if t == ignore_index:\n            t = 0"),
    ("loss", "p[i, t] -= 1.0\n            p[i] *= float(dloss[i])", "p[i] *= float(dloss[i])\n            p[i, t] -= 1.0"),
    ("loss", "p[i] = 0.0", "p[i] *= 1.0"),
    ("loss", "p @ w, p.T @ h", "p @ w, (p / len(p)).T @ h"),
    ("schulz", "b * gram + c * gram @ gram", "b * gram + c * gram * gram"),
    ("schulz", "np.sqrt((x * x).sum())", "np.abs(x).sum()"),
    ("schulz", "return x.T if tall else x", "return x if tall else x.T"),
    ("muon", "m[cut] = mu * m[cut] + gbar[cut]", "m[cut] = mu * m[cut] + (1 - mu) * gbar[cut]"),
    ("muon", "u = gbar[cut] + mu * m[cut] if nesterov else m[cut]", "u = m[cut]"),
    ("muon", "(1.0 - lr * weight_decay)", "(1.0 - weight_decay)"),
    ("muon", "lr * scale * o", "lr * o"),
    ("muon", "/ len(grads)", ""),
]


@pytest.mark.parametrize("pin,old,new", MUTANTS)
def test_planted_mistakes_are_caught(pin, old, new):
    source = open(O.__file__).read()
    assert source.count(old) >= 1, old
    mod = type(O)("mutant")
    exec(compile(source.replace(old, new), "mutant", "exec"), mod.__dict__)
    with pytest.raises((AssertionError, ValueError)):
        PINS[pin](mod)
