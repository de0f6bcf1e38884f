"""Pins of the vocabulary projection's oracle: closed forms, library cross-checks, and the
gradients against differences of the loss."""
import numpy as np
import pytest
from scipy import special

from oracle import head_oracle as H


def _problem(seed, n, v, w, scale=1.0):
    g = np.random.default_rng(seed)
    return g.normal(size=(n, w)), g.normal(size=(v, w)) / np.sqrt(w) * scale, g.integers(0, v, n)


def test_quantize_closed_forms():
    x = np.array([[127.0, -63.5, 0.5, 1.5, 2.5, -2.5], [0.0] * 6, [1e-45] + [0.0] * 5, [2.0, np.inf, 0, 0, 0, 0],
                  [np.nan, 1, 0, 0, 0, 0], [-1.0, 1.0, 0, 0, 0, 0]])
    codes, scales = H.quantize_rows(x)
    assert list(scales[:3]) == [1.0, 0.0, 0.0] and np.isnan(scales[3]) and np.isnan(scales[4])
    assert list(codes[0]) == [127, -64, 0, 2, 2, -2]       # ties to even
    assert not codes[1:5].any() and list(codes[5][:2]) == [-127, 127]
    g = np.random.default_rng(0)
    x = g.normal(size=(5, 300)).astype(np.float32).astype(np.float64)
    codes, scales = H.quantize_rows(x)
    assert np.abs(codes * scales.astype(np.float64)[:, None] - x).max() <= 0.5 * scales.max() * (1 + 1e-6)
    assert (np.abs(codes).max(1) == 127).all()


def test_logits_are_the_product_of_the_values():
    g = np.random.default_rng(1)
    c, w = g.integers(-128, 128, (3, 40)).astype(np.int8), g.integers(-128, 128, (7, 40)).astype(np.int8)
    s, t = g.random(3).astype(np.float32), g.random(7).astype(np.float32)
    want = np.zeros((3, 7))
    for i in range(3):
        for j in range(7):
            want[i, j] = 2.5 * sum((float(c[i, k]) * float(s[i])) * (float(w[j, k]) * float(t[j])) for k in range(40))
    assert np.allclose(H.head_logits(c, s, w, t, 2.5), want, rtol=1e-13)


def test_loss_closed_forms_and_library():
    h, w, y = _problem(2, 6, 50, 8)
    loss, lse, z, _ = H.head_loss(h, w, y, 1.7)
    assert np.allclose(lse, special.logsumexp(1.7 * (h @ w.T), axis=1), rtol=1e-14)
    assert np.allclose(loss, -np.log(special.softmax(z, axis=1))[np.arange(6), y], rtol=1e-12)
    loss, lse, _, _ = H.head_loss(np.zeros((3, 4)), np.ones((10, 4)), [0, -1, 10], 1.0)
    assert np.allclose(lse, np.log(10)) and np.isclose(loss[0], np.log(10)) and loss[1] == 0 and np.isnan(loss[2])


@pytest.mark.parametrize("scale", [1.0, -0.5, 3.0])
def test_gradients_against_differences(scale):
    # central differences of a float64 loss: truncation eps^2 and rounding 1e-16/eps, both far
    # below 1e-7 at eps = 1e-5
    h, w, y = _problem(3, 4, 9, 5)
    y = np.array([0, 8, -1, 3])
    gl = np.array([0.5, -1.0, 2.0, 0.25])
    gh, _, gw, _, _, _ = H.head_loss_grad(h, w, y, gl, scale)

    def total(h, w):
        return float((H.head_loss(h, w, y, scale)[0] * gl).sum())

    eps = 1e-5
    for grad, x, f in ((gh, h, lambda x: total(x, w)), (gw, w, lambda x: total(h, x))):
        for at in np.ndindex(*x.shape):
            a, b = x.copy(), x.copy()
            a[at] += eps
            b[at] -= eps
            assert abs((f(a) - f(b)) / (2 * eps) - grad[at]) < 1e-7
    assert not gh[2].any()                                  # no label, no gradient
