"""Pins of the oracle of the norm of a site, the tail of a residual block and the 8-bit checkpoints: closed forms,
rotation equivariance with the Wigner-D matrices, finite differences of every gradient, and the rounding of a
checkpoint in exact arithmetic."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import sh
from oracle import site as os_

FIELDS = [((0, 3),), ((0, 4), (1, 2), (2, 1)), ((1, 3), (3, 1)), ((2, 2), (0, 5), (0, 1))]


def channels(fields):
    return sum(m * (2 * l + 1) for l, m in fields)


def count(fields):
    return sum(m for _, m in fields)


def rotation(rng):
    w, x, y, z = (lambda q: q / np.linalg.norm(q))(rng.standard_normal(4))
    return np.array([[1 - 2 * (y * y + z * z), 2 * (x * y - z * w), 2 * (x * z + y * w)],
                     [2 * (x * y + z * w), 1 - 2 * (x * x + z * z), 2 * (y * z - x * w)],
                     [2 * (x * z - y * w), 2 * (y * z + x * w), 1 - 2 * (x * x + y * y)]])


@pytest.mark.parametrize("fields", FIELDS)
def test_norm_closed_form(fields):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((7, channels(fields))) + 0.3
    y = os_.norm_forward(fields, x, eps=1e-12)
    for c, _, m, d in os_.entries(fields):
        v = y[:, c:c + m * d]
        if d == 1 and m == 1:
            assert np.all(v == 0)
            continue
        np.testing.assert_allclose((v * v).sum(1) / m, 1, rtol=1e-9)
        if d == 1:
            np.testing.assert_allclose(v.mean(1), 0, atol=1e-12)


@pytest.mark.parametrize("fields", FIELDS)
def test_equivariance(fields):
    rng = np.random.default_rng(2)
    D = sh.block_rep(fields, rotation(rng))
    full = os_.gate_fields(fields)
    Df = np.eye(channels(full))
    Df[:len(D), :len(D)] = D
    x, h, y = (rng.standard_normal((5, channels(f))) for f in (fields, fields, full))
    g, gp, sc = (rng.standard_normal(count(f)) for f in (fields, full, fields))
    np.testing.assert_allclose(os_.norm_forward(fields, x @ D.T, g), os_.norm_forward(fields, x, g) @ D.T, atol=1e-12)
    np.testing.assert_allclose(os_.residual_forward(fields, y @ Df.T, h @ D.T, sc, gp),
                               os_.residual_forward(fields, y, h, sc, gp) @ D.T, atol=1e-12)


def numeric(f, x, step=1e-6):
    """Central differences of a scalar function with respect to an array."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        v = x[i]
        x[i] = v + step
        a = f()
        x[i] = v - step
        b = f()
        x[i] = v
        g[i] = (a - b) / (2 * step)
    return g


@pytest.mark.parametrize("fields", FIELDS)
def test_norm_gradient(fields):
    rng = np.random.default_rng(3)
    x, dy = rng.standard_normal((2, 3, channels(fields)))
    gain = rng.standard_normal(count(fields))
    dx, dgain = os_.norm_backward(fields, x, dy, gain, 1e-2)
    f = lambda: float((os_.norm_forward(fields, x, gain, 1e-2) * dy).sum())  # noqa: E731
    np.testing.assert_allclose(dx, numeric(f, x), atol=1e-6)
    np.testing.assert_allclose(dgain, numeric(f, gain), atol=1e-6)


@pytest.mark.parametrize("fields", FIELDS)
@pytest.mark.parametrize("next_norm", [True, False])
def test_residual_gradient(fields, next_norm):
    rng = np.random.default_rng(4)
    full = os_.gate_fields(fields)
    y, h = rng.standard_normal((3, channels(full))), rng.standard_normal((3, channels(fields)))
    dh, dx = rng.standard_normal((2, 3, channels(fields)))
    sc, gp, gn = (rng.standard_normal(count(f)) for f in (fields, full, fields))
    eps = 1e-2

    def loss():
        ho = os_.residual_forward(fields, y, h, sc, gp, eps)
        v = (ho * dh).sum()
        return float(v + (os_.norm_forward(fields, ho, gn, eps) * dx).sum()) if next_norm else float(v)

    ho = os_.residual_forward(fields, y, h, sc, gp, eps)
    dy, dhin, dsc, dgp, dgn = os_.residual_backward(fields, y, ho, dh, dx if next_norm else None, sc, gp, gn, eps)
    for got, arr in ((dy, y), (dhin, h), (dsc, sc), (dgp, gp)) + (((dgn, gn),) if next_norm else ()):
        np.testing.assert_allclose(got, numeric(loss, arr), atol=2e-6)


def test_pack_against_exact_arithmetic():
    """Every block's exponent is the smallest k >= -126 at which all its values fit 127 steps, and every value the
    nearest step (half steps to even)."""
    rng = np.random.default_rng(5)
    fields = ((0, 33), (1, 11), (0, 2))
    x = (rng.standard_normal((40, 68)) * np.exp2(rng.integers(-130, 120, (40, 1)))).astype(np.float32)
    x[0] = 0
    x[1, :4] = np.array([127, 127.5, -63.25, 0.5]) * 2.0 ** -3
    x[1, 4:] = 0
    q, e = os_.pack(fields, x)
    assert q.shape == (40, 68) and e.shape == (40, 5)
    blocks = [(0, 32), (32, 33), (33, 65), (65, 66), (66, 68)]
    for r in range(40):
        for b, (lo, hi) in enumerate(blocks):
            k = int(e[r, b]) - 127
            amax = max(abs(Fraction(float(v))) for v in x[r, lo:hi])
            assert k >= -126 and amax <= 127 * Fraction(2) ** k
            if k > -126:
                assert amax > 127 * Fraction(2) ** (k - 1)
            for c in range(lo, hi):
                assert int(q[r, c]) == round(Fraction(float(x[r, c])) / Fraction(2) ** k)   # half to even
    assert np.all(q[0] == 0) and np.all(e[0] == 1)


def test_pack_error_and_non_finite():
    rng = np.random.default_rng(6)
    fields = ((0, 40), (2, 9))
    x = rng.standard_normal((50, 85)).astype(np.float32)
    v = os_.unpack(fields, *os_.pack(fields, x))
    for lo, hi in ((0, 32), (32, 40), (40, 72), (72, 85)):
        assert np.all(np.abs(v - x)[:, lo:hi] <= np.abs(x[:, lo:hi]).max(1, keepdims=True) / 127)
    x[3, 35], x[4, 50] = np.nan, -np.inf
    w = os_.unpack(fields, *os_.pack(fields, x))
    bad = np.isnan(w)
    assert bad[3, 32:40].all() and bad[4, 40:72].all() and bad.sum() == 8 + 32
    np.testing.assert_array_equal(w[~bad], v[~bad])
