"""Pins of the layers' oracle: closed forms, special cases, and gradients against differences."""
import numpy as np
import pytest

from oracle import layers as L
from oracle import rng


def _numeric(f, v, eps=1e-6):
    g = np.zeros_like(v)
    for i in np.ndindex(v.shape):
        a, b = v.copy(), v.copy()
        a[i] += eps
        b[i] -= eps
        g[i] = (f(a) - f(b)) / (2 * eps)
    return g


def test_scan_closed_forms():
    T = 20
    x = np.ones((T, 1, 1))
    h, last, _, _ = L.scan(np.full((T, 1, 1), 0.5), x, "decay", h0=np.zeros((1, 1)))
    assert np.allclose(h[:, 0, 0], 2 - 0.5 ** np.arange(T)) and last[0, 0] == h[-1, 0, 0]
    h, _, _, _ = L.scan(np.zeros((T, 1, 1)), x)          # f = 1/2: an average towards 1
    assert np.allclose(h[:, 0, 0], 1 - 0.5 ** (np.arange(T) + 1))


def test_scan_masks():
    r = np.random.default_rng(0)
    T, n, c = 9, 3, 2
    gate, x = r.normal(size=(T, n, c)), r.normal(size=(T, n, c))
    done = np.zeros((T, n))
    done[3, 1] = 1
    h, last, _, _ = L.scan(gate, x, done=done)
    fresh, _, _, _ = L.scan(gate[4:, 1:2], x[4:, 1:2])   # the steps after an end: an episode of their own
    assert np.allclose(h[4:, 1:2], fresh)
    lens = np.array([0, 4, 9])
    h0 = r.normal(size=(n, c))
    gate[:, 0] = np.nan                                  # a sequence of no steps is not looked at
    h, last, _, _ = L.scan(gate, x, lens=lens, h0=h0)
    assert np.array_equal(last[0], h0[0]) and np.array_equal(h[:, 0], np.broadcast_to(h0[0], (T, c)))
    assert np.array_equal(last[1], h[3, 1]) and np.isfinite(h).all()


@pytest.mark.parametrize("kind", ["sigmoid", "decay"])
def test_scan_gradient_against_differences(kind):
    r = np.random.default_rng(1)
    T, n, c = 6, 3, 2
    gate, x, h0 = r.normal(size=(T, n, c)), r.normal(size=(T, n, c)), r.normal(size=(n, c))
    done = (r.random((T, n)) < 0.3).astype(float)
    lens = np.array([6, 2, 0])
    dout, dlast = r.normal(size=(T, n, c)), r.normal(size=(n, c))

    def loss(gate, x, h0):
        h, last, _, _ = L.scan(gate, x, kind, done, lens, h0)
        return (h * dout).sum() + (last * dlast).sum()

    h = L.scan(gate, x, kind, done, lens, h0)[0]
    dgate, dx, dh0, _, _, _ = L.scan_grad(gate, x, h, dout, dlast, kind, done, lens, h0)
    assert np.allclose(dgate, _numeric(lambda v: loss(v, x, h0), gate), atol=1e-8)
    assert np.allclose(dx, _numeric(lambda v: loss(gate, v, h0), x), atol=1e-8)
    assert np.allclose(dh0, _numeric(lambda v: loss(gate, x, v), h0), atol=1e-8)


def test_drop_factor_draws():
    seed, step, site, row0 = 0x123456789ABCDEF0, 7, 5, 1000
    f = L.drop_factor(3, 19, 20000, seed, step, site, row0)
    for row in range(3):
        for c in range(19):
            w = rng.philox4x32_10((row0 + row, step, 3 | site << 8, c // 8), rng.key_of(seed))
            half = w[(c % 8) // 2] >> (16 * (c % 2)) & 0xFFFF
            assert f[row, c] == (65536 / 45536 if half >= 20000 else 0.0)
    assert (L.drop_factor(50, 9, 0, 1) == 1).all()
    big = L.drop_factor(400, 100, 6554, 3)      # 40000 draws: the share dropped within 5 deviations
    assert abs((big == 0).mean() - 6554 / 65536) < 5 * np.sqrt(0.09 / big.size)
    assert np.array_equal(L.drop_factor(10, 9, 30000, 1, row0=4), L.drop_factor(14, 9, 30000, 1)[4:])


@pytest.mark.parametrize("act", ["none", "relu", "silu", "tanh"])
@pytest.mark.parametrize("groups", [1, 2, 6])
def test_norm_and_gradient(act, groups):
    r = np.random.default_rng(2)
    n, s, c = 2, 3, 6
    x, dout = r.normal(size=(n, s, c)), r.normal(size=(n, s, c))
    w, b = r.normal(size=c), r.normal(size=c)
    factor = L.drop_factor(n * s, c, 10000, 5).reshape(n, s, c)
    y, mean, rstd = L.norm(x, groups, act="none", factor=factor, eps=0.0)
    v = y.reshape(n, s, groups, -1)
    assert np.allclose(v.mean(axis=(1, 3)), 0) and np.allclose((v * v).mean(axis=(1, 3)), 1)
    loss = lambda x, w, b: (L.norm(x, groups, w, b, 1e-3, act, factor)[0] * dout).sum()  # noqa: E731
    _, mean, rstd = L.norm(x, groups, w, b, 1e-3, act, factor)
    dx, dw, db = L.norm_grad(x, groups, mean, rstd, dout, w, b, act, factor)
    assert np.allclose(dx, _numeric(lambda q: loss(q, w, b), x), atol=1e-7)
    assert np.allclose(dw, _numeric(lambda q: loss(x, q, b), w), atol=1e-7)
    assert np.allclose(db, _numeric(lambda q: loss(x, w, q), b), atol=1e-7)
