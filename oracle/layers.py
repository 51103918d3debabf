"""Network layers over rollouts (oracle side): the gated linear recurrence, group norm with an
activation, dropout from the counter-based generator, and the gradients of the first two, written out
step by step in float64.

Recurrence of n sequences with c channels, s_{-1} = h0:
    sigmoid: f = sigma(gate), h_t = f s_{t-1} + (1 - f) x_t;   decay: f = gate, h_t = f s_{t-1} + x_t
    s_t = 0 where the episode ended at step t, else h_t; held steps (t >= len): h_t = s_t = s_{t-1}
Its gradient with G_t that of s_t: g_t = dh_t + (1 - done_t) G_t, G_{t-1} = f_t g_t, and
    sigmoid: dx = (1 - f) g, dgate = f (1 - f) (s_{t-1} - x) g;   decay: dx = g, dgate = s_{t-1} g
    held steps: dx = dgate = 0, G_{t-1} = dh_t + G_t.
"""
from __future__ import annotations

import numpy as np

from . import rng

TAG_DROPOUT = 3


def _gates(gate, kind):
    """f and the input's weight."""
    if kind == "decay":
        return gate, np.ones_like(gate)
    e = np.exp(-np.abs(gate))
    big, small = 1 / (1 + e), e / (1 + e)
    return np.where(gate >= 0, big, small), np.where(gate >= 0, small, big)


def _masks(T, n, done, lens):
    hold = np.zeros((T, n), bool) if lens is None else np.arange(T)[:, None] >= np.asarray(lens)[None, :]
    end = np.zeros((T, n), bool) if done is None else np.asarray(done) != 0
    return (end & ~hold)[..., None], hold[..., None]


def scan(gate, x, kind="sigmoid", done=None, lens=None, h0=None, delta=0.0):
    """[T, n, c] -> h, last [n, c], and a bound on the rounding errors of h and last: every step's terms
    are taken as wrong by delta of their size (a number or [T, n, c])."""
    gate, x = np.asarray(gate, np.float64), np.asarray(x, np.float64)
    T, n, c = x.shape
    f, w = _gates(gate, kind)
    end, hold = _masks(T, n, done, lens)
    delta = np.broadcast_to(np.asarray(delta, np.float64), x.shape)
    s = np.zeros((n, c)) if h0 is None else np.array(h0, np.float64)
    err = np.zeros((n, c))
    h, bound = np.zeros_like(x), np.zeros_like(x)
    for t in range(T):
        ht = np.where(hold[t], s, f[t] * s + w[t] * x[t])
        e = np.where(hold[t], err, np.abs(f[t]) * err + delta[t] * (np.abs(f[t] * s) + np.abs(w[t] * x[t])))
        h[t], bound[t] = ht, e
        s, err = np.where(end[t], 0.0, ht), np.where(end[t], 0.0, e)
    return h, s, bound, err


def scan_grad(gate, x, h, dout=None, dlast=None, kind="sigmoid", done=None, lens=None, h0=None, delta=0.0):
    """(dgate, dx, dh0) and bounds on their rounding errors.  The state before a step is the recurrence's own, in 64 bits:
    `h`, the output as it was stored, is rounded to the tensors' type and not looked at."""
    gate, x = (np.asarray(v, np.float64) for v in (gate, x))
    T, n, c = x.shape
    f, w = _gates(gate, kind)
    end, hold = _masks(T, n, done, lens)
    delta = np.broadcast_to(np.asarray(delta, np.float64), x.shape)
    state, _, es, _ = scan(gate, x, kind, done, lens, h0, delta)
    dout = np.zeros_like(x) if dout is None else np.asarray(dout, np.float64)
    G = np.zeros((n, c)) if dlast is None else np.array(dlast, np.float64)
    err = np.zeros((n, c))
    dgate, dx, eg, ex = (np.zeros_like(x) for _ in range(4))
    for t in range(T - 1, -1, -1):
        G, err = np.where(end[t], 0.0, G), np.where(end[t], 0.0, err)
        g = dout[t] + G
        e = err + delta[t] * (np.abs(dout[t]) + np.abs(G))
        if t:
            s, b = np.where(end[t - 1], 0.0, state[t - 1]), np.where(end[t - 1], 0.0, es[t - 1])
        else:
            s, b = np.zeros((n, c)) if h0 is None else np.asarray(h0, np.float64), np.zeros((n, c))
        if kind == "sigmoid":
            d = s - x[t]
            gz, gx = f[t] * w[t] * d * g, w[t] * g
            ez = np.abs(f[t] * w[t]) * ((np.abs(d) + b) * e + (b + 4 * delta[t] * (np.abs(s) + np.abs(x[t]))) * np.abs(g))
            ew = np.abs(w[t]) * (e + delta[t] * np.abs(g))
        else:
            gz, gx, ez, ew = s * g, g, (np.abs(s) + b) * e + (b + np.abs(s) * delta[t]) * np.abs(g), e
        dgate[t], dx[t] = np.where(hold[t], 0.0, gz), np.where(hold[t], 0.0, gx)
        eg[t], ex[t] = np.where(hold[t], 0.0, ez), np.where(hold[t], 0.0, ew)
        G = np.where(hold[t], g, f[t] * g)
        err = np.where(hold[t], e, np.abs(f[t]) * (e + delta[t] * np.abs(g)))
    return dgate, dx, G, eg, ex, err


def drop_factor(rows: int, c: int, drop: int, seed: int, step: int = 0, site: int = 0, row0: int = 0) -> np.ndarray:
    """[rows, c] factors 0 or 65536 / (65536 - drop) of dropout's draws: half j of the Philox block with
    counter (row0 + row, step, 3 | site << 8, channel / 8), low halves of the words first."""
    blocks = -(-c // 8)
    w = rng.philox4x32_10_np(row0 + np.arange(rows)[:, None], step, TAG_DROPOUT | site << 8, np.arange(blocks)[None, :],
                             rng.key_of(seed))                       # [4, rows, blocks]
    halves = np.stack([w & np.uint32(0xFFFF), w >> np.uint32(16)], axis=1).reshape(8, rows, blocks)
    keep = np.moveaxis(halves, 0, 2).reshape(rows, blocks * 8)[:, :c] >= drop
    return np.where(keep, 65536.0 / (65536 - drop), 0.0)


def _act(act, u):
    """act(u) and its derivative."""
    if act == "relu":
        return np.where(u < 0, 0.0, u), (u > 0).astype(np.float64)
    if act == "silu":
        s, _ = _gates(u, "sigmoid")
        return u * s, s * (1 + u * (1 - s))
    if act == "tanh":
        y = np.tanh(u)
        return y, 1 / np.cosh(np.clip(u, -350, 350)) ** 2
    return u, np.ones_like(u)


def norm(x, groups, weight=None, bias=None, eps=1e-5, act="none", factor=None):
    """[n, s, c] -> y, mean [n, groups], rstd [n, groups]; factor [n, s, c]: dropout in front."""
    x = np.asarray(x, np.float64)
    n, s, c = x.shape
    if factor is not None:
        x = np.where(factor == 0, 0.0, x * factor)
    v = x.reshape(n, s, groups, c // groups)
    mean = v.mean(axis=(1, 3))
    d = v - mean[:, None, :, None]
    rstd = 1 / np.sqrt((d * d).mean(axis=(1, 3)) + eps)
    xh = (d * rstd[:, None, :, None]).reshape(n, s, c)
    u = xh * (1.0 if weight is None else np.asarray(weight, np.float64)) + (0.0 if bias is None else np.asarray(bias, np.float64))
    return _act(act, u)[0], mean, rstd


def norm_grad(x, groups, mean, rstd, dout, weight=None, bias=None, act="none", factor=None):
    """(dx, dweight, dbias) for the given statistics."""
    x, dout = np.asarray(x, np.float64), np.asarray(dout, np.float64)
    n, s, c = x.shape
    if factor is not None:
        x = np.where(factor == 0, 0.0, x * factor)
    per = lambda q: np.repeat(np.asarray(q, np.float64), c // groups, axis=1)[:, None, :]  # noqa: E731
    w = np.ones(c) if weight is None else np.asarray(weight, np.float64)
    b = np.zeros(c) if bias is None else np.asarray(bias, np.float64)
    xh = (x - per(mean)) * per(rstd)
    du = dout * _act(act, xh * w + b)[1]
    d = du * w
    avg = lambda q: per(q.reshape(n, s, groups, c // groups).mean(axis=(1, 3)))  # noqa: E731
    dx = per(rstd) * (d - avg(d) - xh * avg(d * xh))
    if factor is not None:
        dx = np.where(factor == 0, 0.0, dx * factor)
    return dx, (du * xh).sum(axis=(0, 1)), du.sum(axis=(0, 1))
