"""GPU parity of the network layers (gated recurrence, group norm, dropout) with their float64 oracle.

Tolerances are bounds, not measurements.  u = 2^-24 is half a step of fp32 and R(t) that of a stored
value (bf16 2^-8, fp32 2^-24).  Recurrence: the oracle carries each step's error along, every term
taken as wrong by delta of its size, delta = (|z| + 24) u for a gate z (the exponent's argument z log2 e
is rounded once, |z| u of e^-z; the exponential, reciprocal, products and the split over step ranges
make less than 24 roundings more).  Norm: sums of m terms over D additions in a row are wrong by D u of the terms'
size, D = 64 + the positions one thread walks over (at most all of them)."""
import numpy as np
import pytest
import torch

from oracle import layers as L
from tests.gpu_util import announce, host, require_gpu

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}
TINY = 2.0 ** -120      # below it hardware functions give zero


def f64(t):
    return None if t is None else host(t.float()).astype(np.float64)


def within(got, want, bound, what):
    got, bound = f64(got), np.broadcast_to(bound, want.shape)
    assert got.shape == want.shape, what
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    bad = np.abs(got - want) > bound + TINY
    bad &= ~((got == want) | np.isnan(want))
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[0], got[bad][:3], want[bad][:3], bound[bad][:3])


def seq(g, T, n, c, typ, order, scale=1.0, shift=0.0):
    """A logical [T][n][c] tensor in a memory order; halves of one wider buffer where it ends in 2."""
    shape = {"tnc": (T, n, c), "ntc": (n, T, c), "ntc2": (n, T, 2 * c), "cnt": (c, T, n), "nct": (n, c, T),
             "tcn": (T, c, n), "odd": (T, n, c + 3)}[order]
    t = (torch.randn(shape, generator=g, device="cuda") * scale + shift).to(TYPES[typ])
    if order in ("ntc", "ntc2"):
        return t[..., :c].permute(1, 0, 2)
    if order == "cnt":
        return t.permute(1, 2, 0)
    if order == "nct":
        return t.permute(2, 0, 1)
    if order == "tcn":
        return t.permute(0, 2, 1)
    return t[..., 1:1 + c] if order == "odd" else t


def scan_inputs(T, n, c, typ, kind, order, masks, seed=0):
    """masks: d episode ends, l lengths (in "plain" too, which has no initial state), h an initial state only, "" nothing."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if order == "ntc2":     # gate and input as the halves of one buffer
        both = torch.randn((n, T, 2 * c), generator=g, device="cuda").to(TYPES[typ])
        gate, x = both[..., :c].permute(1, 0, 2), both[..., c:].permute(1, 0, 2)
    else:
        gate, x = seq(g, T, n, c, typ, order, 2.0, 1.0), seq(g, T, n, c, typ, order)
    if kind == "decay":
        gate.copy_(torch.sigmoid(gate.float()) * 1.25 - 0.3)     # negative, zero-crossing and above one too
    done = lens = None
    h0 = torch.randn((n, c), generator=g, device="cuda") if masks not in ("", "plain") else None
    if "d" in masks:
        done = (torch.rand((T, n), generator=g, device="cuda") < 0.07).float()
        done[:, 0] = 1.0                                         # a sequence that ends at every step
    if "l" in masks:
        lens = torch.randint(0, T + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
        lens[-1] = 0                                             # an empty sequence
        if n > 2:
            lens[1], lens[2] = T + 5, -3
    dout, dlast = seq(g, T, n, c, typ, order if order != "ntc2" else "ntc"), torch.randn((n, c), generator=g, device="cuda")
    return gate, x, done, lens, h0, dout, dlast


def check_scan(T, n, c, typ, kind, order, masks, seed=0):
    from paper_2512_13359_amd import scan_backward, scan_forward
    gate, x, done, lens, h0, dout, dlast = scan_inputs(T, n, c, typ, kind, order, masks, seed)
    more = dict(kind=kind, done=done, lens=lens, h0=h0)
    h, last = scan_forward(gate, x, **more)
    dgate, dx, dh0 = scan_backward(gate, x, h, dout=dout, dh_last=dlast, **more)
    delta = (np.abs(f64(gate)) * (kind == "sigmoid") + 24) * U
    m = dict(kind=kind, done=None if done is None else host(done), lens=None if lens is None else host(lens), h0=f64(h0), delta=delta)
    wh, wl, bh, bl = L.scan(f64(gate), f64(x), **m)
    r = HALF[typ]
    within(h, wh, bh + r * (np.abs(wh) + bh), "h")
    within(last, wl, bl + U * np.abs(wl), "last")
    # the gradient for the h that was stored
    wg, wx, w0, bg, bx, b0 = L.scan_grad(f64(gate), f64(x), f64(h), f64(dout), f64(dlast), **m)
    within(dgate, wg, bg + r * (np.abs(wg) + bg), "dgate")
    within(dx, wx, bx + r * (np.abs(wx) + bx), "dx")
    within(dh0, w0, b0 + U * np.abs(w0), "dh0")


@pytest.mark.parametrize("kind", ["sigmoid", "decay"])
@pytest.mark.parametrize("typ", ["fp32", "bf16"])
@pytest.mark.parametrize("T, n, c", [(1, 1, 1), (1, 5, 3), (2, 3, 8), (5, 33, 17), (33, 9, 16), (70, 65, 1), (130, 3, 23),
                                     (515, 1, 2), (1100, 2, 5), (2500, 3, 17)])
def test_scan_sizes(T, n, c, typ, kind):
    require_gpu()
    for masks in ("plain", "h", "dl"):
        announce(f"scan T={T} n={n} c={c} {typ} {kind} {masks}")
        check_scan(T, n, c, typ, kind, "tnc", masks, seed=T + n + c)


@pytest.mark.parametrize("order", ["tnc", "ntc", "ntc2", "cnt", "nct", "tcn", "odd"])
@pytest.mark.parametrize("typ", ["fp32", "bf16"])
def test_scan_orders(order, typ):
    require_gpu()
    for T, n, c, masks in ((37, 6, 9, "dl"), (37, 9, 6, "plain"), (64, 67, 40, "d"), (3, 1, 13, "l"), (1200, 3, 4, "dl"), (9, 130, 1, "dl")):
        announce(f"scan order {order} T={T} n={n} c={c} {typ} {masks}")
        check_scan(T, n, c, typ, "sigmoid", order, masks, seed=c)


@pytest.mark.parametrize("order", ["tnc", "ntc2", "cnt", "nct", "tcn"])
@pytest.mark.parametrize("kind", ["sigmoid", "decay"])
def test_scan_orders_without_masks(order, kind):
    """No episode ends, no lengths, with and without an initial state, the sequence or the channel as the longer axis."""
    require_gpu()
    for T, n, c in ((20, 50, 6), (20, 6, 50), (1, 9, 40), (1300, 2, 9), (5, 700, 31)):
        for masks in ("", "h"):
            for typ in ("fp32", "bf16"):
                announce(f"scan order {order} T={T} n={n} c={c} {typ} {kind} masks '{masks}'")
                check_scan(T, n, c, typ, kind, order, masks, seed=n)


@pytest.mark.parametrize("typ", ["fp32", "bf16"])
@pytest.mark.parametrize("T, n, c, order", [(3, 16385, 63, "tnc"), (40, 4095, 23, "cnt"), (6, 4099, 64, "ntc2"), (300, 300, 256, "tnc")])
def test_scan_many_columns(T, n, c, order, typ):
    """One wave per workgroup, several, with a ragged end of the columns."""
    require_gpu()
    announce(f"scan many T={T} n={n} c={c} {order} {typ}")
    check_scan(T, n, c, typ, "sigmoid", order, "d", seed=1)


@pytest.mark.parametrize("T", [9, 1500])
@pytest.mark.parametrize("typ", ["fp32", "bf16"])
def test_scan_masked_places_hold_anything(T, typ):
    """NaN and infinities at held steps, and a state that is not finite before an episode's end,
    leave everything behind them as it is."""
    require_gpu()
    from paper_2512_13359_amd import scan_backward, scan_forward
    n, c = 3, 8
    gate, x, _, _, h0, dout, dlast = scan_inputs(T, n, c, typ, "sigmoid", "tnc", "h", 5)
    done = torch.zeros(T, n, device="cuda")
    done[4, 0] = 1.0
    lens = torch.tensor([T, 5, 0], dtype=torch.int32, device="cuda")
    clean = scan_forward(gate, x, done=done, lens=lens, h0=h0)
    dirty_gate, dirty_x, dirty_done = gate.clone(), x.clone(), done.clone()
    for t in (dirty_gate, dirty_x):
        t[5:, 1] = float("nan")
        t[:, 2] = float("-inf")
    dirty_done[5:, 1] = float("nan")
    dirty_x[2, 0] = float("inf")                   # an infinite state until the end at step 4
    h, last = scan_forward(dirty_gate, dirty_x, done=dirty_done, lens=lens, h0=h0)
    assert torch.equal(last, clean[1])
    assert torch.equal(h[5:], clean[0][5:]) and torch.equal(h[:, 1:], clean[0][:, 1:]) and torch.isinf(h[2:5, 0]).all()
    assert torch.equal(last[2], h0[2])
    # The held state against the step before it: one may be P s + S over a range of steps where the other is the
    # steps in turn.  All of a sequence's terms are at most B = max(|h0|, |x|) here (0 <= f <= 1), two per step, each
    # taken as wrong by delta (see above): after 5 steps either is within 5 * 2 delta B of the exact state.
    B = max(float(h0[1].abs().max()), float(x[:5, 1].float().abs().max()))
    delta = (float(gate[:5, 1].float().abs().max()) + 24) * U
    assert (last[1] - h[4, 1].float()).abs().max() <= 2 * 5 * 2 * delta * B + HALF[typ] * B
    # a gradient that is not finite after the end does not reach the steps up to it
    dirty = dout.clone()
    dirty[7, 0] = float("nan")
    a = scan_backward(gate, x, clean[0], dout=dout, dh_last=dlast, done=done, lens=lens, h0=h0)
    b = scan_backward(dirty_gate[:, 1:].contiguous(), dirty_x[:, 1:].contiguous(), clean[0][:, 1:].contiguous(),
                      dout=dout[:, 1:].contiguous(), dh_last=dlast[1:], done=dirty_done[:, 1:].contiguous(), lens=lens[1:], h0=h0[1:])
    for p, q in zip(a[:2], b[:2]):
        assert torch.equal(p[:, 1:], q) and torch.isfinite(q).all() and (q[5:, 0] == 0).all() and (q[:, 1] == 0).all()
    d = scan_backward(gate, x, clean[0], dout=dirty, dh_last=dlast, done=done, lens=lens, h0=h0)
    for p, q in zip(a, d):
        assert torch.equal(p[:5], q[:5])
    assert torch.isnan(d[1][5:8, 0]).all() and torch.equal(d[1][:, 1:], a[1][:, 1:])


@pytest.mark.parametrize("seed", range(6))
def test_scan_drawn(seed):
    """Sizes, orders, kinds, types and masks drawn together."""
    require_gpu()
    r = np.random.default_rng(seed)
    log = lambda lo, hi: int(round(np.exp(r.uniform(np.log(lo), np.log(hi)))))  # noqa: E731
    for _ in range(12):
        T, c = log(1, 3000), log(1, 300)
        n = log(1, max(1, min(3000, 600000 // (T * c))))
        typ, kind = str(r.choice(["fp32", "bf16"])), str(r.choice(["sigmoid", "decay"]))
        order, masks = str(r.choice(["tnc", "ntc", "ntc2", "cnt", "nct", "tcn", "odd"])), str(r.choice(["", "h", "d", "l", "dl"]))
        announce(f"scan T={T} n={n} c={c} {typ} {kind} {order} masks '{masks}'")
        check_scan(T, n, c, typ, kind, order, masks, seed=seed)


def test_scan_extreme_gates():
    """Gates that saturate: f and 1 - f reach 0 and 1 without NaN, and a long product of small f that
    underflows is no episode end: an infinite state stays infinite."""
    require_gpu()
    from paper_2512_13359_amd import scan_forward
    z = torch.tensor([-3e38, -200.0, -90.0, 90.0, 200.0, 3e38], device="cuda").repeat(7, 1, 1).contiguous()
    x = torch.full_like(z, 2.0)
    h, last = scan_forward(z, x, h0=torch.ones(1, 6, device="cuda"))
    assert torch.equal(last, torch.tensor([[2.0, 2.0, 2.0, 1.0, 1.0, 1.0]], device="cuda"))
    T = 3000
    a = torch.full((T, 1, 4), 0.25, device="cuda")
    s = torch.full((1, 4), float("inf"), device="cuda")
    h, last = scan_forward(a, torch.ones_like(a), kind="decay", h0=s)
    assert torch.isinf(h).all() and torch.isinf(last).all()


@pytest.mark.parametrize("T", [60, 400, 1500])
@pytest.mark.parametrize("kind", ["sigmoid", "decay"])
@pytest.mark.parametrize("typ", ["fp32", "bf16"])
@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_scan_gates_that_are_not_finite_end_with_their_episode(bad, typ, kind, T):
    """A gate that is NaN or infinite before an episode's end, in the same range of steps or an earlier one,
    changes nothing after it, and one after the end changes no gradient up to it."""
    require_gpu()
    from paper_2512_13359_amd import scan_backward, scan_forward
    n, c = 3, 8
    gate, x, _, _, h0, dout, dlast = scan_inputs(T, n, c, typ, kind, "tnc", "h", 6)
    for end in (T // 3, T // 2, 2 * T // 3):
        done = torch.zeros(T, n, device="cuda")
        done[end, 1] = 1.0
        more = dict(kind=kind, done=done, h0=h0)
        h, last = scan_forward(gate, x, **more)
        clean = scan_backward(gate, x, h, dout=dout, dh_last=dlast, **more)
        for at in {max(end - k, 0) for k in (0, 1, 9, 40, 70, 150, T)}:
            dirty = gate.clone()
            dirty[at, 1] = float(bad)
            h2, last2 = scan_forward(dirty, x, **more)
            assert torch.equal(last, last2) and torch.equal(h[end + 1:], h2[end + 1:]) and torch.equal(h[:, ::2], h2[:, ::2])
        for at in {min(end + k, T - 1) for k in (1, 9, 40, 70, 150, T)}:
            dirty = gate.clone()
            dirty[at, 1] = float(bad)
            got = scan_backward(dirty, x, h, dout=dout, dh_last=dlast, **more)
            for p, q in zip(clean[:2], got[:2]):
                assert torch.equal(p[:end + 1], q[:end + 1]) and torch.equal(p[:, ::2], q[:, ::2])
            assert torch.equal(clean[2], got[2])


@pytest.mark.parametrize("T", [200, 1500])
@pytest.mark.parametrize("typ", ["fp32", "bf16"])
def test_scan_large_decays_of_an_empty_state(typ, T):
    """Decays whose product over many steps is beyond fp32 while the state, or the gradient, is zero: it stays zero."""
    require_gpu()
    from paper_2512_13359_amd import scan_backward, scan_forward
    n, c, lo, hi = 2, 8, T // 4, 3 * T // 4
    gate, x, _, _, _, dout, _ = scan_inputs(T, n, c, typ, "decay", "tnc", "", 7)
    gate.fill_(0.5)
    gate[lo:hi] = 100.0
    x[:hi] = 0.0
    dout[lo:] = 0.0
    h, last = scan_forward(gate, x, kind="decay")
    delta = np.full(x.shape, 24 * U)
    wh, wl, bh, bl = L.scan(f64(gate), f64(x), kind="decay", delta=delta)
    r = HALF[typ]
    within(h, wh, bh + r * (np.abs(wh) + bh), "h")
    within(last, wl, bl + U * np.abs(wl), "last")
    dgate, dx, dh0 = scan_backward(gate, x, h, dout=dout, kind="decay")
    wg, wx, w0, bg, bx, b0 = L.scan_grad(f64(gate), f64(x), f64(h), f64(dout), None, kind="decay", delta=delta)
    within(dgate, wg, bg + r * (np.abs(wg) + bg), "dgate")
    within(dx, wx, bx + r * (np.abs(wx) + bx), "dx")
    within(dh0, w0, b0 + U * np.abs(w0), "dh0")


def test_scan_broadcast_inputs_and_absent_gradients():
    """One decay for all sequences and steps (strides of zero); dout or dh_last absent stands for zero."""
    require_gpu()
    from paper_2512_13359_amd import scan_backward, scan_forward
    T, n, c = 50, 7, 24
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    a = torch.rand(c, generator=g, device="cuda")
    x, dout, dlast = (torch.randn(s, generator=g, device="cuda") for s in ((T, n, c), (T, n, c), (n, c)))
    wide = a.expand(T, n, c)
    h, last = scan_forward(wide, x, kind="decay")
    h2, last2 = scan_forward(wide.contiguous(), x, kind="decay")
    assert torch.equal(h, h2) and torch.equal(last, last2)
    zero, zs = torch.zeros_like(dout), torch.zeros_like(dlast)
    for kw in (dict(dout=dout), dict(dh_last=dlast), {}):
        p = scan_backward(wide, x, h, kind="decay", **kw)
        q = scan_backward(wide.contiguous(), x, h, kind="decay", **{"dout": zero, "dh_last": zs, **kw})
        for u, v in zip(p, q):
            assert torch.equal(u, v)
    one = scan_forward(x[:1].expand(T, n, c), x, kind="decay")[0]       # stride zero over the steps
    assert torch.equal(one, scan_forward(x[:1].expand(T, n, c).contiguous(), x, kind="decay")[0])


def test_scan_rows_far_apart():
    """Sequences further apart than 32 bits of bytes, next to ones that are not."""
    require_gpu()
    from paper_2512_13359_amd import scan_backward, scan_forward
    T, n, c, far = 40, 3, 24, 1_200_000_000
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    gate, x, dout = (torch.randn(T, n, c, generator=g, device="cuda").bfloat16() for _ in range(3))
    room = torch.empty(n * far, dtype=torch.bfloat16, device="cuda")
    wide = room.as_strided((T, n, c), (c, far, 1))
    wide.copy_(x)
    h, last = scan_forward(gate, x)
    dgate, dx, dh0 = scan_backward(gate, x, h, dout=dout)
    a = scan_forward(gate, wide, out=torch.empty_like(h))
    b = scan_backward(gate, wide, h, dout=dout, out=(torch.empty_like(dgate), torch.empty_like(dx)))
    within(a[0], f64(h), 2.0 ** -7 * np.abs(f64(h)), "h")      # one step of bf16 where the launch's shape adds in another order
    within(a[1], f64(last), 2.0 ** -16 * (1 + np.abs(f64(last))), "last")
    for p, q, what in zip(b, (dgate, dx, dh0), ("dgate", "dx", "dh0")):
        within(p, f64(q), 2.0 ** -7 * np.abs(f64(q)) + 2.0 ** -16, what)
    out = room.as_strided((T, n, c), (c, far, 1), 7 * c * T)   # and an output there
    assert torch.equal(scan_forward(gate, wide, out=out)[0], a[0])


def test_scan_steps_in_place():
    """A controller's single steps: the state updated in place by every call, one captured step replayed."""
    require_gpu()
    from paper_2512_13359_amd import _abi as A
    T, n, c = 12, 256, 64
    gate, x, done, _, h0, _, _ = scan_inputs(T, n, c, "bf16", "sigmoid", "tnc", "d", 4)
    delta = (np.abs(f64(gate)) + 24) * U
    wh, wl, bh, bl = L.scan(f64(gate), f64(x), done=host(done), h0=f64(h0), delta=delta)
    z, v, d, out, s = gate[0].clone(), x[0].clone(), done[0].clone(), torch.empty_like(x[0]), h0.clone()
    step = A.AuvScan(1, n, c, A.AUV_BF16, A.AUV_SCAN_SIGMOID, z.data_ptr(), n * c, c, 1, v.data_ptr(), n * c, c, 1,
                     out.data_ptr(), n * c, c, 1, d.data_ptr(), None, s.data_ptr(), c, 1, s.data_ptr(), c, 1)
    assert A.auv_scan_work_bytes(step) == 0
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.auv_scan_forward(step, None)
    hs = []
    for t in range(T):
        z.copy_(gate[t]), v.copy_(x[t]), d.copy_(done[t])
        graph.replay()
        hs.append(out.clone())
    within(torch.stack(hs), wh, bh + HALF["bf16"] * (np.abs(wh) + bh), "h")
    within(s, wl, bl + U * np.abs(wl), "state")


# ---------------------------------------------------------------------------- norm --

def norm_bounds(x, groups, mean, rstd, w, b, act, factor, positions):
    """u, its error bound, the slope's, and what they are made of, for statistics taken as exact."""
    n, s, c = x.shape
    per = lambda q: np.repeat(q, c // groups, axis=1)[:, None, :]  # noqa: E731
    v = x if factor is None else np.where(factor == 0, 0.0, x * factor)
    xh = (v - per(mean)) * per(rstd)
    exh = per(rstd) * 3 * U * (np.abs(v) + np.abs(per(mean))) + 2 * U * np.abs(xh)
    return v, xh, exh


def check_norm(n, s, c, groups, typ, act, drop=0, pitch=0, affine=True, seed=0, shift=0.3):
    from paper_2512_13359_amd import make_drop, norm_backward, norm_forward
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    shape = (n, s, c) if s > 1 else (n, c)
    t = lambda: torch.randn((*shape[:-1], c + pitch), generator=g, device="cuda")  # noqa: E731
    x, dout = (t() * 1.5 + shift).to(TYPES[typ])[..., :c], t().to(TYPES[typ])[..., :c]
    w = torch.randn(c, generator=g, device="cuda") if affine else None
    b = torch.randn(c, generator=g, device="cuda") * 0.1 if affine else None
    d = make_drop(drop / 65536, 0xABCDEF0123456789, 11, 4, 100) if drop else None
    factor = L.drop_factor(n * s, c, drop, 0xABCDEF0123456789, 11, 4, 100).reshape(n, s, c) if drop else None
    y, mean, rstd = norm_forward(x, groups, weight=w, bias=b, eps=1e-5, act=act, drop=d)
    dx, dw, db = norm_backward(x, groups, mean, rstd, dout, weight=w, bias=b, act=act, drop=d)
    X, DY, W, B = f64(x).reshape(n, s, c), f64(dout).reshape(n, s, c), f64(w), f64(b)
    wy, wm, wr = L.norm(X, groups, W, B, 1e-5, act, factor)
    half, D = HALF[typ], 64 + s
    ab = lambda q: 0.0 if q is None else np.abs(q)  # noqa: E731
    per = lambda q: np.repeat(q, c // groups, axis=1)[:, None, :]  # noqa: E731
    avg = lambda q: q.reshape(n, s, groups, -1).mean(axis=(1, 3))  # noqa: E731
    v, xh, exh = norm_bounds(X, groups, wm, wr, W, B, act, factor, s)
    em = D * U * avg(np.abs(v)) + U * np.abs(wm)
    within(mean, wm, em, "mean")
    # the sum of squares about a mean that is wrong by em, and about shifts that are members of the set (4 D u)
    er = wr * (4 * D * U + (em * wr) ** 2 + 4 * U)
    within(rstd, wr, er, "rstd")
    exh = exh + per(em * wr) + np.abs(xh) * per(er / wr)
    aw = 1.0 if W is None else np.abs(W)
    u = xh * (1.0 if W is None else W) + (0.0 if B is None else B)
    eu = aw * exh + 2 * U * (np.abs(xh) * aw + ab(B))
    ey = 1.2 * eu + (np.abs(u) + 24) * U * np.abs(wy)      # slopes reach 1.1 (silu) at most
    within(y.reshape(n, s, c), wy, ey + half * (np.abs(wy) + ey), "y")

    M, R = f64(mean), f64(rstd)
    gx, gw, gb = L.norm_grad(X, groups, M, R, DY, W, B, act, factor)
    v, xh, exh = norm_bounds(X, groups, M, R, W, B, act, factor, s)
    u = xh * (1.0 if W is None else W) + (0.0 if B is None else B)
    eu = aw * exh + 2 * U * (np.abs(xh) * aw + ab(B))
    slope = np.abs(L._act(act, u)[1])
    es = 1.0 * eu + (2 * np.abs(u) + 24) * U * slope + (act == "silu") * 24 * U * (1 + np.abs(u)) * slope
    if act == "relu":
        es = (np.abs(u) <= eu).astype(float)               # the slope itself where u may have either sign
    edu = np.abs(DY) * (es + U * slope)
    du = np.abs(DY) * slope
    d_, ed = du * aw, (edu + U * du) * aw
    e1 = per(avg(ed) + D * U * avg(d_))
    e2 = per(avg(ed * np.abs(xh) + d_ * exh) + D * U * avg(d_ * np.abs(xh)))
    m1, m2 = per(avg(d_)), per(avg(d_ * np.abs(xh)))
    ex = per(R) * (ed + e1 + np.abs(xh) * e2 + exh * (m2 + e2) + 4 * U * (d_ + m1 + np.abs(xh) * m2))
    if factor is not None:
        ex = ex * factor
    within(dx.reshape(n, s, c), gx, ex + half * (np.abs(gx) + ex), "dx")
    if affine:
        Dp = 64 + n * s
        within(dw, gw, (edu * np.abs(xh) + du * exh + Dp * U * du * np.abs(xh)).sum((0, 1)), "dw")
        within(db, gb, (edu + Dp * U * du).sum((0, 1)), "db")
    else:
        assert dw is None and db is None


@pytest.mark.parametrize("act", ["none", "relu", "silu", "tanh"])
@pytest.mark.parametrize("typ", ["fp32", "bf16"])
@pytest.mark.parametrize("n, c", [(1, 8), (7, 1), (300, 3), (33, 17), (1000, 256), (65, 511), (9, 1000), (5, 1024), (4, 1025), (3, 2500)])
def test_norm_rows(n, c, typ, act):
    require_gpu()
    announce(f"norm rows n={n} c={c} {typ} {act}")
    check_norm(n, 1, c, 1, typ, act, seed=c)
    check_norm(n, 1, c, 1, typ, act, drop=6554, pitch=5, seed=c + 1)


@pytest.mark.parametrize("typ", ["fp32", "bf16"])
@pytest.mark.parametrize("n, s, c, groups", [(3, 1, 24, 3), (50, 1, 96, 32), (7, 1, 35, 5), (2, 1, 6, 6), (4, 2, 5, 1), (9, 12, 7, 1),
                                             (2, 9, 64, 8), (3, 5, 30, 2), (1, 1001, 90, 6), (5, 77, 3, 3), (2, 300, 257, 1),
                                             (1, 4096, 40, 5), (600, 4, 16, 4), (1, 40, 1300, 13), (2, 3, 2100, 2)])
def test_norm_groups(n, s, c, groups, typ):
    require_gpu()
    announce(f"norm groups n={n} s={s} c={c} g={groups} {typ}")
    check_norm(n, s, c, groups, typ, "silu", seed=c)
    check_norm(n, s, c, groups, typ, "none", drop=20000, pitch=3, affine=False, seed=c)


@pytest.mark.parametrize("seed", range(6))
def test_norm_drawn(seed):
    """Sizes, groups, types, activations, dropout and pitches drawn together, all three forms."""
    require_gpu()
    r = np.random.default_rng(100 + seed)
    log = lambda lo, hi: int(round(np.exp(r.uniform(np.log(lo), np.log(hi)))))  # noqa: E731
    for _ in range(12):
        groups = int(r.choice([1, 1, 2, 3, 8, 32]))
        c = groups * log(1, 3000 // groups)
        s = 1 if r.random() < 0.4 else log(2, 4000)
        n = log(1, max(1, min(3000, 600000 // (s * c))))
        typ, act = str(r.choice(["fp32", "bf16"])), str(r.choice(["none", "relu", "silu", "tanh"]))
        drop, pitch, affine = int(r.choice([0, 655, 20000])), int(r.choice([0, 0, 1, 8])), bool(r.random() < 0.8)
        announce(f"norm n={n} s={s} c={c} g={groups} {typ} {act} drop={drop} pitch={pitch} affine={affine}")
        check_norm(n, s, c, groups, typ, act, drop, pitch, affine, seed=seed)


@pytest.mark.parametrize("s, c, groups", [(1, 256, 1), (500, 16, 2)])
def test_norm_far_from_zero(s, c, groups):
    """A mean of 1000 standard deviations costs the statistics no more than its own rounding."""
    require_gpu()
    check_norm(5, s, c, groups, "fp32", "none", shift=1500.0, seed=8)


@pytest.mark.parametrize("n, s, c, groups", [(40, 1, 32, 1), (3, 5, 24, 3), (2, 3000, 16, 2)])
def test_norm_weight_or_bias_alone(n, s, c, groups):
    """A parameter that is not given stands for 1 or 0 and has no gradient; the other's is the same."""
    require_gpu()
    from paper_2512_13359_amd import norm_backward, norm_forward
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x, dy = (torch.randn(n, s, c, generator=g, device="cuda") for _ in range(2))
    p, one, zero = torch.randn(c, generator=g, device="cuda"), torch.ones(c, device="cuda"), torch.zeros(c, device="cuda")
    for alone, both in ((dict(weight=p), dict(weight=p, bias=zero)), (dict(bias=p), dict(weight=one, bias=p)), ({}, dict(weight=one, bias=zero))):
        y, mean, rstd = norm_forward(x, groups, act="silu", **alone)
        y2, _, _ = norm_forward(x, groups, act="silu", **both)
        assert torch.equal(y, y2)
        a = norm_backward(x, groups, mean, rstd, dy, act="silu", **alone)
        b = norm_backward(x, groups, mean, rstd, dy, act="silu", **both)
        assert torch.equal(a[0], b[0])
        for k, name in ((1, "weight"), (2, "bias")):
            assert torch.equal(a[k], b[k]) if name in alone else a[k] is None


def test_norm_statistics_of_constant_and_empty_groups():
    """A group of one value has variance zero, and so has one whose every element is dropped."""
    require_gpu()
    from paper_2512_13359_amd import make_drop, norm_backward, norm_forward
    for s in (1, 2000):
        x = torch.full((2, s, 16), 3.25, device="cuda")
        y, mean, rstd = norm_forward(x, 2, eps=1e-4)
        assert (y == 0).all() and (mean == 3.25).all() and (rstd - 100).abs().max() <= 100 * 8 * U
        d = make_drop(65535 / 65536, 1)
        x[:, 0] = float("nan")         # dropped places may hold anything
        keep = L.drop_factor(2 * s, 16, 65535, 1).reshape(2, s, 16) != 0
        y, mean, rstd = norm_forward(x, 2, eps=1e-4, drop=d)
        dx, _, _ = norm_backward(x, 2, mean, rstd, torch.ones_like(x), drop=d)
        if not keep[:, 0].any():
            assert torch.isfinite(y).all() and torch.isfinite(dx).all() and (host(dx)[~keep] == 0).all()


# -------------------------------------------------------------------------- dropout --

@pytest.mark.parametrize("typ", ["fp32", "bf16"])
@pytest.mark.parametrize("n, s, c, pitch", [(1, 1, 1, 0), (5, 1, 7, 3), (64, 1, 8, 0), (3, 4, 257, 7), (1001, 1, 33, 1), (2, 3, 2048, 0)])
def test_dropout(n, s, c, pitch, typ):
    require_gpu()
    from paper_2512_13359_amd import dropout, make_drop
    announce(f"dropout n={n} s={s} c={c} {typ}")
    g = torch.Generator(device="cuda")
    g.manual_seed(c)
    shape = (n, s, c) if s > 1 else (n, c)
    x = torch.randn((*shape[:-1], c + pitch), generator=g, device="cuda").to(TYPES[typ])[..., :c]
    add = torch.randn(shape, generator=g, device="cuda").to(TYPES[typ])
    for p in (0.0, 0.1, 0.5, 0.9):
        d = make_drop(p, 0x1122334455667788, 3, 9, 50)
        factor = L.drop_factor(n * s, c, d.drop, 0x1122334455667788, 3, 9, 50).reshape(shape)
        want = f64(x) * factor
        within(dropout(x, d), want, (2 * U + HALF[typ]) * np.abs(want), "dropout")
        both = want + f64(add)
        b = 2 * U * (np.abs(want) + np.abs(both))
        within(dropout(x, d, add), both, b + HALF[typ] * (np.abs(both) + b), "dropout + add")
        mine = x.clone()
        assert torch.equal(dropout(mine, d, out=mine), dropout(x, d))           # in place
        acc = add.clone()
        assert torch.equal(dropout(x, d, acc, out=acc), dropout(x, d, add))
    bad = x.clone()
    d = make_drop(0.5, 2)
    gone = torch.from_numpy(L.drop_factor(n * s, c, d.drop, 2).reshape(shape) == 0).cuda()
    bad[gone] = float("nan")
    assert (dropout(bad, d)[gone] == 0).all()
    half = n // 2                                                               # a batch in two parts
    if half:
        a, b = dropout(x[:half], make_drop(0.5, 2)), dropout(x[half:], make_drop(0.5, 2, row0=half * s))
        assert torch.equal(torch.cat([a, b]), dropout(x, d))


# ------------------------------------------------------------------ together, as used --

def block(feat, done, P, seed, T, n, c, dlast):
    """A critic's block with a memory: linear, dropout, layer norm and ReLU, linear, recurrence cut at the episodes'
    ends; and its gradient.  Returns every result."""
    from paper_2512_13359_amd import make_drop, norm_backward, norm_forward, scan_backward, scan_forward
    drop = make_drop(0.1, seed, step=2, site=1)
    a = feat @ P["W1"]
    y, mean, rstd = norm_forward(a, 1, weight=P["w"], bias=P["b"], act="tanh", drop=drop)
    both = (y @ P["W2"]).view(T, n, 2 * c)
    gate, x = both[..., :c], both[..., c:]
    h, last = scan_forward(gate, x, done=done)
    dboth = torch.empty_like(both)
    scan_backward(gate, x, h, dout=h, dh_last=dlast, done=done, out=(dboth[..., :c], dboth[..., c:]))
    dy = dboth.view(T * n, 2 * c) @ P["W2t"]
    da, dw, db = norm_backward(a, 1, mean, rstd, dy, weight=P["w"], bias=P["b"], act="tanh", drop=drop)
    return dict(y=y, h=h, last=last, dboth=dboth, da=da, dw=dw, db=db)


def block_setup(T, n, c):
    import workloads as W
    from tests.gpu_util import gpu_env
    env = gpu_env(W.config("c2", n_envs=n, episode_len=max(2, T // 3)))
    env.reset()
    bufs = env.rollout_buffers(T, record=("obs", "done"))
    env.rollout(T, W.MODE_RANDOM, bufs=bufs)
    feat = bufs["obs"].permute(1, 2, 0).reshape(T * n, 23).contiguous()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    P = dict(W1=r(23, 64) / 5, w=1 + r(64) / 10, b=r(64) / 10, W2=r(64, 2 * c) / 8)
    P["W2t"] = P["W2"].t().contiguous()
    return feat, bufs["done"], P, r(n, c)


def test_block_on_a_rollout():
    """The layers one after the other on a recorded rollout, against float64 autograd."""
    require_gpu()
    T, n, c = 40, 50, 33
    feat, done, P, dlast = block_setup(T, n, c)
    got = block(feat, done, P, 77, T, n, c, dlast)
    assert 0 < host(done).sum() < T * n
    q = {k: v.double() for k, v in P.items()}
    a = (feat.double() @ q["W1"]).requires_grad_()
    w, b = q["w"].requires_grad_(), q["b"].requires_grad_()
    f = torch.from_numpy(L.drop_factor(T * n, 64, 6554, 77, 2, 1)).cuda()
    y = torch.tanh(torch.nn.functional.layer_norm(a * f, (64,), w, b, 1e-5))
    both = (y @ q["W2"]).view(T, n, 2 * c)
    both.retain_grad()
    s, hs = torch.zeros(n, c, dtype=torch.float64, device="cuda"), []
    for t in range(T):
        z = torch.sigmoid(both[t, :, :c])
        h = z * s + (1 - z) * both[t, :, c:]
        hs.append(h)
        s = h * (1 - done[t].double())[:, None]
    h = torch.stack(hs)
    (0.5 * (h * h).sum() + (s * dlast).sum()).backward()
    want = dict(y=y, h=h, last=s, dboth=both.grad, da=a.grad, dw=w.grad, db=b.grad)
    for k, v in want.items():
        v = v.detach()
        # fp32 throughout: products over 64 and 66 terms, 40 steps, sums over 2000 rows: some hundred roundings in a row
        # at most in any value, each 2^-24 of the terms' size
        err = (got[k].double() - v).abs().max() / v.abs().max()
        assert err <= 1000 * U, (k, float(err))


def test_block_captured_replayed_and_on_another_stream():
    """The same bits from a graph, replayed with eager work between, and from another stream."""
    require_gpu()
    T, n, c = 24, 65, 17
    feat, done, P, dlast = block_setup(T, n, c)
    want = {k: v.clone() for k, v in block(feat, done, P, 5, T, n, c, dlast).items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = block(feat, done, P, 5, T, n, c, dlast)
    torch.cuda.synchronize()
    for k, v in want.items():
        assert torch.equal(other[k], v), k
    f = feat.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block(f, done, P, 5, T, n, c, dlast)
    for rep in range(4):
        f.copy_(feat if rep % 2 == 0 else feat.flip(0))
        graph.replay()
        torch.cuda.synchronize()
        eager = block(f, done, P, 5, T, n, c, dlast)
        for k, v in eager.items():
            assert torch.equal(out[k], v), (rep, k)
    for k, v in want.items():
        assert rep % 2 == 1 or torch.equal(out[k], v), k


def test_stream_argument_and_two_streams_at_once():
    """Calls on two streams at once with a workspace each (long sequences split over workgroups)."""
    require_gpu()
    from paper_2512_13359_amd import norm_forward, scan_forward
    gate, x, done, _, h0, _, _ = scan_inputs(4000, 2, 24, "bf16", "sigmoid", "tnc", "d", 9)
    want = scan_forward(gate, x, done=done, h0=h0)
    wide = torch.randn(2, 3000, 24, device="cuda")
    wn = norm_forward(wide, 3)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = []
    for k in range(6):
        s = streams[k % 2]
        outs.append((scan_forward(gate, x, done=done, h0=h0, stream=s), norm_forward(wide, 3, stream=s)))
    torch.cuda.synchronize()
    for a, b in outs:
        assert all(torch.equal(p, q) for p, q in zip(a, want)) and all(torch.equal(p, q) for p, q in zip(b, wn))


def test_offsets_beyond_32_bits():
    """Tensors of more than 2^31 elements: their ends equal the same calls on the ends alone."""
    require_gpu()
    from paper_2512_13359_amd import dropout, make_drop, norm_backward, norm_forward, scan_backward, scan_forward
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    rand = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda").normal_(generator=g)  # noqa: E731
    T, n, c, tail = 33000, 1024, 64, 10
    announce("scan of 2.2e9 elements")
    gate, x = rand(T, n, c), rand(T, n, c)
    done = torch.zeros(T, n, device="cuda")
    done[T - tail - 1] = 1.0                    # the last steps are an episode of their own
    assert gate.numel() > 2 ** 31
    h, last = scan_forward(gate, x, done=done)
    zt, xt = gate[-tail:], x[-tail:]
    delta = (np.abs(f64(zt)) + 24) * U
    wh, wl, bh, bl = L.scan(f64(zt), f64(xt), delta=delta)
    within(h[-tail:], wh, bh + HALF["bf16"] * (np.abs(wh) + bh), "h")
    within(last, wl, bl + U * np.abs(wl), "last")
    dgate, dx, _ = scan_backward(gate, x, h, dout=x, done=done)
    wg, wx, _, bg, bx, _ = L.scan_grad(f64(zt), f64(xt), f64(h[-tail:]), f64(xt), None, delta=delta)
    within(dgate[-tail:], wg, bg + HALF["bf16"] * (np.abs(wg) + bg), "dgate")
    within(dx[-tail:], wx, bx + HALF["bf16"] * (np.abs(wx) + bx), "dx")
    del h, dgate, dx, gate
    announce("norm and dropout of 2.2e9 elements")
    for shape in ((T * 128, 512), (2, T * 32, 1024)):       # the rows form, the chunk form (two samples)
        v = x.view(shape)
        y, mean, rstd = norm_forward(v, 1, act="silu")
        d, _, _ = norm_backward(v, 1, mean, rstd, v, act="silu")
        end = v[-50:] if len(shape) == 2 else v[1:]
        y2, mean2, rstd2 = norm_forward(end, 1, act="silu")
        d2, _, _ = norm_backward(end, 1, mean2, rstd2, end, act="silu")
        # another number of chunks joins the statistics in another order: a few ulps, then one step of bf16
        near = lambda a, b: float((a.float() - b.float()).abs().max()) <= 2.0 ** -7 * float(b.float().abs().max())  # noqa: E731
        assert near(y[-len(end):][..., -40:, :], y2[..., -40:, :]) and near(d[-len(end):][..., -40:, :], d2[..., -40:, :])
        del y, d, y2, d2
    v = x.view(T * 256, 256)
    y = dropout(v, make_drop(0.5, 9))
    assert torch.equal(y[-1000:], dropout(v[-1000:], make_drop(0.5, 9, row0=T * 256 - 1000)))
