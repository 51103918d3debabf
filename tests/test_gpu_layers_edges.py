"""More GPU parity of the network layers with their float64 oracle: states that follow their input, and other uses where an
error hides behind random numbers.  Tolerances as derived in test_gpu_layers.py."""
import numpy as np
import pytest
import torch

from oracle import layers as L
from tests.gpu_util import announce, host, require_gpu
from tests.test_gpu_layers import HALF, TYPES, U, block, block_setup, check_norm, f64, scan_inputs, seq, within

pytestmark = pytest.mark.gpu


def check_following_state(T, n, c, typ, kind, order, masks):
    """x = 1 + 0.01 noise: the state lies next to its input, and dgate = f (1 - f) (s - x) g is their small difference.
    dgate is compared with the gradient of the recurrence itself; a state rounded to bf16 would leave an error of 2^-9
    beside differences of about 2^-7.  The oracle runs on a few sequences (they are independent)."""
    from paper_2512_13359_amd import scan_backward, scan_forward
    announce(f"scan following T={T} n={n} c={c} {typ} {kind} {order} '{masks}'")
    _, _, done, lens, h0, _, dlast = scan_inputs(T, n, 1, typ, kind, "tnc", masks, T + c)
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    gate, x, dout = seq(g, T, n, c, typ, order, 1.5, 2.2), seq(g, T, n, c, typ, order, 0.01, 1.0), seq(g, T, n, c, typ, order)
    if kind == "decay":
        gate.copy_(torch.sigmoid(gate.float()))
    h0 = None if h0 is None else 1 + 0.01 * torch.randn(n, c, generator=g, device="cuda")
    dlast = dlast.expand(n, c).contiguous()
    more = dict(kind=kind, done=done, lens=lens, h0=h0)
    h, _ = scan_forward(gate, x, **more)
    dgate, dx, dh0 = scan_backward(gate, x, h, dout=dout, dh_last=dlast, **more)
    some = sorted({*range(min(n, 4)), n // 2, *range(max(n - 3, 0), n)})
    pick = lambda t, axis=1: None if t is None else f64(t.index_select(axis, torch.tensor(some, device="cuda")))  # noqa: E731
    delta = (np.abs(pick(gate)) * (kind == "sigmoid") + 24) * U
    m = dict(kind=kind, done=pick(done), lens=None if lens is None else host(lens)[some], h0=pick(h0, 0), delta=delta)
    wg, wx, w0, bg, bx, b0 = L.scan_grad(pick(gate), pick(x), None, pick(dout), pick(dlast, 0), **m)
    r = HALF[typ]
    within(pick_f(dgate, some), wg, bg + r * (np.abs(wg) + bg), "dgate")
    within(pick_f(dx, some), wx, bx + r * (np.abs(wx) + bx), "dx")
    within(dh0[some], w0, b0 + U * np.abs(w0), "dh0")


def pick_f(t, some):
    return t.index_select(1, torch.tensor(some, device=t.device))


@pytest.mark.parametrize("kind", ["sigmoid", "decay"])
@pytest.mark.parametrize("typ", ["fp32", "bf16"])
@pytest.mark.parametrize("T, n, c", [(1, 3, 5), (5, 40, 8), (16, 7, 24), (17, 7, 24), (100, 3, 70), (127, 33, 9), (128, 33, 9), (129, 33, 9),
                                     (512, 6, 64), (4001, 2, 33), (700, 2049, 8), (9, 4100, 64), (127, 4100, 64), (150, 4100, 64), (40, 16500, 5)])
def test_scan_gradient_of_states_that_follow_their_input(T, n, c, typ, kind):
    """Every width of a lane's columns, one workgroup to many, the marks in LDS and in the workspace, split steps."""
    require_gpu()
    check_following_state(T, n, c, typ, kind, "tnc", "dl")


@pytest.mark.parametrize("order", ["tnc", "ntc", "cnt", "nct", "tcn", "odd"])
@pytest.mark.parametrize("masks", ["", "h", "d", "l"])
def test_scan_gradient_of_following_states_by_order(order, masks):
    require_gpu()
    for T, n, c in ((37, 9, 6), (300, 70, 40), (2000, 3, 20)):
        for kind in ("sigmoid", "decay"):
            check_following_state(T, n, c, "bf16", kind, order, masks)


def test_scan_gradient_captured_and_on_two_streams():
    """A bf16 gradient's workspace is the call's own: two streams at once, a graph replayed with eager work between."""
    require_gpu()
    from paper_2512_13359_amd import scan_backward, scan_forward
    T, n, c = 1500, 4, 40
    gate, x, done, _, h0, dout, dlast = scan_inputs(T, n, c, "bf16", "sigmoid", "tnc", "d", 3)
    other = scan_inputs(T, n, c, "bf16", "sigmoid", "tnc", "d", 4)[1]

    def both(x, stream=None):
        h, last = scan_forward(gate, x, done=done, h0=h0, stream=stream)
        return (h, last, *scan_backward(gate, x, h, dout=dout, dh_last=dlast, done=done, h0=h0, stream=stream))

    want = {False: both(x), True: both(other)}
    assert not torch.equal(want[False][2], want[True][2])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [both(other if k % 2 else x, streams[k % 2]) for k in range(6)]
    torch.cuda.synchronize()
    for k, out in enumerate(outs):
        assert all(torch.equal(p, q) for p, q in zip(out, want[k % 2 == 1])), k
    held = x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both(held)
    for rep in range(4):
        held.copy_(other if rep % 2 else x)
        graph.replay()
        both(x)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want[rep % 2 == 1])), rep


@pytest.mark.parametrize("typ", ["fp32", "bf16"])
@pytest.mark.parametrize("n, s, c, groups", [(700, 1, 4104, 1), (500, 1, 4101, 1), (600, 1, 4200, 2), (600, 5, 3000, 3), (800, 30, 272, 8), (40, 1, 40000, 4),
                                             (1100, 1, 2052, 1)])
def test_norm_of_many_samples_that_no_workgroup_holds(n, s, c, groups, typ):
    """Workgroups that walk over several samples and keep the parameters' sums, and the same without parameters."""
    require_gpu()
    announce(f"norm many n={n} s={s} c={c} g={groups} {typ}")
    check_norm(n, s, c, groups, typ, "silu", seed=c)
    check_norm(n, s, c, groups, typ, "tanh", drop=6554, pitch=3, seed=n)
    check_norm(n, s, c, groups, typ, "none", affine=False, seed=s)


def test_norm_of_single_channels_in_wide_rows():
    """As many groups as channels over several tiles: each tile has shares of its own groups."""
    require_gpu()
    check_norm(3, 40, 5000, 5000, "fp32", "tanh", seed=1)
    check_norm(2, 300, 4500, 1500, "bf16", "relu", drop=9000, seed=2)


def test_norm_inside_an_autograd_function():
    """From a torch.autograd.Function, which does not record, the functions take parameters and graph tensors as they are."""
    require_gpu()
    from paper_2512_13359_amd import AuvError, norm_backward, norm_forward

    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, b):
            y, mean, rstd = norm_forward(x, 2, weight=w, bias=b, act="silu")
            ctx.save_for_backward(x, w, b, mean, rstd)
            return y

        @staticmethod
        def backward(ctx, dy):
            x, w, b, mean, rstd = ctx.saved_tensors
            return norm_backward(x, 2, mean, rstd, dy.contiguous(), weight=w, bias=b, act="silu")

    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    x, dy = (torch.randn(50, 48, generator=g, device="cuda") for _ in range(2))
    w, b = (torch.nn.Parameter(torch.randn(48, generator=g, device="cuda")) for _ in range(2))
    x.requires_grad_()
    with pytest.raises(AuvError, match="requires grad"):
        norm_forward(x, 2, weight=w, bias=b, act="silu")
    got = torch.autograd.grad(Norm.apply(x, w, b), (x, w, b), dy)
    X, Wt, B = f64(x.detach()).reshape(50, 1, 48), f64(w.detach()), f64(b.detach())
    _, mean, rstd = L.norm(X, 2, Wt, B, 1e-5, "silu")
    for p, q in zip(got, L.norm_grad(X, 2, mean, rstd, f64(dy).reshape(50, 1, 48), Wt, B, "silu")):
        # sums of 24 and 50 terms and some thirty roundings of each, relative to the largest value
        assert np.abs(f64(p).reshape(q.shape) - q).max() <= 256 * U * np.abs(q).max()


def test_stream_of_another_device_is_refused():
    """It would be entered and left again for the current stream of x's device, on which the call then ran."""
    require_gpu()
    from types import SimpleNamespace

    from paper_2512_13359_amd import AuvError, dropout, make_drop, norm_backward, norm_forward, scan_backward, scan_forward
    other = SimpleNamespace(device=torch.device("cuda", 1))     # all that is looked at
    x = torch.zeros(4, 3, 8, device="cuda")
    stat = torch.zeros(4, 2, device="cuda")
    for f in (lambda **k: scan_forward(x, x, **k), lambda **k: scan_backward(x, x, x, **k), lambda **k: dropout(x, make_drop(0.5, 1), **k),
              lambda **k: norm_forward(x, 2, **k), lambda **k: norm_backward(x, 2, stat, stat, x, **k)):
        with pytest.raises(AuvError, match="stream"):
            f(stream=other)
        f(stream=torch.cuda.Stream())
        f(stream=torch.cuda.current_stream())
    torch.cuda.synchronize()


@pytest.mark.parametrize("n, s, c, groups", [(300, 1, 200, 1), (40, 1, 90, 6), (9, 20, 24, 3), (3, 2500, 20, 2), (300, 1, 4200, 2)])
def test_captured_dropout_draws_by_its_counter(n, s, c, groups):
    """A counter on the device tells the replays of a captured training step apart, in every form of the norm: replay k is the eager
    step k.  Without one every replay draws what the captured call drew."""
    require_gpu()
    from paper_2512_13359_amd import dropout, make_drop, norm_backward, norm_forward
    announce(f"dropout counter n={n} s={s} c={c} g={groups}")
    g = torch.Generator(device="cuda")
    g.manual_seed(c)
    x, dy = (torch.randn(n, s, c, generator=g, device="cuda") for _ in range(2))
    w, b = torch.randn(c, generator=g, device="cuda"), torch.randn(c, generator=g, device="cuda")

    def step(**at):
        d = make_drop(0.3, 99, site=2, **at)
        v = dropout(x, d, x)
        y, mean, rstd = norm_forward(v, groups, weight=w, bias=b, act="tanh", drop=d)
        return (v, y, mean, rstd, *norm_backward(v, groups, mean, rstd, dy, weight=w, bias=b, act="tanh", drop=d))

    first = 0xFFFFFFFE      # the sum passes 2^32
    eager = [step(step=(first + k) % 2 ** 32) for k in range(5)]
    assert not torch.equal(eager[0][0], eager[1][0]) and not torch.equal(eager[0][1], eager[2][1])
    counter = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph, fixed = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(step=first, counter=counter)
        counter.add_(1)
    with torch.cuda.graph(fixed):
        same = step(step=first)
    for k in range(5):
        graph.replay()
        fixed.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, eager[k])), k
        assert all(torch.equal(p, q) for p, q in zip(same, eager[0])), k
        mine = step(step=first, counter=counter)     # eager, with the counter as it now is
        if k < 4:
            assert all(torch.equal(p, q) for p, q in zip(mine, eager[k + 1])), k


def test_block_replays_equal_the_calls_before_the_capture():
    """Replays against results from before the capture, not only against eager calls beside them; and the refilled input counts."""
    require_gpu()
    T, n, c = 24, 65, 17
    feat, done, P, dlast = block_setup(T, n, c)
    want = {k: v.clone() for k, v in block(feat, done, P, 5, T, n, c, dlast).items()}
    flip = {k: v.clone() for k, v in block(feat.flip(0).contiguous(), done, P, 5, T, n, c, dlast).items()}
    f = feat.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block(f, done, P, 5, T, n, c, dlast)
    for rep in range(5):
        f.copy_(feat.flip(0) if rep % 2 else feat)
        graph.replay()
        block(feat, done, P, 6, T, n, c, dlast)     # the program's own work between
        torch.cuda.synchronize()
        for k, v in (flip if rep % 2 else want).items():
            assert torch.equal(out[k], v), (rep, k)
    # the two differ, but for the last state: episodes of 8 steps all end with step 24
    assert (want["last"] == 0).all() and all(not torch.equal(want[k], flip[k]) for k in want if k != "last")
