"""Network layers over rollouts as functions of torch tensors on the GPU: the gated linear
recurrence, group norm with an activation, dropout from the counter-based generator, each with its
gradient (auv_scan_*, auv_norm_*, auv_dropout).  Argument checks, allocation and marshalling only.

Outputs and workspaces are torch allocations made on the stream that the call runs on: the current
stream of the tensors' device, or `stream`.  Nothing is kept between calls, so calls may be captured
into a graph; a captured dropout draws the same elements at every replay unless make_drop's counter
tells the replays apart.  The functions are not part of torch's autograd: gradients come from the
*_backward functions, and a tensor that requires grad is refused where torch records (call under
torch.no_grad(), or from a torch.autograd.Function, whose forward and backward do not record).  Wrong
arguments raise AuvError before anything is enqueued."""
from __future__ import annotations

import struct

import torch

from . import _abi as A

TYPES = {torch.float32: A.AUV_FP32, torch.bfloat16: A.AUV_BF16}
KINDS = {"sigmoid": A.AUV_SCAN_SIGMOID, "decay": A.AUV_SCAN_DECAY}
ACTS = {"none": A.AUV_ACTIVATION_NONE, "relu": A.AUV_ACTIVATION_RELU, "silu": A.AUV_ACTIVATION_SILU,
        "tanh": A.AUV_ACTIVATION_TANH}

# The larger structures packed at once, in half the time of setting their fields one by one; _NONE
# stands for a tensor that is not given.
_SCAN, _SCAN_GRAD, _NORM = struct.Struct("@5i4x4q4q4q2q3q3q"), struct.Struct("@4q3q4q4q3q"), struct.Struct("@6if4x3q5q")
_NONE = (0, 0, 0)


def _refuse(fn: str, msg: str):
    raise A.AuvError(A.AUV_EINVAL, f"{fn}: {msg}")


def _one_of(fn, what, choices, v):
    if v not in choices:
        _refuse(fn, f"{what} must be one of {', '.join(map(str, choices))}, got {v}")
    return choices[v]


def _like(fn, name, t, shape, dtype, index, contiguous=False):
    """Checks a tensor; index: its device's."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == index and (not contiguous or t.is_contiguous()):
        return
    if t.dtype is not dtype or t.shape != shape:
        _refuse(fn, f"{name} must be {dtype} of shape {tuple(shape)}, got {t.dtype} of {tuple(t.shape)}")
    if t.get_device() != index:
        _refuse(fn, f"{name} is on another device than x: {t.device}")
    _refuse(fn, f"{name} must be contiguous")


def _unrecorded(fn, *tensors):
    """Results are cut from torch's graph: refused where a gradient would be lost by it."""
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                _refuse(fn, "a tensor requires grad and the result would not: call under torch.no_grad(), gradients come from "
                            "the *_backward functions")


def _drop_here(fn, drop, x):
    if not isinstance(drop, A.AuvDrop):
        _refuse(fn, f"drop must be one of make_drop, got {type(drop).__name__}")
    if drop.tensor is not None and drop.tensor.get_device() != x.get_device():
        _refuse(fn, f"drop's counter is on another device than x: {drop.tensor.device}")


def _here(fn, x, stream) -> bool:
    """Whether x's device is the current one and the stream its current stream."""
    index = x.get_device()
    if index < 0:
        _refuse(fn, f"tensors must be on a GPU, x is on {x.device}")
    if stream is not None:
        if stream.device.index != index:    # entering it would make its device the current one
            _refuse(fn, f"the stream is {stream.device}'s, x is on {x.device}")
        return False
    return index == torch.cuda.current_device()


def _packed(fn, kind, layout, *words):
    try:
        return kind.from_buffer_copy(layout.pack(*words))
    except (struct.error, OverflowError) as e:
        _refuse(fn, f"a size, stride or number is out of range: {e}")


class _Moved:
    """Makes x's device and the stream current: the call inside allocates and launches there."""

    def __init__(self, x, stream):
        self.scopes = (torch.cuda.device(x.device), torch.cuda.stream(stream))

    def __enter__(self):
        for s in self.scopes:
            s.__enter__()

    def __exit__(self, *e):
        for s in reversed(self.scopes):
            s.__exit__(*e)


def _work(n: int, x) -> torch.Tensor | None:
    return torch.empty(n, dtype=torch.uint8, device=x.device) if n else None


# ---- gated linear recurrence ---------------------------------------------------------

def _scan(fn, gate, x, kind, done, lens, h0):
    """The structure's first words and its inputs' addresses and strides."""
    shape, dtype, dev = x.shape, x.dtype, x.get_device()
    if len(shape) != 3 or dtype not in TYPES:
        _refuse(fn, f"x must be a float32 or bfloat16 tensor [T][n][c], got {dtype} of {tuple(shape)}")
    T, n, c = shape
    _like(fn, "gate", gate, shape, dtype, dev)
    if done is not None:
        _like(fn, "done", done, (T, n), torch.float32, dev, True)
    if lens is not None:
        _like(fn, "lens", lens, (n,), torch.int32, dev, True)
    if h0 is not None:
        _like(fn, "h0", h0, (n, c), torch.float32, dev)
    return (T, n, c, TYPES[dtype], _one_of(fn, "kind", KINDS, kind), gate.data_ptr(), *gate.stride(), x.data_ptr(), *x.stride())


def _at(t):
    """Address and strides of a tensor, of a state that may be absent."""
    return _NONE if t is None else (t.data_ptr(), *t.stride())


def _masks(done, lens, h0):
    return (0 if done is None else done.data_ptr(), 0 if lens is None else lens.data_ptr(), *_at(h0))


def scan_forward(gate, x, *, kind="sigmoid", done=None, lens=None, h0=None, out=None, stream=None):
    """Gated linear recurrence over the steps of a rollout; returns (h, last).

    gate, x: [T][n][c], float32 or bfloat16, in any memory order.  With s_{-1} = h0 (zero if None):
      kind "sigmoid": f = sigma(gate), h_t = f s_{t-1} + (1 - f) x_t
      kind "decay":   f = gate,        h_t = f s_{t-1} + x_t
    and s_t = 0 where done [T][n] (float32, contiguous, as a rollout records it) is nonzero, else h_t.
    lens [n] (int32): from a sequence's length on the state is held, h_t = s_t = s_{t-1}.
    h has x's type and memory order, or is `out`; last = s_{T-1} and h0 are float32 [n][c].  One step
    (T = 1) is the form for a controller: pass `last` back as the next h0."""
    fn = "scan_forward"
    _unrecorded(fn, gate, x, h0, out)
    head = _scan(fn, gate, x, kind, done, lens, h0)
    if out is not None:
        _like(fn, "out", out, x.shape, x.dtype, x.get_device())
    if not _here(fn, x, stream):
        with _Moved(x, stream):
            return scan_forward(gate, x, kind=kind, done=done, lens=lens, h0=h0, out=out)
    h = torch.empty_like(x) if out is None else out
    last = torch.empty(x.shape[1:], dtype=torch.float32, device=x.device) if h0 is None else torch.empty_like(h0)
    d = _packed(fn, A.AuvScan, _SCAN, *head, *_at(h), *_masks(done, lens, h0), *_at(last))
    A.auv_scan_forward(d, _work(A.auv_scan_work_bytes(d) if x.shape[0] >= A.AUV_SCAN_SPLIT_STEPS else 0, x))
    return h, last


def scan_backward(gate, x, h, *, dout=None, dh_last=None, kind="sigmoid", done=None, lens=None, h0=None, out=None,
                  stream=None):
    """Gradients (dgate, dx, dh0) of scan_forward from those of its results, dout (of h) and dh_last
    (of last); None stands for zero.  h is scan_forward's result, the other arguments its own.  States are
    float32 here too: those of bfloat16 tensors are formed again from the inputs, not read from the rounded h.
    dgate and dx have x's type (zero at held steps), or are the pair `out`: the halves of one
    buffer, say, where gate and x are the halves of one projection.  dh0 is float32 [n][c]."""
    fn = "scan_backward"
    _unrecorded(fn, gate, x, h, dout, dh_last, h0, *(() if out is None else out))
    head = _scan(fn, gate, x, kind, done, lens, h0)
    _like(fn, "h", h, x.shape, x.dtype, x.get_device())
    if dout is not None:
        _like(fn, "dout", dout, x.shape, x.dtype, x.get_device())
    if dh_last is not None:
        _like(fn, "dh_last", dh_last, x.shape[1:], torch.float32, x.get_device())
    if out is not None:
        if len(out) != 2:
            _refuse(fn, "out must be the pair (dgate, dx)")
        for o in out:
            _like(fn, "out", o, x.shape, x.dtype, x.get_device())
    if not _here(fn, x, stream):
        with _Moved(x, stream):
            return scan_backward(gate, x, h, dout=dout, dh_last=dh_last, kind=kind, done=done, lens=lens, h0=h0, out=out)
    dgate, dx = (torch.empty_like(gate), torch.empty_like(x)) if out is None else out
    like = h0 if h0 is not None else dh_last
    dh0 = torch.empty(x.shape[1:], dtype=torch.float32, device=x.device) if like is None else torch.empty_like(like)
    d = _packed(fn, A.AuvScan, _SCAN, *head, *_at(h), *_masks(done, lens, h0), *_NONE)
    g = _packed(fn, A.AuvScanGrad, _SCAN_GRAD, *(_at(dout) if dout is not None else (0, 0, 0, 0)), *_at(dh_last), *_at(dgate),
                *_at(dx), *_at(dh0))
    A.auv_scan_backward(d, g, _work(A.auv_scan_work_bytes(d, g) if x.shape[0] >= A.AUV_SCAN_SPLIT_STEPS else 0, x))
    return dgate, dx, dh0


# ---- group norm and dropout ----------------------------------------------------------

def _sizes(fn, x):
    """(n, s, c) of a channels-last tensor [n][c] or [n][s][c]."""
    shape = x.shape
    if len(shape) not in (2, 3) or x.dtype not in TYPES:
        _refuse(fn, f"x must be a float32 or bfloat16 tensor [n][c] or [n][s][c], got {x.dtype} of {tuple(shape)}")
    return (shape[0], 1, shape[1]) if len(shape) == 2 else shape


def _rows(fn, name, t):
    """Address and strides (sample, position) of a channels-last tensor."""
    st = t.stride()
    if st[-1] != 1 and t.shape[-1] != 1:
        _refuse(fn, f"{name} must have its channels last with stride 1, got strides {st}")
    return (t.data_ptr(), st[0], 0 if len(st) == 2 else st[1])


def _fresh(x):
    """A new tensor of x's shape and type whose channels have stride 1."""
    return torch.empty(x.shape, dtype=x.dtype, device=x.device)


def dropout(x, drop, add=None, *, out=None, stream=None):
    """Dropout of x, [n][c] or [n][s][c] with channels last, by the draws of `drop` (make_drop), plus `add` where given.
    No mask is stored: the gradient is dropout of the gradient with the same `drop`.  `out` may be x or
    add itself."""
    fn = "dropout"
    _unrecorded(fn, x, add, out)
    n, s, c = _sizes(fn, x)
    _drop_here(fn, drop, x)
    if add is not None:
        _like(fn, "add", add, x.shape, x.dtype, x.get_device())
    if out is not None:
        _like(fn, "out", out, x.shape, x.dtype, x.get_device())
    if not _here(fn, x, stream):
        with _Moved(x, stream):
            return dropout(x, drop, add, out=out)
    y = _fresh(x) if out is None else out
    A.auv_dropout(drop, TYPES[x.dtype], n, s, c, A.AuvRows(*_rows(fn, "x", x)),
                  None if add is None else A.AuvRows(*_rows(fn, "add", add)), A.AuvRows(*_rows(fn, "out", y)))
    return y


def _norm(fn, x, groups, weight, bias, eps, act, drop):
    """The structure without mean and rstd; the callers hold `drop` while it is in use."""
    n, s, c = _sizes(fn, x)
    if drop is not None:
        _drop_here(fn, drop, x)
    if weight is not None:
        _like(fn, "weight", weight, (c,), torch.float32, x.get_device(), True)
    if bias is not None:
        _like(fn, "bias", bias, (c,), torch.float32, x.get_device(), True)
    return _packed(fn, A.AuvNorm, _NORM, n, s, c, groups, TYPES[x.dtype], _one_of(fn, "act", ACTS, act), eps, *_rows(fn, "x", x),
                   0 if weight is None else weight.data_ptr(), 0 if bias is None else bias.data_ptr(), 0, 0,
                   0 if drop is None else A.address(drop))


def norm_forward(x, groups, *, weight=None, bias=None, eps=1e-5, act="none", drop=None, out=None, stream=None):
    """Group norm with an activation; returns (y, mean, rstd).

    x: [n][c] or [n][s][c], float32 or bfloat16, channels last.  Mean and variance are taken over the s
    positions and c / groups channels of each group of each sample (groups = 1 and no positions: layer
    norm); y = act(weight xhat + bias), weight and bias float32 [c] or None, act one of "none", "relu",
    "silu", "tanh".  With `drop` (make_drop) x is dropped out first, its mask never stored.  mean and
    rstd are float32 [n][groups]; y has x's type, or is `out`."""
    fn = "norm_forward"
    _unrecorded(fn, x, weight, bias, out)
    d = _norm(fn, x, groups, weight, bias, eps, act, drop)
    if out is not None:
        _like(fn, "out", out, x.shape, x.dtype, x.get_device())
    if not _here(fn, x, stream):
        with _Moved(x, stream):
            return norm_forward(x, groups, weight=weight, bias=bias, eps=eps, act=act, drop=drop, out=out)
    work = _work(A.auv_norm_work_bytes(d, False), x)
    y = _fresh(x) if out is None else out
    mean = torch.empty((d.n, groups), dtype=torch.float32, device=x.device)
    rstd = torch.empty_like(mean)
    d.mean, d.rstd = mean.data_ptr(), rstd.data_ptr()
    A.auv_norm_forward(d, A.AuvRows(*_rows(fn, "out", y)), work)
    return y, mean, rstd


def norm_backward(x, groups, mean, rstd, dout, *, weight=None, bias=None, act="none", drop=None, out=None, stream=None):
    """Gradients (dx, dweight, dbias) of norm_forward from that of y; mean and rstd are its results, the
    other arguments its own.  dx has x's type, or is `out`; dweight is None where weight is, dbias
    where bias is, else float32 [c]."""
    fn = "norm_backward"
    _unrecorded(fn, x, mean, rstd, dout, weight, bias, out)
    d = _norm(fn, x, groups, weight, bias, 0.0, act, drop)
    for name, t in (("mean", mean), ("rstd", rstd)):
        _like(fn, name, t, (d.n, groups), torch.float32, x.get_device(), True)
    d.mean, d.rstd = mean.data_ptr(), rstd.data_ptr()
    _like(fn, "dout", dout, x.shape, x.dtype, x.get_device())
    if out is not None:
        _like(fn, "out", out, x.shape, x.dtype, x.get_device())
    if not _here(fn, x, stream):
        with _Moved(x, stream):
            return norm_backward(x, groups, mean, rstd, dout, weight=weight, bias=bias, act=act, drop=drop, out=out)
    work = _work(A.auv_norm_work_bytes(d, True), x)
    dx = _fresh(x) if out is None else out
    dweight = None if weight is None else torch.empty_like(weight)
    dbias = None if bias is None else torch.empty_like(bias)
    A.auv_norm_backward(d, A.AuvNormGrad(*_rows(fn, "dout", dout), *_rows(fn, "out", dx), A.ptr(dweight), A.ptr(dbias)), work)
    return dx, dweight, dbias
