"""Performance cases of the network layers: the gated linear recurrence over a rollout, group
norm with an activation, and dropout from the counter-based generator.

    own                  False: `run` computes the operators in elementary torch operations, in
                         32 bits; True: through the framework's entry points
    listed()             the named cases
    draw(rng)            one more case of the same ranges
    prepare(case, seed)  what a program has in hand before the call
    run(state)           one pass, its outputs
    work(case)           bytes and operations that one pass cannot do without
    exact(case, seed)    the outputs of one pass from the operators' definitions in 64 bits

Recurrence over steps t, sequences n and channels c, with the state s (s_{-1} = h0):
    sigmoid: f = sigma(gate), h_t = f s_{t-1} + (1 - f) x_t;  decay: f = gate, h_t = f s_{t-1} + x_t
    s_t = 0 where the episode ended at step t (done), else h_t
    steps from a sequence's length on hold the state: h_t = s_t = s_{t-1}
Norm over the S positions and C / G channels of each group of each sample, then act(w xhat + b),
with dropout in front of it where the case says so.
Dropout of element (row, c): one of eight 16-bit halves of the Philox4x32-10 block with counter
(row, step, 3 | site << 8, c >> 3) and the seed as key; kept where the half is at least 65536 p.
"""
import math

import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "bf16": 2}
STEP, SITE = 7, 2     # update number and layer of the dropout draws


def listed():
    return [
        # one control step of a recurrent controller for 256 vehicles: latency
        dict(name="scan_step_256", op="scan", T=1, N=256, C=256, type="fp32", kind="sigmoid", order="tnc", done=False,
             lens=False, train=False),
        # the features of a 64-step collection run through the recurrence, no gradient
        dict(name="scan_collect_16384", op="scan", T=64, N=16384, C=64, type="bf16", kind="sigmoid", order="tnc",
             done=True, lens=False, train=False),
        # one training iteration of the paper's task: 4096 vehicles, 512-step episodes
        dict(name="scan_train_4096x512", op="scan", T=512, N=4096, C=64, type="bf16", kind="sigmoid", order="tnc",
             done=True, lens=False, train=True),
        # two very long logs, gate and input as the halves of one projection: few sequences, much time
        dict(name="scan_train_long", op="scan", T=32768, N=2, C=256, type="bf16", kind="sigmoid", order="ntc2",
             done=False, lens=False, train=True),
        # an odd batch in the layout of the recorded observations, ragged lengths, given decays
        dict(name="scan_train_ragged_soa", op="scan", T=500, N=4095, C=23, type="fp32", kind="decay", order="cnt",
             done=True, lens=True, train=True),
        # layer norm and ReLU behind a hidden layer of 256, a handful of vehicles: latency
        dict(name="norm_rows_256", op="norm", N=256, S=1, C=256, G=1, type="bf16", act="relu", drop=0.0, train=False),
        # a critic's block (dropout, layer norm, activation) on the minibatch of the PPO update
        dict(name="norm_rows_train_262144", op="norm", N=262144, S=1, C=256, G=1, type="bf16", act="silu", drop=0.01,
             train=True),
        # groups of eight channels over whole feature maps
        dict(name="norm_groups_32x4096", op="norm", N=32, S=4096, C=256, G=32, type="bf16", act="silu", drop=0.0,
             train=False),
        # a small odd batch of feature maps, groups of 15 channels, with dropout
        dict(name="norm_odd_train", op="norm", N=5, S=1001, C=90, G=6, type="fp32", act="tanh", drop=0.1, train=True),
        # dropout of a hidden layer of a handful of vehicles: latency
        dict(name="dropout_256", op="dropout", N=256, S=1, C=256, type="fp32", p=0.1, add=False, pitch=0),
        # dropout into a residual stream, a quarter of the paper's training batch
        dict(name="dropout_residual_524288", op="dropout", N=524288, S=1, C=256, type="bf16", p=0.1, add=True, pitch=0),
        # odd rows inside a wider buffer
        dict(name="dropout_odd_pitched", op="dropout", N=100003, S=1, C=257, type="fp32", p=0.5, add=False, pitch=7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["scan", "scan", "norm", "norm", "dropout"])
    typ = rng.choice(["fp32", "bf16", "bf16"])
    if op == "scan":
        train, order = rng.random() < 0.6, rng.choice(["tnc", "tnc", "ntc2", "cnt"])
        T = 1 if rng.random() < 0.15 else _log(rng, 2, 20000)
        C = _log(rng, 1, 512)
        N = _log(rng, 1, max(2, min(65536, 40000000 // (T * C))))
        return dict(op=op, T=T, N=N, C=C, type=typ, kind=rng.choice(["sigmoid", "sigmoid", "decay"]), order=order,
                    done=rng.random() < 0.6, lens=rng.random() < 0.3, train=train)
    if op == "norm":
        G = rng.choice([1, 1, 2, 3, 8, 32])
        C = G * _log(rng, 1, 1024 // G)
        S = 1 if rng.random() < 0.5 else _log(rng, 2, 8192)
        N = _log(rng, 1, max(2, min(262144, 40000000 // (S * C))))
        if S * C // G < 8:      # a group of a few numbers has no variance to speak of
            S = 8
            N = max(1, N // 8)
        return dict(op=op, N=N, S=S, C=C, G=G, type=typ, act=rng.choice(["none", "tanh", "silu"]),
                    drop=rng.choice([0.0, 0.01, 0.1]), train=rng.random() < 0.6)
    C = _log(rng, 1, 2048)
    return dict(op=op, N=_log(rng, 1, max(2, min(1 << 20, 60000000 // C))), S=1, C=C, type=typ,
                p=rng.choice([0.01, 0.1, 0.5]), add=rng.random() < 0.5, pitch=rng.choice([0, 0, 1, 8, 13]))


# ---------------------------------------------------------------------------- inputs --

def _normal(g, shape, typ, scale=1.0, shift=0.0):
    return torch.randn(shape, generator=g, device=DEV).mul_(scale).add_(shift).to(TYPES[typ])


def _ordered(g, case, scale=1.0, shift=0.0):
    """A logical [T][N][C] tensor in the case's memory order."""
    T, N, C = case["T"], case["N"], case["C"]
    if case["order"] == "cnt":
        return _normal(g, (C, T, N), case["type"], scale, shift).permute(1, 2, 0)
    if case["order"] == "ntc2":
        return _normal(g, (N, T, C), case["type"], scale, shift).permute(1, 0, 2)
    return _normal(g, (T, N, C), case["type"], scale, shift)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    st = dict(case=case)
    if case["op"] == "scan":
        T, N, C, typ = case["T"], case["N"], case["C"], case["type"]
        if case["order"] == "ntc2":     # one projection [N][T][2C], its halves
            both = _normal(g, (N, T, 2 * C), typ)
            both[..., :C] += 2.2
            st["gate"], st["x"] = both[..., :C].permute(1, 0, 2), both[..., C:].permute(1, 0, 2)
        else:
            st["gate"], st["x"] = _ordered(g, case, 1.5, 2.2), _ordered(g, case)
        if case["kind"] == "decay":
            st["gate"].copy_(1.0 - 0.3 * torch.sigmoid(-st["gate"].float()))
        st["done"] = (torch.rand((T, N), generator=g, device=DEV) < 0.01).float() if case["done"] else None
        st["lens"] = torch.randint(0, T + 1, (N,), generator=g, device=DEV, dtype=torch.int32) if case["lens"] else None
        h0 = torch.randn((C, N) if case["order"] == "cnt" else (N, C), generator=g, device=DEV)
        st["h0"] = h0.t() if case["order"] == "cnt" else h0
        if case["train"]:
            st["dout"] = _ordered(g, case)
            dl = torch.randn(h0.shape, generator=g, device=DEV)
            st["dlast"] = dl.t() if case["order"] == "cnt" else dl
        return st
    shape = (case["N"], case["S"], case["C"])
    if case["op"] == "norm":
        st["x"] = _normal(g, shape, case["type"], 1.5, 0.3)
        st["w"] = _normal(g, (case["C"],), "fp32", 0.1, 1.0)
        st["b"] = _normal(g, (case["C"],), "fp32", 0.1)
        if case["train"]:
            st["dout"] = _normal(g, shape, case["type"])
    else:
        wide = _normal(g, shape[:2] + (shape[2] + case["pitch"],), case["type"])
        st["x"] = wide[..., :shape[2]]
        st["add"] = _normal(g, shape, case["type"]) if case["add"] else None
    st["seed"] = int(torch.randint(0, 1 << 62, (1,), generator=g, device=DEV).item())
    return st


# ------------------------------------------------------------------- one pass, either way --

def _halves_plain(rows, C, seed):
    """[rows][C] 16-bit halves of the dropout draws: Philox4x32-10 on 64-bit integers, whose
    products keep their low 64 bits."""
    m = 0xFFFFFFFF
    c0 = torch.arange(rows, dtype=torch.int64, device=DEV)[:, None]
    c3 = torch.arange((C + 7) // 8, dtype=torch.int64, device=DEV)[None, :]
    c1, c2 = torch.full_like(c0, STEP), torch.full_like(c3, 3 | SITE << 8)
    k0, k1 = seed & m, seed >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (p1 >> 32 & m) ^ c1 ^ k0, p1 & m, (p0 >> 32 & m) ^ c3 ^ k1, p0 & m
        k0, k1 = k0 + 0x9E3779B9 & m, k1 + 0xBB67AE85 & m
    words = [w.expand(rows, -1).to(torch.int32) if w.shape[0] == rows else w for w in (c0, c1, c2, c3)]
    return torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16 & 0xFFFF)], 2).reshape(rows, -1)[:, :C]


def _mask_plain(case, p, seed):
    k = round(p * 65536)
    keep = _halves_plain(case["N"] * case["S"], case["C"], seed) >= k
    return keep.reshape(case["N"], case["S"], case["C"]), 65536.0 / (65536 - k)


def _prefix(c, b):
    """h_t = c_t h_{t-1} + b_t along the first axis, by doubling."""
    d, T = 1, b.shape[0]
    while d < T:
        b = torch.cat([b[:d], b[d:] + c[d:] * b[:-d]])
        c = torch.cat([c[:d], c[d:] * c[:-d]])
        d *= 2
    return b


def _scan_plain(st):
    case = st["case"]
    T, sig = case["T"], case["kind"] == "sigmoid"
    z, x = st["gate"].float(), st["x"].float()
    f = 1 / (1 + torch.exp(-z)) if sig else z
    inw = 1 / (1 + torch.exp(z)) if sig else torch.ones_like(z)
    nd = torch.ones((T, case["N"], 1), device=DEV)
    if st["done"] is not None:
        nd = 1 - st["done"][..., None]
    if st["lens"] is not None:
        hold = torch.arange(T, device=DEV)[:, None, None] >= st["lens"][None, :, None]
        one, zero = torch.ones((), device=DEV), torch.zeros((), device=DEV)
        f, inw, nd = torch.where(hold, one, f), torch.where(hold, zero, inw), torch.where(hold, one, nd)
    c = torch.cat([f[:1], f[1:] * nd[:-1]])
    b = inw * x
    b = torch.cat([b[:1] + f[:1] * st["h0"], b[1:]])
    h = _prefix(c, b)
    outs = [h.to(st["x"].dtype), nd[-1] * h[-1]]
    if case["train"]:
        e = st["dout"].float()
        e = torch.cat([e[:-1], e[-1:] + nd[-1:] * st["dlast"]])
        g = _prefix(torch.cat([c[:1], c[1:].flip(0)]), e.flip(0)).flip(0)
        s = torch.cat([st["h0"][None], nd[:-1] * h[:-1]])
        dx = inw * g
        dgate = f * inw * (s - x) * g if sig else s * g
        if st["lens"] is not None:
            dgate, dx = torch.where(hold, zero, dgate), torch.where(hold, zero, dx)
        outs += [dgate.to(st["x"].dtype), dx.to(st["x"].dtype), f[0] * g[0]]
    return outs


def _act_plain(act, u):
    """act(u) and act'(u)."""
    if act == "tanh":
        y = torch.tanh(u)
        return y, 1 - y * y
    if act == "silu":
        s = 1 / (1 + torch.exp(-u))
        return u * s, s * (1 + u * (1 - s))
    if act == "relu":
        return torch.where(u > 0, u, torch.zeros_like(u)), (u > 0).float()
    return u, torch.ones_like(u)


def _norm_plain(st):
    case = st["case"]
    N, S, C, G = case["N"], case["S"], case["C"], case["G"]
    x = st["x"].float()
    if case["drop"]:
        keep, scale = _mask_plain(case, case["drop"], st["seed"])
        x = torch.where(keep, x * scale, torch.zeros_like(x))
    x = x.reshape(N, S, G, C // G)
    w, b = st["w"].reshape(G, -1), st["b"].reshape(G, -1)
    mean = x.mean((1, 3), keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean((1, 3), keepdim=True) + 1e-5)
    xh = (x - mean) * rstd
    y, dact = _act_plain(case["act"], xh * w + b)
    outs = [y.reshape(N, S, C).to(st["x"].dtype), mean.reshape(N, G), rstd.reshape(N, G)]
    if case["train"]:
        du = st["dout"].float().reshape(N, S, G, C // G) * dact
        dxh = du * w
        dx = rstd * (dxh - dxh.mean((1, 3), keepdim=True) - xh * (dxh * xh).mean((1, 3), keepdim=True))
        dx = dx.reshape(N, S, C)
        if case["drop"]:
            dx = torch.where(keep, dx * scale, torch.zeros_like(dx))
        outs += [dx.to(st["x"].dtype), (du * xh).sum((0, 1)).reshape(C), du.sum((0, 1)).reshape(C)]
    return outs


def _dropout_plain(st):
    keep, scale = _mask_plain(st["case"], st["case"]["p"], st["seed"])
    y = torch.where(keep, st["x"].float() * scale, torch.zeros((), device=DEV))
    if st["add"] is not None:
        y = y + st["add"].float()
    return [y.to(st["x"].dtype)]


def _scan_own(st):
    from paper_2512_13359_amd import scan_backward, scan_forward
    more = dict(kind=st["case"]["kind"], done=st["done"], lens=st["lens"], h0=st["h0"])
    h, last = scan_forward(st["gate"], st["x"], **more)
    if not st["case"]["train"]:
        return [h, last]
    return [h, last, *scan_backward(st["gate"], st["x"], h, dout=st["dout"], dh_last=st["dlast"], **more)]


def _norm_own(st):
    from paper_2512_13359_amd import make_drop, norm_backward, norm_forward
    case = st["case"]
    drop = make_drop(case["drop"], st["seed"], step=STEP, site=SITE) if case["drop"] else None
    more = dict(weight=st["w"], bias=st["b"], act=case["act"], drop=drop)
    y, mean, rstd = norm_forward(st["x"], case["G"], eps=1e-5, **more)
    if not case["train"]:
        return [y, mean, rstd]
    return [y, mean, rstd, *norm_backward(st["x"], case["G"], mean, rstd, st["dout"], **more)]


def _dropout_own(st):
    from paper_2512_13359_amd import dropout, make_drop
    return [dropout(st["x"], make_drop(st["case"]["p"], st["seed"], step=STEP, site=SITE), add=st["add"])]


def run(state):
    if own:
        return {"scan": _scan_own, "norm": _norm_own, "dropout": _dropout_own}[state["case"]["op"]](state)
    return {"scan": _scan_plain, "norm": _norm_plain, "dropout": _dropout_plain}[state["case"]["op"]](state)


def work(case):
    e = BYTES[case["type"]]
    if case["op"] == "scan":
        M, state = case["T"] * case["N"] * case["C"], 4 * case["N"] * case["C"]
        side = 4 * case["T"] * case["N"] * case["done"] + 4 * case["N"] * case["lens"]
        # forward: gate, x in, h out; backward: the gradient of h in, those of gate and x out (gate, x and h are
        # read again by any backward pass)
        tensors = 3 + ((6 if case["kind"] == "sigmoid" else 5) if case["train"] else 0)
        return {"bytes": M * e * tensors + 2 * state + side + (3 * state + side if case["train"] else 0),
                "flops": M * (5 + (9 if case["train"] else 0))}
    M = case["N"] * case["S"] * case["C"]
    if case["op"] == "norm":
        small = 8 * case["C"] + 8 * case["N"] * case["G"]
        return {"bytes": M * e * (5 if case["train"] else 2) + small * (3 if case["train"] else 1),
                "flops": M * (10 + (25 if case["train"] else 0))}
    return {"bytes": M * e * (3 if case["add"] else 2), "flops": 2 * M}


# ----------------------------------------------------------------------- 64-bit values --

def _halves_exact(rows, C, seed):
    """The same halves with the 32 x 32 products taken by 16-bit limbs."""
    def product(a, b):      # (high, low) words of a b
        al, ah, bl, bh = a & 0xFFFF, a >> 16, b & 0xFFFF, b >> 16
        mid = ah * bl + (al * bl >> 16)
        mid2 = al * bh + (mid & 0xFFFF)
        return ah * bh + (mid >> 16) + (mid2 >> 16), (mid2 & 0xFFFF) << 16 | (al * bl & 0xFFFF)

    nb = -(-C // 8)
    i = torch.arange(rows * nb, dtype=torch.int64, device=DEV)
    ctr = [torch.div(i, nb, rounding_mode="floor"), torch.full_like(i, STEP), torch.full_like(i, 3 + 256 * SITE), i % nb]
    key = [seed % (1 << 32), seed // (1 << 32)]
    for r in range(10):
        (h0, l0), (h1, l1) = product(ctr[0], 0xD2511F53), product(ctr[2], 0xCD9E8D57)
        ctr = [h1 ^ ctr[1] ^ (key[0] + r * 0x9E3779B9) % (1 << 32), l1, h0 ^ ctr[3] ^ (key[1] + r * 0xBB67AE85) % (1 << 32), l0]
    out = torch.empty((rows, nb * 8), dtype=torch.int32, device=DEV)
    for j in range(8):
        out[:, j::8] = (ctr[j // 2] // (1 << 16 * (j % 2)) % 65536).reshape(rows, nb)
    return out[:, :C]


def _dropped_exact(x, case, p, seed):
    k = round(p * 65536)
    keep = (_halves_exact(case["N"] * case["S"], case["C"], seed) >= k).reshape(x.shape)
    return x * keep.double() * (65536 / (65536 - k))


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "dropout":
        y = _dropped_exact(st["x"].double(), case, case["p"], st["seed"])
        return [y if st["add"] is None else y + st["add"].double()]
    train = case["train"]
    x = st["x"].double().requires_grad_(train)
    if case["op"] == "norm":
        N, S, C, G = case["N"], case["S"], case["C"], case["G"]
        w, b = st["w"].double().requires_grad_(train), st["b"].double().requires_grad_(train)
        xd = _dropped_exact(x, case, case["drop"], st["seed"]) if case["drop"] else x
        groups = xd.reshape(N, S, G, C // G).permute(0, 2, 1, 3).reshape(N, G, -1)
        var, mean = torch.var_mean(groups, 2, correction=0)
        rstd = (var + 1e-5).rsqrt()
        u = ((groups - mean[..., None]) * rstd[..., None]).reshape(N, G, S, C // G).permute(0, 2, 1, 3).reshape(N, S, C) * w + b
        y = {"none": lambda v: v, "relu": torch.relu, "tanh": torch.tanh, "silu": lambda v: v * torch.sigmoid(v)}[case["act"]](u)
        outs = [y.detach(), mean.detach(), rstd.detach()]
        return outs + list(torch.autograd.grad(y, (x, w, b), st["dout"].double())) if train else outs
    gate, h0 = st["gate"].double().requires_grad_(train), st["h0"].double().requires_grad_(train)
    s, hs = h0, []
    f = torch.sigmoid(gate).unbind(0) if case["kind"] == "sigmoid" else gate.unbind(0)
    v = (torch.sigmoid(-gate) * x).unbind(0) if case["kind"] == "sigmoid" else x.unbind(0)
    ended = None if st["done"] is None else (st["done"] != 0)[..., None]
    for t in range(case["T"]):
        h = torch.addcmul(v[t], f[t], s)
        after = h if ended is None else h.masked_fill(ended[t], 0.0)
        if st["lens"] is not None:
            hold = (t >= st["lens"])[:, None]
            h, after = torch.where(hold, s, h), torch.where(hold, s, after)
        hs.append(h)
        s = after
    h = torch.stack(hs)
    if not train:
        return [h.detach(), s.detach()]
    grads = torch.autograd.grad((h, s), (gate, x, h0), (st["dout"].double(), st["dlast"].double()))
    return [h.detach(), s.detach(), *grads]
