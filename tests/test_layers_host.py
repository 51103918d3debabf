"""The layers' refusals, without a GPU: arguments are checked before anything is enqueued."""
import ctypes

import pytest
import torch

P = 0x10000     # fake addresses: a refused call never follows them


def _scan(A, **kw):
    d = dict(T=4, n=3, c=8, type=A.AUV_FP32, kind=0, gate=P, gate_st=24, gate_sn=8, gate_sc=1, x=2 * P, x_st=24, x_sn=8,
             x_sc=1, h=3 * P, h_st=24, h_sn=8, h_sc=1)
    d.update(kw)
    return A.AuvScan(**d)


def _grad(A, **kw):
    d = dict(dout=4 * P, dout_st=24, dout_sn=8, dout_sc=1, dgate=5 * P, dgate_st=24, dgate_sn=8, dgate_sc=1, dx=6 * P,
             dx_st=24, dx_sn=8, dx_sc=1)
    d.update(kw)
    return A.AuvScanGrad(**d)


@pytest.mark.parametrize("change, word", [
    (dict(T=0), "T"), (dict(n=-1), "T"), (dict(c=0), "T"), (dict(n=1 << 20, c=1 << 20), "2^30"), (dict(type=2), "type"),
    (dict(kind=7), "kind"), (dict(gate=None), "gate"), (dict(x=None), "x"), (dict(h=None), "h"), (dict(x=P + 2), "aligned"),
    (dict(h_st=8), "share"), (dict(h_sc=0), "share"), (dict(h=P), "input"), (dict(x_st=-1), "negative"),
    (dict(x_st=1 << 50), "2^44"), (dict(h0=P, h0_sn=1 << 44), "2^44"), (dict(last=P, last_sn=-8, last_sc=1), "negative"), (dict(h0=P + 1), "h0"), (dict(last=P, last_sn=0, last_sc=1), "last"),
    (dict(done=P + 3), "done"), (dict(h0=P, h0_sn=8, h0_sc=1, last=P, last_sn=1, last_sc=3), "last")])
def test_scan_forward_refuses(change, word):
    from paper_2512_13359_amd import _abi as A
    rc = A.lib.auv_scan_forward(_scan(A, **change), None, None)
    assert rc == A.AUV_EINVAL and word in A.auv_last_error(), A.auv_last_error()


@pytest.mark.parametrize("change, word", [
    (dict(dgate=None), "dgate"), (dict(dx=5 * P), "same"), (dict(dx=2 * P), "input"), (dict(dgate=4 * P), "input"),
    (dict(dx_st=23), "share"), (dict(dh0=P + 2), "dh0"), (dict(dlast=P, dlast_sn=8, dlast_sc=1, dh0=P, dh0_sn=8, dh0_sc=1), "dh0"),
    (dict(dout_sn=-8), "negative")])
def test_scan_backward_refuses(change, word):
    from paper_2512_13359_amd import _abi as A
    rc = A.lib.auv_scan_backward(_scan(A), _grad(A, **change), None, None)
    assert rc == A.AUV_EINVAL and word in A.auv_last_error(), A.auv_last_error()


def test_scan_workspace():
    """Many columns need none; few columns of many steps do, and a call without it is refused."""
    from paper_2512_13359_amd import _abi as A
    assert A.auv_scan_work_bytes(_scan(A)) == 0
    long = _scan(A, T=100000)
    assert A.auv_scan_work_bytes(long) > 0 and A.auv_scan_work_bytes(long, _grad(A)) > 0
    assert A.lib.auv_scan_forward(long, None, None) == A.AUV_EINVAL and "work" in A.auv_last_error()
    assert A.lib.auv_scan_backward(long, _grad(A), None, None) == A.AUV_EINVAL and "work" in A.auv_last_error()
    # and never below the steps that the header names
    for n, c in ((1, 1), (3, 8), (64, 64), (1, 5000)):
        few = dict(T=A.AUV_SCAN_SPLIT_STEPS - 1, n=n, c=c)
        few |= {f"{t}_{k}": v for t in ("gate", "x", "h") for k, v in (("st", n * c), ("sn", c))}
        grad = {f"{t}_{k}": v for t in ("dout", "dgate", "dx") for k, v in (("st", n * c), ("sn", c))}
        for typ in (A.AUV_FP32, A.AUV_BF16):
            assert A.auv_scan_work_bytes(_scan(A, type=typ, **few)) == 0
            assert A.auv_scan_work_bytes(_scan(A, type=typ, **few), _grad(A, **grad)) == 0
    # with the state updated in place the steps are not split: no chunk may read what the last one writes
    assert A.auv_scan_work_bytes(_scan(A, T=100000, h0=7 * P, h0_sn=8, h0_sc=1, last=7 * P, last_sn=8, last_sc=1)) == 0
    with pytest.raises(A.AuvError):
        A.auv_scan_work_bytes(_scan(A, T=0))


def _norm(A, **kw):
    d = dict(n=2, s=3, c=8, groups=2, type=A.AUV_FP32, act=0, eps=1e-5, x=P, x_sn=24, x_ss=8, mean=4 * P, rstd=5 * P)
    d.update(kw)
    return A.AuvNorm(**d)


@pytest.mark.parametrize("change, word", [
    (dict(n=0), ">= 1"), (dict(groups=0), ">= 1"), (dict(groups=3), "divide"), (dict(type=5), "type"), (dict(act=9), "activation"),
    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(weight=P + 1), "aligned"), (dict(x=None), "x"),
    (dict(x=P + 1), "aligned"), (dict(x_ss=-8), "negative"), (dict(mean=None), "NULL"), (dict(c=1 << 21, groups=1), "large")])
def test_norm_refuses(change, word):
    from paper_2512_13359_amd import _abi as A
    rc = A.lib.auv_norm_forward(_norm(A, **change), A.AuvRows(2 * P, 24, 8), P, None)
    assert rc == A.AUV_EINVAL and word in A.auv_last_error(), A.auv_last_error()
    if "x" not in change:
        rc = A.lib.auv_norm_backward(_norm(A, **change), A.AuvNormGrad(2 * P, 24, 8, 3 * P, 24, 8), P, None)
        assert rc == A.AUV_EINVAL and word in A.auv_last_error(), A.auv_last_error()


def test_norm_refuses_outputs_and_workspace():
    from paper_2512_13359_amd import _abi as A
    for y, word in ((A.AuvRows(P, 24, 8), "memory of 'x'"), (A.AuvRows(2 * P, 24, 7), "share"), (A.AuvRows(2 * P, 8, 8), "share"),
                    (A.AuvRows(None, 24, 8), "NULL")):
        rc = A.lib.auv_norm_forward(_norm(A), y, P, None)
        assert rc == A.AUV_EINVAL and word in A.auv_last_error(), A.auv_last_error()
    # small samples need no workspace forward, long ones do
    assert A.auv_norm_work_bytes(_norm(A), False) == 0
    long = _norm(A, s=5000, x_sn=40000)
    assert A.auv_norm_work_bytes(long, False) > 0 and A.auv_norm_work_bytes(long, True) > 0
    assert A.lib.auv_norm_forward(long, A.AuvRows(2 * P, 40000, 8), None, None) == A.AUV_EINVAL and "work" in A.auv_last_error()
    assert A.lib.auv_norm_work_bytes(_norm(A, n=1 << 24, s=64, c=256), 1) == -1 and "2^24" in A.auv_last_error()
    for g, word in ((A.AuvNormGrad(2 * P, 24, 8, P, 24, 8), "input"), (A.AuvNormGrad(2 * P, 24, 8, 2 * P, 24, 8), "input"),
                    (A.AuvNormGrad(2 * P, 24, 8, 3 * P, 24, 8, 6 * P, 6 * P), "same"),
                    (A.AuvNormGrad(2 * P, 24, 8, 3 * P, 24, 8, 6 * P + 2, None), "aligned")):
        rc = A.lib.auv_norm_backward(_norm(A), g, P, None)
        assert rc == A.AUV_EINVAL and word in A.auv_last_error(), A.auv_last_error()
    assert A.lib.auv_norm_backward(_norm(A), A.AuvNormGrad(2 * P, 24, 8, 3 * P, 24, 8), None, None) == A.AUV_EINVAL
    for bad in (A.AuvDrop(1, 0, 1 << 24, 0, 10), A.AuvDrop(1, 0, 0, 0, 65536), A.AuvDrop(1, 0, 0, (1 << 32) - 1, 10)):
        rc = A.lib.auv_norm_forward(_norm(A, drop=ctypes.addressof(bad)), A.AuvRows(2 * P, 24, 8), P, None)
        assert rc == A.AUV_EINVAL


def test_dropout_refuses():
    from paper_2512_13359_amd import _abi as A
    d, x = A.make_drop(0.5, 1), A.AuvRows(P, 24, 8)

    def call(drop=d, type=0, n=2, s=3, c=8, x=x, add=None, y=A.AuvRows(2 * P, 24, 8)):
        return A.lib.auv_dropout(drop, type, n, s, c, x, add, y, None)

    for kw, word in ((dict(drop=None), "NULL"), (dict(y=None), "NULL"), (dict(n=0), ">= 1"), (dict(type=3), "type"),
                     (dict(x=A.AuvRows(P + 2, 24, 8)), "aligned"), (dict(y=A.AuvRows(2 * P, 24, 4)), "share"),
                     (dict(y=A.AuvRows(P, 32, 8)), "other strides"), (dict(add=A.AuvRows(P + 1, 24, 8)), "add"),
                     (dict(add=A.AuvRows(2 * P, 48, 8)), "other strides"),
                     (dict(drop=A.AuvDrop(1, 0, 0, (1 << 32) - 5, 10)), "2^32")):
        assert call(**kw) == A.AUV_EINVAL and word in A.auv_last_error(), (kw, A.auv_last_error())
    for kw in (dict(p=1.0), dict(p=-0.1), dict(p=0.999999), dict(p=float("nan")), dict(seed=1 << 64), dict(seed=-1),
               dict(step=1 << 32), dict(site=1 << 24), dict(row0=-1)):
        with pytest.raises(A.AuvError):
            A.make_drop(**{**dict(p=0.1, seed=3), **kw})
    assert A.make_drop(0.1, 3).drop == 6554 and A.make_drop(0.0, 3).drop == 0


def test_functions_refuse():
    """The functions on tensors: shapes, types, devices and layouts, before any GPU call."""
    import paper_2512_13359_amd as M
    x = torch.zeros(4, 3, 8)
    st = torch.zeros(3, 8)
    bad = [lambda: M.scan_forward(x, x), lambda: M.scan_forward(x, x[0]), lambda: M.scan_forward(x, x.half()),
           lambda: M.scan_forward(x.bfloat16(), x), lambda: M.scan_forward(x, x, kind="tanh"),
           lambda: M.scan_forward(x, x, done=torch.zeros(3, 4)), lambda: M.scan_forward(x, x, done=torch.zeros(3, 4).t()),
           lambda: M.scan_forward(x, x, done=torch.zeros(4, 3, dtype=torch.bool)),
           lambda: M.scan_forward(x, x, lens=torch.zeros(3, dtype=torch.int64)), lambda: M.scan_forward(x, x, h0=st.bfloat16()),
           lambda: M.scan_forward(x, x, h0=st.t()), lambda: M.scan_forward(x, x, out=x[:2]),
           lambda: M.scan_backward(x, x, x[:1]), lambda: M.scan_backward(x, x, x, dh_last=st[:1]),
           lambda: M.norm_forward(x, 1), lambda: M.norm_forward(x[0, 0], 1), lambda: M.norm_forward(x.double(), 1),
           lambda: M.norm_forward(x, 1, weight=torch.zeros(7)), lambda: M.norm_forward(x, 1, act="gelu"),
           lambda: M.norm_forward(x.permute(0, 2, 1), 1), lambda: M.norm_backward(x, 2, torch.zeros(4, 1), torch.zeros(4, 2), x),
           lambda: M.norm_backward(x, 2, torch.zeros(4, 2), torch.zeros(4, 2), x[:, :1]),
           lambda: M.norm_forward(x, 1 << 40), lambda: M.norm_forward(x, 1.5), lambda: M.norm_forward(x, 1, eps=1e300),
           lambda: M.dropout(x, M.make_drop(0.1, 1)), lambda: M.dropout(x, M.make_drop(0.1, 1), x.bfloat16())]
    for f in bad:
        with pytest.raises(M.AuvError):
            f()


def test_packed_structures_are_the_bindings_own():
    """The words that the functions pack land in the fields they are meant for, and the fields where a C++
    compiler puts the header's."""
    from paper_2512_13359_amd import _abi as A
    from paper_2512_13359_amd import layers as L
    for kind, layout in ((A.AuvScan, L._SCAN), (A.AuvScanGrad, L._SCAN_GRAD), (A.AuvNorm, L._NORM)):
        names = [f[0] for f in kind._fields_]
        got = kind.from_buffer_copy(layout.pack(*range(1, len(names) + 1)))
        assert ctypes.sizeof(kind) == layout.size and [getattr(got, k) for k in names] == list(range(1, len(names) + 1))


def test_structures_match_the_header(tmp_path):
    """Sizes and offsets of the layers' structures, asked of a C++ compiler."""
    import os
    import shutil
    import subprocess
    from paper_2512_13359_amd import _abi as A
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("needs a C++ compiler")
    want = {"auv_scan": (A.AuvScan, {"gate_st": "gate.st", "x": "x.p", "h_sc": "h.sc", "done": "done", "h0": "h0.p", "last_sc": "last.sc"}),
            "auv_scan_grad": (A.AuvScanGrad, {"dlast": "dlast.p", "dgate": "dgate.p", "dx_sn": "dx.sn", "dh0_sc": "dh0.sc"}),
            "auv_drop": (A.AuvDrop, {"step": "step", "drop": "drop"}), "auv_rows": (A.AuvRows, {"ss": "ss"}),
            "auv_norm": (A.AuvNorm, {"eps": "eps", "x_ss": "x.ss", "weight": "weight", "drop": "drop"}),
            "auv_norm_grad": (A.AuvNormGrad, {"dx": "dx.p", "dweight": "dweight"})}
    lines, expect = [], []
    for name, (kind, fields) in want.items():
        lines.append(f"sizeof({name})")
        expect.append(ctypes.sizeof(kind))
        for f, member in fields.items():
            lines.append(f"offsetof({name}, {member})")
            expect.append(getattr(kind, f).offset)
    src = tmp_path / "a.cpp"
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src.write_text('#include <cstddef>\n#include <cstdio>\n#include "auv.h"\nint main() {\n'
                   + "".join(f'  std::printf("%zu\\n", (size_t){x});\n' for x in lines) + "}\n")
    subprocess.run([cxx, "-std=c++17", f"-I{root}/include", str(src), "-o", str(tmp_path / "a")], check=True)
    out = subprocess.run([str(tmp_path / "a")], check=True, capture_output=True, text=True).stdout
    assert [int(x) for x in out.split()] == expect
