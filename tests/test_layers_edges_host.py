"""More of the layers' host side, without a GPU: workspaces beside their tensors, refusals that the header promises."""
import pytest
import torch

P = 0x10000     # fake addresses: a refused call never follows them


@pytest.mark.parametrize("typ, size", [(0, 4), (1, 2)])
@pytest.mark.parametrize("n, s, c, groups", [(65536, 1, 8192, 1), (65536, 1, 4104, 1), (65536, 1, 4104, 27), (8192, 2, 65536, 8), (100000, 3, 6000, 5),
                                             (3000, 70, 8192, 64), (1, 1, 1 << 20, 1 << 20), (300, 1, 1 << 20, 1 << 10), (16, 8192, 4096, 4096), (5, 100, 3000, 1)])
def test_norm_workspace_beside_its_tensors(n, s, c, groups, typ, size):
    """A workspace is a small part of the tensor, beside what the results of a group and a parameter take themselves:
    parameters' partial sums are bounded by the workgroups, not one row per sample, and a tile has shares of its own groups only."""
    from paper_2512_13359_amd import _abi as A
    d = A.AuvNorm(n=n, s=s, c=c, groups=groups, type=typ, act=0, eps=1e-5, x=P, x_sn=s * c, x_ss=c, mean=4 * P, rstd=5 * P)
    x, stats, params = n * s * c * size, 8 * n * groups, 8 * c
    # one partial row at least; a chunk's shares beside the groups' statistics: a sample is at most 512 chunks and tiles, each
    # with at most one more group than its own
    shares = max(512, (n * s * c) // 2048) * 8 + stats * (min(512 // n, s) + 2)
    assert A.auv_norm_work_bytes(d, False) <= shares + x // 16
    assert A.auv_norm_work_bytes(d, True) <= shares + x // 16 + params + (32 << 20)


@pytest.mark.parametrize("s, c, groups, taken", [(1, 4096, 1, True), (1, 4104, 1, False), (4, 4096, 2, True), (5, 2048, 1, True), (5, 2056, 1, False),
                                                 (9, 1368, 1, False), (64, 256, 2, True), (65, 256, 2, False), (1, 8192, 8, True)])
def test_norm_of_more_samples_than_a_launch_takes(s, c, groups, taken):
    """The header's bound: 2^24 samples where p ceil(s / 4) > 512 with p the 16-byte pieces of a row."""
    from paper_2512_13359_amd import _abi as A
    assert taken == (-(-c // 8) * -(-s // 4) <= 512) or groups == 8
    d = A.AuvNorm(n=1 << 24, s=s, c=c, groups=groups, type=A.AUV_BF16, act=0, eps=1e-5, x=P, x_sn=s * c, x_ss=c, mean=4 * P, rstd=5 * P)
    assert (A.lib.auv_norm_work_bytes(d, 1) >= 0) == taken, A.auv_last_error()
    if not taken:
        assert "2^24" in A.auv_last_error()


def _scan(A, **kw):
    d = dict(T=4, n=3, c=8, type=A.AUV_FP32, kind=0, gate=P, gate_st=24, gate_sn=8, gate_sc=1, x=2 * P, x_st=24, x_sn=8, x_sc=1,
             h=3 * P, h_st=24, h_sn=8, h_sc=1, done=4 * P, lens=5 * P, h0=6 * P, h0_sn=8, h0_sc=1, last=7 * P, last_sn=8, last_sc=1)
    d.update(kw)
    return A.AuvScan(**d)


def pairs(outs, others):
    """Every output of a call with every other tensor of it; the exception is a state updated in place."""
    return [(o, i) for o in outs for i in others if o != i and (o, i) != ("last", "h0")]


@pytest.mark.parametrize("out, other", pairs(("h", "last"), ("gate", "x", "done", "lens", "h0", "h", "last")))
def test_scan_forward_refuses_an_output_over_another_tensor(out, other):
    from paper_2512_13359_amd import _abi as A
    d = _scan(A)
    rc = A.lib.auv_scan_forward(_scan(A, **{out: getattr(d, other)}), None, None)
    assert rc == A.AUV_EINVAL and f"'{out}'" in A.auv_last_error() and f"'{other}'" in A.auv_last_error(), A.auv_last_error()


@pytest.mark.parametrize("out, other", pairs(("dgate", "dx", "dh0"), ("gate", "x", "h", "dout", "done", "lens", "h0", "dlast", "dgate", "dx", "dh0")))
def test_scan_backward_refuses_an_output_over_another_tensor(out, other):
    from paper_2512_13359_amd import _abi as A
    g = dict(dout=8 * P, dout_st=24, dout_sn=8, dout_sc=1, dlast=9 * P, dlast_sn=8, dlast_sc=1, dgate=10 * P, dgate_st=24, dgate_sn=8,
             dgate_sc=1, dx=11 * P, dx_st=24, dx_sn=8, dx_sc=1, dh0=12 * P, dh0_sn=8, dh0_sc=1)
    d = _scan(A, last=None)
    g[out] = g[other] if other in g else getattr(d, other)
    rc = A.lib.auv_scan_backward(d, A.AuvScanGrad(**g), None, None)
    assert rc == A.AUV_EINVAL and f"'{out}'" in A.auv_last_error() and f"'{other}'" in A.auv_last_error(), A.auv_last_error()


@pytest.mark.parametrize("out, other", pairs(("y", "mean", "rstd"), ("x", "weight", "bias", "y", "mean", "rstd")))
def test_norm_forward_refuses_an_output_over_another_tensor(out, other):
    from paper_2512_13359_amd import _abi as A
    t = {k: (i + 1) * P for i, k in enumerate(("x", "weight", "bias", "y", "mean", "rstd"))}
    t[out] = t[other]
    d = A.AuvNorm(n=2, s=3, c=8, groups=2, type=0, act=0, eps=1e-5, x=t["x"], x_sn=24, x_ss=8, weight=t["weight"], bias=t["bias"],
                  mean=t["mean"], rstd=t["rstd"])
    rc = A.lib.auv_norm_forward(d, A.AuvRows(t["y"], 24, 8), None, None)
    assert rc == A.AUV_EINVAL and f"'{out}'" in A.auv_last_error() and f"'{other}'" in A.auv_last_error(), A.auv_last_error()


@pytest.mark.parametrize("out, other", pairs(("dx", "dweight", "dbias"), ("x", "dout", "weight", "bias", "mean", "rstd", "dx", "dweight", "dbias")))
def test_norm_backward_refuses_an_output_over_another_tensor(out, other):
    from paper_2512_13359_amd import _abi as A
    t = {k: (i + 1) * P for i, k in enumerate(("x", "weight", "bias", "mean", "rstd", "dout", "dx", "dweight", "dbias"))}
    t[out] = t[other]
    d = A.AuvNorm(n=2, s=3, c=8, groups=2, type=0, act=0, eps=1e-5, x=t["x"], x_sn=24, x_ss=8, weight=t["weight"], bias=t["bias"],
                  mean=t["mean"], rstd=t["rstd"])
    rc = A.lib.auv_norm_backward(d, A.AuvNormGrad(t["dout"], 24, 8, t["dx"], 24, 8, t["dweight"], t["dbias"]), 20 * P, None)
    assert rc == A.AUV_EINVAL and f"'{out}'" in A.auv_last_error() and f"'{other}'" in A.auv_last_error(), A.auv_last_error()


def test_functions_refuse_tensors_whose_gradient_would_be_lost():
    """Results are no part of torch's graph: a tensor that requires grad is refused, unless torch does not record."""
    import paper_2512_13359_amd as M
    x, w, st = torch.zeros(4, 3, 8), torch.zeros(8), torch.zeros(3, 8)
    leaf = lambda t: t.clone().requires_grad_()  # noqa: E731
    d, stat = M.make_drop(0.1, 1), torch.zeros(4, 2)
    calls = [lambda: M.scan_forward(leaf(x), x), lambda: M.scan_forward(x, leaf(x)), lambda: M.scan_forward(x, x, h0=leaf(st)),
             lambda: M.scan_forward(x, x, out=leaf(x)), lambda: M.scan_backward(x, leaf(x), x), lambda: M.scan_backward(x, x, leaf(x)),
             lambda: M.scan_backward(x, x, x, dout=leaf(x)), lambda: M.scan_backward(x, x, x, dh_last=leaf(st)),
             lambda: M.scan_backward(x, x, x, out=(x, leaf(x))), lambda: M.dropout(leaf(x), d), lambda: M.dropout(x, d, leaf(x)),
             lambda: M.dropout(x, d, out=leaf(x)), lambda: M.norm_forward(leaf(x), 2), lambda: M.norm_forward(x, 2, weight=leaf(w)),
             lambda: M.norm_forward(x, 2, bias=torch.nn.Parameter(w)), lambda: M.norm_forward(x, 2, out=leaf(x)),
             lambda: M.norm_backward(leaf(x), 2, stat, stat, x), lambda: M.norm_backward(x, 2, stat, stat, leaf(x)),
             lambda: M.norm_backward(x, 2, stat, stat, x, weight=leaf(w))]
    for k, f in enumerate(calls):
        with pytest.raises(M.AuvError, match="requires grad"):
            f()
        with torch.no_grad(), pytest.raises(M.AuvError, match="on a GPU"):      # taken as far as the next check
            f()


def test_dropout_counter_is_checked():
    import paper_2512_13359_amd as M
    from paper_2512_13359_amd import _abi as A
    d = M.make_drop(0.5, 1)
    assert d.counter is None and d.tensor is None
    for bad in (torch.zeros(1, dtype=torch.int32), torch.zeros(1), torch.zeros(2, dtype=torch.int32)):     # on the host, too
        with pytest.raises(M.AuvError, match="counter"):
            M.make_drop(0.5, 1, counter=bad)
    rows = A.AuvRows(P, 24, 8), None, A.AuvRows(2 * P, 24, 8)
    odd = A.AuvDrop(1, 0, 0, 0, 10, P + 2)
    assert A.lib.auv_dropout(odd, 0, 2, 3, 8, *rows, None) == A.AUV_EINVAL and "counter" in A.auv_last_error()
    x = torch.zeros(4, 8)
    for f in (lambda: M.dropout(x, 0.5), lambda: M.dropout(x, None), lambda: M.norm_forward(x, 2, drop=0.5)):
        with pytest.raises(M.AuvError, match="make_drop"):
            f()


def test_scan_backward_takes_both_results_as_one_tensor():
    """`out` may be any pair: a tensor whose first axis has the two."""
    import paper_2512_13359_amd as M
    x = torch.zeros(4, 3, 8)
    for out in (torch.zeros(2, 4, 3, 8), [x, x], (x, x)):
        with pytest.raises(M.AuvError, match="on a GPU"):
            M.scan_backward(x, x, x, out=out)
    with pytest.raises(M.AuvError, match="pair"):
        M.scan_backward(x, x, x, out=torch.zeros(3, 4, 3, 8))
