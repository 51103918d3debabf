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
