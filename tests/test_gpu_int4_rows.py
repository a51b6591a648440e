"""4-bit weights whose scales and zero points stand as they are made, a row of n/group for every
weight row: the same bits as from a row of m for every group, of which the other tests show that
they are the definition's."""
import numpy as np
import pytest
import test_gpu_int4 as int4

pytestmark = pytest.mark.gpu

lc = int4.lc


def _both(lc, a, group, dtype):
    """The result from scales by row, after it is the one from scales by group."""
    z = None if a[2] is None else a[2].t().contiguous()
    got = lc.linear_fwd_int4(a[0], a[1].t().contiguous(), a[3], group, zeros=z, out_dtype=dtype)
    assert got.equal(lc.linear_fwd_int4(a[0], a[1], a[3], group, zeros=a[2], out_dtype=dtype))
    return got


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128, 384])
@pytest.mark.parametrize("N,m", [(1, 1), (1, 4097), (3, 33), (16, 250), (5, 1000), (16, 64), (37, 100)])
def test_sizes(lc, N, m, group, zeros):
    import torch
    for n, dtype in ((group, torch.float32), (3 * group, torch.bfloat16), (13 * group, torch.float32)):
        a = int4._draw(N, m, n, group, zeros, N + m)
        int4._check(_both(lc, a, group, dtype), *a, group)


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("mr", [1, 2, 3, 4, 5, 6, 7, 8])
def test_every_tile(lc, mr, group, zeros):
    import torch
    m = 256 * 16 * mr - 5
    for N in (2, 7):
        _both(lc, int4._draw(N, m, 640 if group == 128 else 544 // group * group, group, zeros, mr), group, torch.float32)


@pytest.mark.parametrize("N,m,n,group", [(1, 16, 28672, 128), (16, 100, 8192, 64), (9, 2000, 4096 + 32, 32), (2, 257, 65536, 4096),
                                         (16, 4100, 16384, 64)])
def test_k_split_over_blocks(lc, N, m, n, group):
    import torch
    _both(lc, int4._draw(N, m, n, group, True, 5), group, torch.float32)


def test_as_many_rows_as_groups(lc):
    """The shape does not tell then: the caller has to."""
    import torch
    a = int4._draw(3, 16, 512, 32, True, 6)
    with pytest.raises(ValueError, match="by_group"):
        lc.linear_fwd_int4(a[0], a[1], a[3], 32, zeros=a[2])
    want = lc.linear_fwd_int4(a[0], a[1], a[3], 32, zeros=a[2], out_dtype=torch.float32, by_group=True)
    int4._check(want, *a, 32)
    got = lc.linear_fwd_int4(a[0], a[1].t().contiguous(), a[3], 32, zeros=a[2].t().contiguous(), out_dtype=torch.float32,
                             by_group=False)
    assert got.equal(want)


def test_refusals(lc):
    a = int4._draw(2, 48, 256, 64, True, 10)
    rows = a[1].t().contiguous(), a[2].t().contiguous()
    for scales, zeros, kw in ((rows[0], a[2], {}), (a[1], rows[1], {}), (rows[0], rows[1], dict(by_group=True)), (a[1], a[2], dict(by_group=False)),
                              (rows[0][:, :3], rows[1], {}), (a[1].t(), rows[1], {}), (rows[0].float(), rows[1], {}), (None, None, {})):
        with pytest.raises((TypeError, ValueError)):
            lc.linear_fwd_int4(a[0], scales, a[3], 64, zeros=zeros, **kw)
    assert np.isfinite(lc.linear_fwd_int4(a[0], rows[0], a[3], 64, zeros=rows[1]).float().cpu().numpy()).all()
