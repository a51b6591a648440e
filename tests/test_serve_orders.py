"""Scales of 4-bit weights in either order, without a GPU: what is refused before the library
runs anything."""
import pytest
import torch
from test_serve_abi import FAKE, MIS, lib  # noqa: F401

import paper_2606_10531_amd as lc
from paper_2606_10531_amd import _lib as L


def call(lib, N=2, m=48, n=256, group=64, packed=FAKE, scales=FAKE, zeros=None, order=L.SCALES_BY_ROW, X=FAKE, Y=FAKE, dt=L.BF16,
         ws=FAKE, wsb=1 << 40):
    return lib.lcvq_linear_fwd_int4_ex(N, m, n, group, packed, scales, zeros, order, X, Y, dt, ws, wsb, None)


def test_refusals(lib):  # noqa: F811
    for kw, status in [(dict(order=2), L.EINVAL), (dict(order=-1), L.EINVAL), (dict(N=-1), L.EINVAL), (dict(group=16), L.EUNSUPPORTED),
                       (dict(n=200), L.EINVAL), (dict(m=(1 << 21) - 8, n=1 << 20, group=32), L.EUNSUPPORTED), (dict(scales=None), L.EINVAL),
                       (dict(scales=MIS), L.EALIGN), (dict(zeros=MIS), L.EALIGN), (dict(n=8192, m=16, ws=None), L.EWORKSPACE)]:
        for order in (L.SCALES_BY_GROUP, L.SCALES_BY_ROW):
            assert call(lib, **{"order": order, **kw}) == status, kw
            assert L.last_error()
    for kw in (dict(N=0, X=None, Y=None), dict(m=0, packed=None, Y=None)):
        assert call(lib, **kw) == L.OK, kw


def test_binding_asks_where_the_shape_does_not_tell(monkeypatch):
    """With the device's checks out of the way: the order that the library is told."""
    seen = []

    class Lib:
        def lcvq_int4_workspace_bytes(self, *a):
            return 0

        def lcvq_linear_fwd_int4_ex(self, *a):
            seen.append(a[7])
            return 0
    monkeypatch.setattr(lc._lib, "load", lambda: Lib())
    monkeypatch.setattr(lc, "_stream", lambda dev: 0)
    monkeypatch.setattr(lc, "_dev", lambda t, name: t.data_ptr())

    def run(m, n, shape, zeros=None, **kw):
        z = None if zeros is None else torch.zeros(zeros, dtype=torch.bfloat16)
        lc.linear_fwd_int4(torch.zeros((m, n // 2), dtype=torch.uint8), torch.zeros(shape, dtype=torch.bfloat16),
                           torch.zeros((2, n), dtype=torch.bfloat16), 32, zeros=z, **kw)
        return seen.pop()
    assert run(48, 128, (48, 4), (48, 4)) == L.SCALES_BY_ROW
    assert run(48, 128, (4, 48), (4, 48)) == L.SCALES_BY_GROUP
    assert run(1, 32, (1, 1)) in (L.SCALES_BY_ROW, L.SCALES_BY_GROUP)
    with pytest.raises(ValueError, match="by_group"):
        run(4, 128, (4, 4))
    assert run(4, 128, (4, 4), by_group=True) == L.SCALES_BY_GROUP
    assert run(4, 128, (4, 4), by_group=False) == L.SCALES_BY_ROW
    for shape, zeros, kw in (((48, 4), (4, 48), {}), ((4, 48), (48, 4), {}), ((48, 4), None, dict(by_group=True)),
                             ((4, 48), None, dict(by_group=False)), ((48, 3), None, {})):
        with pytest.raises(ValueError):
            run(48, 128, shape, zeros, **kw)
    assert not seen
