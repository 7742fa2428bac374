"""Arrays of the calls around a feature network's step that must not overlap:
refused before any device call (the pointers are never followed)."""
import pytest

from paper_1706_05544_amd import native as nv
from test_network_abi import INV, arr, group_back, needs_no_gpu

# 2 samples of 2 groups: statistics of 16 bytes each, here at 8 << 20 and
# 9 << 20
STATS = dict(mean=8 << 20, rstd=9 << 20)


@pytest.mark.parametrize("kw", [
    dict(dX=arr(6, 4, at=8 << 20)), dict(dX=arr(6, 4, at=9 << 20)),
    dict(dX=arr(6, 4, at=(8 << 20) - 92)), dict(dX=arr(6, 4, at=(9 << 20) + 12)),
    dict(dw=arr(1, 4, at=8 << 20)), dict(dw=arr(1, 4, at=(9 << 20) - 12)),
    dict(db=arr(1, 4, at=(8 << 20) + 12)), dict(db=arr(1, 4, at=9 << 20)),
    # dX on dY as well
    dict(dX=arr(6, 4, at=8 << 20), dY=arr(6, 4, at=8 << 20))])
def test_gradients_on_the_statistics(kw):
    assert group_back(**STATS, **kw) == INV
    assert "overlaps" in nv.svm_last_error()


@needs_no_gpu
def test_gradients_beside_the_statistics():
    for kw in (dict(dX=arr(6, 4, at=(8 << 20) - 96)),
               dict(dw=arr(1, 4, at=(9 << 20) + 16)),
               dict(db=arr(1, 4, at=(8 << 20) - 16))):
        assert group_back(**STATS, **kw) == nv.SVM_E_DEVICE
