"""Lists whose matrices hold no values: both calls take them and ask nothing of the device (host code only, no GPU needed)."""
import numpy as np
import pytest

from paper_2601_02609_amd import binding as B
from paper_2601_02609_amd import build

ABC = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def L():
    if not build.is_built():
        build.build(verbose=False)
    return B.lib()


@pytest.mark.parametrize("sizes", [[(0, 7)], [(7, 0)], [(0, 0)], [(0, 1 << 40), (3, 0), (0, 1)]])
def test_accepted(L, sizes):
    t = np.zeros(len(sizes), dtype=np.dtype(B._Matrix))
    t["rows"], t["cols"] = zip(*sizes)
    c = np.ascontiguousarray(np.broadcast_to(np.asarray(ABC, dtype=np.float32), (5, 3)))
    assert L.cce_muon_workspace_bytes(t.ctypes.data, len(t)) == 256
    assert L.cce_orthogonalize_multi(t.ctypes.data, len(t), c.ctypes.data, 5, 1e-7, 1 << 20, 256, None) == B.CCE_OK
    assert L.cce_muon_multi_step(t.ctypes.data, len(t), 0.1, 0.9, 1, c.ctypes.data, 5, 1e-7, None, 1 << 20, 256, None) == B.CCE_OK
