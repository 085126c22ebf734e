"""Arguments of windowed views that the binding itself refuses (no GPU)."""
import numpy as np
import pytest

from paper_2606_08476_amd import flashcp as F

CU, PLAN = np.array([0, 10], dtype=np.int32), [[0, 0, 0, 10]]


@pytest.mark.parametrize("kw", [dict(window=2 ** 32 + 1), dict(window=2 ** 31), dict(window=4, sinks=2 ** 32),
                                dict(window=-2 ** 32)])
def test_beyond_32_bits(kw):
    """Not another window, modulo 2^32."""
    with pytest.raises(ValueError):
        F.View(CU, PLAN, 1, 0, 4, 2, 64, **kw)


@pytest.mark.parametrize("kw", [dict(window=2.5), dict(window=4, sinks=1.0), dict(window="4")])
def test_not_integers(kw):
    with pytest.raises(TypeError):
        F.View(CU, PLAN, 1, 0, 4, 2, 64, **kw)


def test_the_largest():
    v = F.View(CU, PLAN, 1, 0, 4, 2, 64, window=2 ** 31 - 1, sinks=2 ** 31 - 1)
    assert v.window == (2 ** 31 - 1, 2 ** 31 - 1) and v.export_window() is None
    v = F.View(CU, PLAN, 1, 0, 4, 2, 64, window=np.int64(1), sinks=2 ** 31 - 1)   # sinks: all there is
    assert v.export_window() is not None and v.info["pairs_loc"] + v.info["pairs_recv"] == 55
