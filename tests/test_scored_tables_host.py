"""Tables and workspaces of views with slopes, no GPU: what they may take against
the plain view of the same plan, and values at the ends of what is accepted."""
import os

import numpy as np
import pytest

from paper_2606_08476_amd import flashcp as F


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(F._LIB_PATH):
        from paper_2606_08476_amd import build
        build.build()


def view(lens, hq, hkv, d, cp=1, rank=0, **kw):
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    return F.View(cu, F.fc_plan_per_doc(cu, cp), cp, rank, hq, hkv, d, **kw)


@pytest.mark.parametrize("lens,cp,rank", [([16384], 1, 0), ([9000, 300, 5000], 2, 1)])
def test_a_slope_of_minus_zero_is_zero(lens, cp, rank):
    """Its sign changes nothing: the same tables and workspaces."""
    rest = [0.5] * 7
    a, b = (view(lens, 8, 4, 128, cp, rank, slopes=np.array([z] + rest, dtype=np.float32)) for z in (0.0, -0.0))
    assert a.info == b.info
    for mode in (F.FC_TWO_PASS, F.FC_FUSED):
        assert a.workspace_size(mode) == b.workspace_size(mode)
    for x, y in ((a.export_launch(), b.export_launch()), (a.export_split(), b.export_split())):
        assert all(np.array_equal(x[k], y[k]) for k in x)
    assert not np.signbit(b.score[1]).any()
