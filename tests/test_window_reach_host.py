"""Which windowed views with slopes look for keys out of reach (no GPU): those whose windows
are longer than that, at the price of the row norms' workspace."""
import numpy as np
import pytest

import _cases
from paper_2606_08476_amd import flashcp as F


def workspaces(lens, cp, rank, hq, hkv, d, window, sinks, **score):
    c = _cases.make_case("reach", "llama8b", lens=lens, cp=cp, rank=rank, hq=hq, hkv=hkv, d=d, plan="per_doc")
    v = F.View(c.cu, c.plan, cp, rank, hq, hkv, d, window=window, sinks=sinks, **score)
    return np.array([*v.workspace_size(F.FC_TWO_PASS), *v.workspace_size(F.FC_FUSED)])


@pytest.mark.parametrize("lens,cp,rank,hq,hkv,d", [([131072], 1, 0, 32, 8, 128), ([9000, 300, 7000], 4, 3, 8, 2, 64),
                                                  ([9000, 300, 7000], 4, 0, 4, 1, 128)])
@pytest.mark.parametrize("window,sinks,slope,looks", [
    # reach of unit normal rows: (2 sqrt(d) + 100 / 1.4427) / slope, 85 to 92 tokens / slope
    (16384, 4, 0.5, True), (1000, 0, 0.5, True), (1000, 70, 1.0, True),
    (100, 0, 0.5, False), (1000, 0, 0.05, False), (1, 3, 8.0, False), (64, 64, 8.0, False)])
def test_windows_longer_than_the_reach(lens, cp, rank, hq, hkv, d, window, sinks, slope, looks):
    s = np.full(hq, slope, dtype=np.float32)
    # (as many chunks and parts either way: those of the plain window)
    a = workspaces(lens, cp, rank, hq, hkv, d, window, sinks)
    b = workspaces(lens, cp, rank, hq, hkv, d, window, sinks, slopes=s)
    extra = (hq + 2 * hkv) * 1024 if looks else 0
    for i in (0, 3):  # forward
        assert b[i] - a[i] == extra
    assert (b - a >= extra - 2 ** 28).all()
