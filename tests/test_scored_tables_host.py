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


LAYOUTS = [
    # documents, cp, rank, hq, hkv, d
    ([16384], 1, 0, 8, 8, 128), ([131072], 1, 0, 32, 8, 128), ([131072], 16, 15, 32, 8, 128),
    ([98304, 20000, 12768], 16, 15, 32, 8, 128), ([262144], 32, 31, 64, 8, 128), ([65536], 8, 7, 4, 4, 64),
    ([32768], 4, 3, 8, 1, 128), ([8192], 1, 0, 32, 8, 128), ([700, 1300, 48, 9001], 2, 1, 16, 16, 64),
]


@pytest.mark.parametrize("lens,cp,rank,hq,hkv,d", LAYOUTS)
@pytest.mark.parametrize("slope", ["geometric", 0.02, 0.1, 0.25, 0.5, 2.0, 1024.0])
def test_steep_slopes_take_no_more_backward_workspace(lens, cp, rank, hq, hkv, d, slope):
    """Beside the row norms and the dQ slots (which are bounded, and only there where
    fc_attn_bwd_noalloc's scratch has room for them if it has for the rest), a view
    with slopes takes what the plain view takes, and cuts its key tiles as that does."""
    s = 2.0 ** (-8.0 * np.arange(1, hq + 1) / hq) if slope == "geometric" else np.full(hq, slope)
    plain, biased = view(lens, hq, hkv, d, cp, rank), view(lens, hq, hkv, d, cp, rank, slopes=s)
    norms = 256 * 4 * (hq + 2 * hkv)
    dq_most = max(256 << 20, 4 * 4 * plain.info["t_q"] * hq * d)

    for got, want in zip(biased.workspace_size()[1:], plain.workspace_size()[1:]):
        assert got <= want + norms + dq_most
        if want <= F.NOALLOC_SCRATCH_BYTES:
            assert got <= F.NOALLOC_SCRATCH_BYTES + norms
    a, b = plain.export_launch(), biased.export_launch()
    assert all(np.array_equal(a[k], b[k]) for k in ("bwd_launch", "bwd_reduce", "bwd_qfirst"))
    assert biased.info["n_bwd_slots"] == plain.info["n_bwd_slots"]


@pytest.mark.parametrize("lens,cp,rank,hq,hkv,d", LAYOUTS)
@pytest.mark.parametrize("slope", ["geometric", 0.1, 0.5, 1024.0])
def test_steep_slopes_take_no_more_forward_workspace(lens, cp, rank, hq, hkv, d, slope):
    """Beside the row norms, a view with slopes takes what the plain view takes, and
    splits its key ranges as that does."""
    s = 2.0 ** (-8.0 * np.arange(1, hq + 1) / hq) if slope == "geometric" else np.full(hq, slope)
    plain, biased = view(lens, hq, hkv, d, cp, rank), view(lens, hq, hkv, d, cp, rank, slopes=s)
    for mode in (F.FC_TWO_PASS, F.FC_FUSED):
        more = biased.workspace_size(mode)[0] - plain.workspace_size(mode)[0]
        assert more in (0, 256 * 4 * (hq + 2 * hkv))
    a, b = plain.export_split(), biased.export_split()
    assert a["fwd_chunk"] == b["fwd_chunk"]
    assert all(np.array_equal(a[k], b[k]) for k in ("fwd_units", "fwd_comb"))
