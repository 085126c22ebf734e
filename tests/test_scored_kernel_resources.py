"""Vector registers of the scored backward kernels at head dim 64 (no GPU): those that
leave room for three waves per SIMD (168 at most), as they are meant to."""
import pytest

from test_kernel_resources import kernels  # noqa: F401

# dK/dV alone: <head dim, heads per iteration, kind of score>; dQ alone: <head dim,
# heads per tile, kind>. Kinds: 1 cap, 2 bias, 3 both.
DKDV = [f"attn_bwd_scored_kernel<64, {h}, {k}>" for h in (1, 2, 4) for k in (1, 2, 3) if (h, k) != (4, 3)]
DQ = ["attn_bwd_dq_scored_kernel<64, 4, 1>", "attn_bwd_dq_scored_kernel<64, 4, 3>"]


@pytest.mark.parametrize("name", DKDV + DQ)
def test_three_waves_per_simd(kernels, name):  # noqa: F811
    assert kernels[name][".vgpr_count"] <= 168 and kernels[name][".agpr_count"] == 0


def test_every_scored_kernel_is_there_without_spills(kernels):  # noqa: F811
    scored = {n: k for n, k in kernels.items() if "scored" in n}
    # forward: 2 head dims x 3 heads per tile x 6 outputs x 3 kinds; grid: 2 x 6 x 3;
    # dK/dV, its atomic form and dQ: 2 x 3 x 3 each
    assert len(scored) == 108 + 36 + 3 * 18
    assert all(k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0 for k in scored.values())
