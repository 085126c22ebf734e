"""Vector registers of the kernels of windowed views and of the head norms (no GPU)."""
import re

from test_kernel_resources import kernels  # noqa: F401


def test_every_windowed_kernel_is_there_without_spills(kernels):  # noqa: F811
    windowed = {n: k for n, k in kernels.items() if "window" in n}
    # forward: 2 head dims x 3 heads per tile x 6 outputs x 4 kinds of score; grid: 2 x 6 x 4;
    # dK/dV, its atomic form and dQ: 2 x 3 x 4 each
    assert len(windowed) == 144 + 48 + 3 * 24
    assert all(k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0 for k in windowed.values())


def test_two_waves_per_simd_but_with_slopes(kernels):  # noqa: F811
    for n, k in kernels.items():
        if "window" not in n:
            continue
        args = [int(a) for a in re.findall(r"\d+", n[n.index("<"):])]
        biased = args[-1] & 2
        ungrouped = n.startswith("attn_bwd_atomic") and args[1] == 1
        if args[0] == 64 or not (biased or ungrouped):
            assert k[".vgpr_count"] + k[".agpr_count"] <= 256, n


def test_norm_kernels_are_there_without_spills(kernels):  # noqa: F811
    norms = {n: k for n, k in kernels.items() if re.match("norm_(fwd|bwd|sum)_", n)}
    # 2 head dims x 3 layouts, forward and twice backward; the sums twice
    assert len(norms) == 6 + 12 + 2
    assert all(k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0 for k in norms.values())
