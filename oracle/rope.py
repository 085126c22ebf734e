"""Oracle rotary positions in fp64.

Test infrastructure only (see the package docstring).

Pair i of the first m values of a head, (x_i, x_{i + m/2}) or, interleaved,
(x_2i, x_2i+1), as a complex number, is multiplied by A e^(j pos w_i); its gradient
by the conjugate A e^(-j pos w_i). Frequencies are computed here in plain Python
from their published definitions (rotary embedding; position interpolation; the
scaled base; interpolation by wavelength; YaRN).

Parity: pinned in tests/test_oracle_scores.py by an explicit loop with math.cos and
math.sin, by the invariance of products of rotated pairs under a common shift, and
by the gradient's being the transposed map.
"""
from __future__ import annotations

import math

import torch


def frequencies(m, base=10000.0, scaling="none", factor=1.0, low=1.0, high=None, context=0.0):
    """(w_i for i < m/2, amplitude)."""
    high = (32.0 if scaling == "yarn" else 4.0) if high is None else high
    if scaling == "base":
        base = base * factor ** (m / (m - 2))
    w, amp = [base ** (-2 * i / m) for i in range(m // 2)], 1.0
    if scaling == "linear":
        w = [x / factor for x in w]
    if scaling == "bands":
        out = []
        for x in w:
            wavelength = 2 * math.pi / x
            if wavelength < context / high:
                out.append(x)
            elif wavelength > context / low:
                out.append(x / factor)
            else:
                s = (context / wavelength - low) / (high - low)
                out.append((1 - s) * x / factor + s * x)
        w = out
    if scaling == "yarn":
        dim_of = lambda turns: m * math.log(context / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        a, b = max(math.floor(dim_of(high)), 0), min(math.ceil(dim_of(low)), m - 1)
        out = []
        for i, x in enumerate(w):
            ramp = min(max((i - a) / max(b - a, 0.001), 0), 1)
            out.append(x / factor * ramp + x * (1 - ramp))
        w, amp = out, 0.1 * math.log(factor) + 1.0
    return w, amp


def rotate(x, pos, w, interleaved=False, amplitude=1.0, back=False):
    """x [T, H, d] (any type) with its first 2 len(w) values rotated, fp64."""
    x = x.to(torch.float64)
    m = 2 * len(w)
    t = pos.to(torch.float64)[:, None, None] * torch.tensor(w, dtype=torch.float64, device=x.device)
    c, s = amplitude * torch.cos(t), amplitude * torch.sin(t) * (-1 if back else 1)
    y = x.clone()
    ia = slice(0, m, 2) if interleaved else slice(0, m // 2)
    ib = slice(1, m, 2) if interleaved else slice(m // 2, m)
    y[..., ia] = c * x[..., ia] - s * x[..., ib]
    y[..., ib] = c * x[..., ib] + s * x[..., ia]
    return y


def rotate_bound(e, pos, w, interleaved=False, amplitude=1.0, back=False):
    """What an elementwise bound `e` of x becomes: |c| e_a + |s| e_b per pair."""
    m = 2 * len(w)
    t = pos.to(torch.float64)[:, None, None] * torch.tensor(w, dtype=torch.float64, device=e.device)
    c, s = abs(amplitude) * torch.cos(t).abs(), abs(amplitude) * torch.sin(t).abs()
    y = e.clone()
    ia = slice(0, m, 2) if interleaved else slice(0, m // 2)
    ib = slice(1, m, 2) if interleaved else slice(m // 2, m)
    y[..., ia] = c * e[..., ia] + s * e[..., ib]
    y[..., ib] = c * e[..., ib] + s * e[..., ia]
    return y
