"""Oracle head norms in fp64, with the rotation of rope.py after them.

Test infrastructure only (see the package docstring).

For a head's row x of d values: n = (x - m) s, s = (mean (x - m)^2 + eps)^(-1/2), m = 0
or mean x; y = R(pos) ((w + offset) n). Back, with g = R(pos)^T dy and a = (w + offset) g:
dw = sum g n (over tokens, and heads that share w), dx = s (a - [mean a] - n mean(a n)).

``bounds``, elementwise, follow from the roundings of an fp32 implementation (E: half a
step of fp32): d products summed in any order, (d + 2) E of the sum of their sizes; 1 /
sqrt within 2 E; each product, sum or fused product-sum E of its result; a rotation's
sines and cosines within 2^-20 of the amplitude with its two products and sum. A weight's
gradient is summed over up to 80 roundings in fp32 (a thread's rows, then its
workgroup's threads) and beyond these in fp64. The results' own rounding is added by
``rounded``.

Parity: pinned in tests/test_oracle_norm.py by fp64 autograd and central differences.
"""
from __future__ import annotations

import torch

from . import rope as R

E = 2.0 ** -24
F64 = torch.float64


def rounded(bound, want, dtype):
    """The bound of a result rounded to `dtype`."""
    h = torch.finfo(dtype).eps / 2
    return bound + h * (want.abs() + bound) + torch.finfo(dtype).tiny


def _pairs_sum(x, m, inter):
    """Per value, the sum over its pair; values that are not rotated: 0."""
    y = torch.zeros_like(x)
    ia, ib = (slice(0, m, 2), slice(1, m, 2)) if inter else (slice(0, m // 2), slice(m // 2, m))
    y[..., ia] = y[..., ib] = x[..., ia] + x[..., ib]
    return y


def _rows(x, eps, centred):
    """n, s, and the bounds of n (absolute) and s (relative)."""
    x, d = x.to(F64), x.shape[-1]
    m, dm = torch.zeros_like(x[..., :1]), torch.zeros_like(x[..., :1])
    if centred:
        m = x.mean(-1, keepdim=True)
        dm = (d + 1) * E * x.abs().mean(-1, keepdim=True)
    y = x - m
    s = (y.square().mean(-1, keepdim=True) + eps).rsqrt()
    rs = 0.5 * ((d + 8) * E + 4 * (dm * s).square()) + 4 * E
    n = y * s
    return n, s, s * (dm + E * y.abs()) + n.abs() * (rs + 2 * E), rs.expand_as(s)


def forward(x, weight, pos, w=(), inter=False, amp=1.0, eps=1e-6, offset=0.0, centred=False):
    """(y, bound) of rows x [T, H, d]; weight [d], [H, d] or None; w: radians per position."""
    n, _, dn, _ = _rows(x, eps, centred)
    k = torch.ones((), dtype=F64, device=x.device) if weight is None else weight.to(F64) + offset
    y, b = n * k, dn * k.abs() + 2 * E * (n * k).abs()
    if len(w):
        b = R.rotate_bound(b, pos, w, inter, amp) + 2.0 ** -20 * abs(amp) * _pairs_sum(y.abs(), 2 * len(w), inter)
        y = R.rotate(y, pos, w, inter, amp)
    return y, b


def backward(dy, x, weight, pos, w=(), inter=False, amp=1.0, eps=1e-6, offset=0.0, centred=False):
    """(dx, its bound, dw per head [H, d], its bound) of rows."""
    d = x.shape[-1]
    n, s, dn, rs = _rows(x, eps, centred)
    g, dg = dy.to(F64), torch.zeros_like(n)
    if len(w):
        dg = 2.0 ** -20 * abs(amp) * _pairs_sum(g.abs(), 2 * len(w), inter)
        g = R.rotate(g, pos, w, inter, amp, back=True)
    dw = (g * n).sum(0)
    bw = (dg * n.abs() + g.abs() * dn + 80 * E * (g * n).abs()).sum(0)
    k = torch.ones((), dtype=F64, device=x.device) if weight is None else weight.to(F64) + offset
    a, da = g * k, dg * k.abs() + 2 * E * (g * k).abs()
    mean = lambda t: t.mean(-1, keepdim=True)  # noqa: E731
    m2 = mean(a * n)
    dm2 = mean(da * n.abs() + a.abs() * dn + (d + 2) * E * (a * n).abs())
    m1, dm1 = torch.zeros_like(m2), torch.zeros_like(m2)
    if centred:
        m1, dm1 = mean(a), mean(da + (d + 2) * E * a.abs())
    dx = s * (a - m1 - n * m2)
    b = s * (da + dm1 + dn * m2.abs() + n.abs() * dm2 + 3 * E * (a.abs() + m1.abs() + (n * m2).abs()))
    return dx, b + dx.abs() * (rs + E), dw, bw
