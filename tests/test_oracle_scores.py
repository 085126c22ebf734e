"""Pins of the oracles of scored attention and rotary positions (CPU, fp64)."""
import math

import numpy as np
import pytest
import torch

from oracle import attention as A
from oracle import rope as R
from oracle import scores as S

F64 = torch.float64


def _problem(seed, lens=(5, 1, 7), hq=4, hkv=2, d=8):
    g = torch.Generator().manual_seed(seed)
    T = sum(lens)
    doc = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(lens))
    pos = torch.cat([torch.arange(n) for n in lens])
    e = lambda h: torch.randn(T, h, d, generator=g, dtype=F64)  # noqa: E731
    return doc, pos, 2 * e(hq), e(hkv), e(hkv), e(hq)


KINDS = [(0.0, False), (1.5, False), (0.0, True), (2.0, True)]
SLOPES = [0.0, 0.3, 1.0, 0.05]


def _dense(doc, pos, q, k, v, cap, slopes):
    """Attention over explicit T x T masks, differentiable."""
    G, d = q.shape[1] // k.shape[1], q.shape[2]
    K, V = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
    s = torch.einsum("thd,uhd->htu", q, K) / math.sqrt(d)
    if cap:
        s = cap * torch.tanh(s / cap)
    if slopes is not None:
        s = s - torch.tensor(slopes, dtype=F64)[:, None, None] * (pos[:, None] - pos[None])
    seen = (doc[:, None] == doc[None]) & (pos[:, None] >= pos[None])
    s = s.masked_fill(~seen, -math.inf)
    return torch.einsum("htu,uhd->thd", torch.softmax(s, -1), V), torch.logsumexp(s, -1)


@pytest.mark.parametrize("cap,bias", KINDS)
def test_against_autograd(cap, bias):
    doc, pos, q, k, v, do = _problem(1)
    slopes = SLOPES if bias else None
    out, bnd = S.attention(doc, pos, q, doc, pos, k, v, cap, slopes, do)
    a = [t.clone().requires_grad_() for t in (q, k, v)]
    o, lse = _dense(doc, pos, *a, cap, slopes)
    o.backward(do)
    for n, t in (("o", o), ("lse", lse), ("dq", a[0].grad), ("dk", a[1].grad), ("dv", a[2].grad)):
        assert torch.allclose(out[n], t, rtol=0, atol=1e-12), n
        assert bool((bnd[n] >= 0).all()) and bnd[n].shape == out[n].shape


def test_against_differences():
    doc, pos, q, k, v, do = _problem(2, (4, 3), 2, 1, 4)
    f = lambda q, k, v: float((S.attention(doc, pos, q, doc, pos, k, v, 1.2, [0.2, 0.7])[0]["o"] * do).sum())  # noqa: E731
    out, _ = S.attention(doc, pos, q, doc, pos, k, v, 1.2, [0.2, 0.7], do)
    h = 1e-5
    for n, i in (("dq", 0), ("dk", 1), ("dv", 2)):
        t = [q, k, v][i]
        for e in range(0, t.numel(), 3):
            w = torch.zeros_like(t).view(-1)
            w[e] = h
            w = w.view_as(t)
            hi, lo = [x.clone() for x in (q, k, v)], [x.clone() for x in (q, k, v)]
            hi[i], lo[i] = t + w, t - w
            assert abs((f(*hi) - f(*lo)) / (2 * h) - float(out[n].view(-1)[e])) < 1e-8


def test_without_a_function_it_is_the_plain_oracle():
    doc, pos, q, k, v, do = _problem(3)
    out, _ = S.attention(doc, pos, q, doc, pos, k, v, dout=do)
    cu, g = np.array([0, 5, 6, 13]), np.arange(13)
    O, L = A.attention_fwd(cu, g, q, g, k, v)
    dq, dk, dv = A.attention_bwd(cu, g, q, g, k, v, do)
    for a, b in ((out["o"], O), (out["lse"], L), (out["dq"], dq), (out["dk"], dk), (out["dv"], dv)):
        assert torch.allclose(a, b, rtol=0, atol=1e-12)


def test_rows_without_keys():
    doc, pos, q, k, v, _ = _problem(4)
    out, _ = S.attention(doc, pos, q, doc[6:], pos[6:] + 3, k[6:], v[6:], 2.0, SLOPES)
    assert torch.isinf(out["lse"][:, :9]).all() and (out["o"][:9] == 0).all()
    assert torch.isfinite(out["lse"][:, 9:]).all()


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("m", [2, 6, 8])
def test_rotation(m, inter):
    g = torch.Generator().manual_seed(5)
    x, y = torch.randn(6, 2, 8, generator=g, dtype=F64), torch.randn(6, 2, 8, generator=g, dtype=F64)
    pos = torch.tensor([0, 1, 2, 7, 1000, 123456])
    w, _ = R.frequencies(m)
    rx = R.rotate(x, pos, w, inter, 1.5)
    for t in range(6):
        for i in range(m // 2):
            a, b = (2 * i, 2 * i + 1) if inter else (i, i + m // 2)
            c, s = math.cos(int(pos[t]) * w[i]), math.sin(int(pos[t]) * w[i])
            assert torch.allclose(rx[t, :, a], 1.5 * (x[t, :, a] * c - x[t, :, b] * s), rtol=0, atol=1e-12)
            assert torch.allclose(rx[t, :, b], 1.5 * (x[t, :, b] * c + x[t, :, a] * s), rtol=0, atol=1e-12)
    assert torch.equal(rx[..., m:], x[..., m:])
    # products of rows depend on their distance only (the values left alone apart)
    p = lambda a, b: (R.rotate(x, torch.full((6,), a), w, inter)[..., :m] *  # noqa: E731
                      R.rotate(y, torch.full((6,), b), w, inter)[..., :m]).sum(-1)
    assert torch.allclose(p(11, 4), p(511, 504), rtol=0, atol=1e-10)
    # the gradient is the transposed map, and its bound holds what it moves
    gx = R.rotate(y, pos, w, inter, 1.5, back=True)
    assert torch.allclose((rx * y).sum(), (x * gx).sum(), rtol=1e-12)
    e = x.abs()
    assert bool((R.rotate_bound(e, pos, w, inter, 1.5) >= rx.abs() - 1e-12).all())


def test_frequencies():
    w, amp = R.frequencies(64, 10000.0)
    assert w[0] == 1.0 and amp == 1.0 and abs(w[-1] - 10000.0 ** (-62 / 64)) < 1e-18
    lin, _ = R.frequencies(64, scaling="linear", factor=4.0)
    assert all(abs(a - b / 4) < 1e-18 for a, b in zip(lin, w))
    # the scaled base leaves the first pair and divides the last by the factor
    b, _ = R.frequencies(64, scaling="base", factor=4.0)
    assert b[0] == 1.0 and abs(b[-1] - w[-1] / 4) < 1e-15
    for s in ("bands", "yarn"):
        v, amp = R.frequencies(64, scaling=s, factor=8.0, context=8192)
        assert v[0] == w[0] and abs(v[-1] - w[-1] / 8) < 1e-18
        assert all(x / 8 - 1e-18 <= y <= x + 1e-18 for x, y in zip(w, v))
        assert amp == (1.0 if s == "bands" else 0.1 * math.log(8.0) + 1)
