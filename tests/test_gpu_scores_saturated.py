"""Gradients through scores far beyond the cap, where 1 - tanh^2 is all that is left of
them: each document's products lie in one band of so many caps, above or below zero, so
that its dQ and dK are tiny as a whole, and each is held to its own size.

1 - tanh^2(y) = 4 u / (1 + u)^2 with u = e^2y keeps its relative accuracy at either end:
a product x off by e makes it 2 e / cap off, and the exponential's argument, 2 |x| / cap
log2(e), rounds by half a step (2 E |x| / cap counts two of them). dK's is kept in fp16
(FP16, half a step; the bands end where it would be below the smallest normal number:
4 * 2^-30, at 10.4 caps). The rest of the bounds are those of oracle/scores.py."""
import math

import numpy as np
import pytest
import torch

from oracle.scores import BF16, E, FP16
from paper_2606_08476_amd import flashcp as F
from test_gpu_parity import dev, say  # noqa: F401

pytestmark = pytest.mark.gpu

BANDS = [(0.1, 0.5), (4, 5), (-5, -4), (6, 6.5), (7, 7.5), (-7.5, -7), (8, 8.5), (-8.5, -8), (9, 9.5), (-10, -9.5),
         (9.7, 10.2)]
LENS = [150, 33, 170, 129, 64, 201, 90, 140, 257, 111, 75]


def reference(q, k, v, do, cap, slopes):
    """fp64 o, lse, dq, dk, the bounds of dq, dk, and their terms' sizes summed (|dX| times
    |k|, |q|), of one document, own rows only."""
    q, k, v, do = (t.double() for t in (q, k, v, do))
    n, hq, d = q.shape
    G, scale = hq // k.shape[1], 1.0 / math.sqrt(d)
    o, lse = torch.zeros_like(q), torch.zeros(hq, n, dtype=q.dtype, device=q.device)
    dq, bq, tq = (torch.zeros_like(q) for _ in range(3))
    dk, bk, tk = (torch.zeros_like(k) for _ in range(3))
    at = torch.arange(n, device=q.device)
    dist = (at[:, None] - at[None]).double()
    for h in range(hq):
        Q, K, V, dO = q[:, h], k[:, h // G], v[:, h // G], do[:, h]
        x = scale * (Q @ K.T)
        off = (d + 2) * E * scale * (Q.abs() @ K.abs().T)
        s, f = cap * torch.tanh(x / cap), 1 / torch.cosh(x / cap) ** 2
        if slopes is not None:
            s = s - float(slopes[h]) * dist
        s = s.masked_fill(dist < 0, -math.inf)
        L = torch.logsumexp(s, 1)
        P = torch.exp(s - L[:, None])
        O = P @ V
        serr = torch.where(dist < 0, 0.0, off * f + cap * 4 * E + 2 * E * s.abs())
        if slopes is not None:
            serr = serr + torch.where(dist < 0, 0.0, 2 * E * float(slopes[h]) * dist)
        dP, D = dO @ V.T, (dO * O).sum(1, keepdim=True)
        # (o and lse are given, rounded to fp32)
        gerr = 2 * d * E * ((dO.abs() * O.abs()).sum(1, keepdim=True) + dO.abs() @ V.abs().T)
        dX = P * f * (dP - D)
        rel = 2 * off / cap + 2 * E * x.abs() / cap * 2 + FP16 + 16 * E + serr + 4 * E * (L.abs()[:, None] + 1)
        xe = dX.abs() * rel + P * f * gerr
        xe = xe + BF16 * (dX.abs() + xe) + 2.0 ** -18 * dX.abs()
        o[:, h], lse[h], dq[:, h] = O, L, scale * (dX @ K)
        bq[:, h] = scale * (xe @ K.abs())
        dk[:, h // G] += scale * (dX.T @ Q)
        bk[:, h // G] += scale * (xe.T @ Q.abs())
        tq[:, h] = scale * (dX.abs() @ K.abs())
        tk[:, h // G] += scale * (dX.abs().T @ Q.abs())
    return o, lse, dq, dk, bq, bk, tq, tk


@pytest.mark.parametrize("hq,hkv,d,biased,tiles", [
    (4, 1, 64, False, None), (2, 2, 64, True, None), (2, 1, 128, False, None), (4, 1, 128, True, None),
    (4, 1, 64, True, (64, 0, 0, 0)), (1, 1, 128, False, None), (8, 1, 128, False, (128, 0, 0, 0)),
])
@pytest.mark.parametrize("cap", [2.0 ** -6, 0.5, 30.0, 60.0])
def test_saturated_scores(hq, hkv, d, biased, tiles, cap, dev):  # noqa: F811
    say(f"[gpu] saturated heads={hq}/{hkv} d={d} cap={cap} biased={biased}")
    n = sum(LENS)
    cu = np.concatenate([[0], np.cumsum(LENS)]).astype(np.int32)
    slopes = np.linspace(0.001, 0.05, hq).astype(np.float32) if biased else None
    view = F.View(cu, F.fc_plan_per_doc(cu, 1), 1, 0, hq, hkv, d, tiles=tiles, cap=cap, slopes=slopes).bind(dev)
    g = torch.Generator(device=dev).manual_seed(5)
    e = lambda h: torch.randn(n, h, d, generator=g, device=dev)  # noqa: E731
    # rows along one direction, so that every product of a document is in its band
    way = torch.sign(torch.randn(d, generator=g, device=dev))
    lo = torch.tensor([b[0] for b in BANDS], device=dev).repeat_interleave(torch.tensor(LENS, device=dev))
    hi = torch.tensor([b[1] for b in BANDS], device=dev).repeat_interleave(torch.tensor(LENS, device=dev))
    x = (lo + (hi - lo) * torch.rand(n, generator=g, device=dev)) * cap
    unit = math.sqrt(math.sqrt(d))  # q.k / sqrt(d) of `unit * way / sqrt(d)` is 1
    q = (unit * way / math.sqrt(d) + 1e-3 * e(hq)).bfloat16()
    k = (x[:, None, None] * (unit * way / math.sqrt(d) + 1e-3 * e(hkv))).bfloat16()
    v, do = e(hkv).bfloat16(), e(hq).bfloat16()
    none = torch.empty(0, hkv, d, dtype=torch.bfloat16, device=dev)
    refs = [reference(*(t[a:b] for t in (q, k, v, do)), cap, slopes) for a, b in zip(cu, cu[1:])]
    o, dq, dk, bq, bk, tq, tk = (torch.cat([r[i] for r in refs]) for i in (0, 2, 3, 4, 5, 6, 7))
    lse = torch.cat([r[1] for r in refs], 1).float().contiguous()
    z = lambda *s: torch.full(s, float("nan"), device=dev)  # noqa: E731

    def near(name, got, want, bound, terms):
        over = ((got.double() - want).abs() - bound)
        assert bool(torch.isfinite(got).all()) and float(over.max()) <= 0, f"{name}: {float(over.max()):.2e} over"
        for a, b, band in zip(cu, cu[1:], BANDS):
            # the bounds say something: in norm they are under 2^-6 of the terms (BF16 +
            # FP16 = 2^-7.8; products, LSE and score, 1e-3 at the most here; gerr / |dP - D|,
            # 2 d E times some 160 / 11, 5e-4). A document's dQ itself may be much less than
            # its terms: where f is the same for every key a row's dX sum to 0, and these
            # keys are parallel.
            assert float(bound[a:b].norm()) <= 2.0 ** -6 * float(terms[a:b].norm()), f"{name} {band}"

    ws = torch.empty(view.workspace_size()[1], dtype=torch.uint8, device=dev)
    for det in (True, False):
        gr = z(n, hq, d), z(n, hkv, d), z(n, hkv, d), z(0, hkv, d), z(0, hkv, d)
        F.fc_attn_bwd(view, q, k, v, none, none, None, lse, do, 0.0, *gr, ws, deterministic=det, o_f32=o.float())
        torch.cuda.synchronize()
        near(f"dq {det}", gr[0], dq, bq, tq)
        near(f"dk {det}", gr[1], dk, bk, tk)
    delta, alone = z(hq, n), z(n, hq, d)
    F.fc_bwd_preprocess(view, None, do, delta, o_f32=o.float())
    F.fc_attn_bwd_dq(view, q, k, v, none, none, lse, delta, do, 0.0, alone)
    torch.cuda.synchronize()
    near("dq alone", alone, dq, bq, tq)
    view.close()


@pytest.mark.parametrize("lens,cp,rank,hq,hkv,d,tiles", [
    ([1, 300, 700, 70], 2, 1, 4, 1, 64, None), ([900, 37, 1500], 4, 2, 4, 2, 128, None),
    ([900, 37, 1500], 3, 0, 2, 2, 64, None), ([9001, 1, 70], 8, 7, 8, 1, 128, None),  # (split)
    ([640, 129, 1, 70], 1, 0, 8, 1, 128, (64, 0, 0, 0)),
])
@pytest.mark.parametrize("cap", [2.0 ** -6, 0.07, 0.6, 4.0, 55.0])
def test_lse_of_capped_scores(lens, cp, rank, hq, hkv, d, tiles, cap, dev):  # noqa: F811
    """Within the oracle's bound however small the cap and the LSE, from every forward
    call: the exponentials' reference, far above the scores, costs it nothing."""
    import _cases
    from oracle import scores as S
    c = _cases.make_case("lse", "llama8b", lens=lens, cp=cp, rank=rank, hq=hq, hkv=hkv, d=d, plan="per_doc")
    v = F.View(c.cu, c.plan, cp, rank, hq, hkv, d, tiles=tiles, cap=cap).bind(dev)
    tq, tr = v.info["t_q"], v.info["t_recv"]
    g = torch.Generator(device=dev).manual_seed(11)
    e = lambda n, h: torch.randn(n, h, d, generator=g, device=dev, dtype=torch.bfloat16)  # noqa: E731
    q, kv = 2 * e(tq, hq), (e(tq, hkv), e(tq, hkv), e(tr, hkv), e(tr, hkv))
    cu = np.asarray(c.cu)
    at = [np.asarray(a, dtype=np.int64) for a in (c.oview.q_gpos, c.oview.recv_gpos)]
    doc = [torch.from_numpy(np.searchsorted(cu, a, side="right") - 1).to(dev) for a in at]
    pos = [torch.from_numpy(a).to(dev) for a in at]

    def oracle(srcs):
        cat = lambda x: torch.cat([x[i] for i in srcs])  # noqa: E731
        return S.attention(doc[0], pos[0], q, cat(doc), cat(pos), cat(kv[::2]), cat(kv[1::2]), cap)

    def near(name, got, srcs):
        want, bound = oracle(srcs)
        some = torch.isfinite(want["lse"])
        assert torch.equal(torch.isfinite(got), some), name
        over = float(torch.where(some, (got.double() - want["lse"]).abs() / bound["lse"], 0.0).max())
        say(f"[gpu]   lse cap {cap} {name}: {over:.2f} of its bound")
        assert over <= 1, f"{name}: {over:.2f} of its bound"

    z = lambda *s, dt=torch.float32: torch.full(s, float("nan"), dtype=dt, device=dev)  # noqa: E731
    for mode in (F.FC_TWO_PASS, F.FC_FUSED):
        lse, ws = z(hq, tq), torch.empty(max(1, v.workspace_size(mode)[0]), dtype=torch.uint8, device=dev)
        F.fc_attn_fwd(v, q, *kv, 0.0, mode, z(tq, hq, d, dt=torch.bfloat16), None, lse, ws)
        torch.cuda.synchronize()
        near(f"mode {mode}", lse, (0, 1))
    part = [z(tq, hq, d), z(hq, tq), z(tq, hq, d), z(hq, tq)]
    F.fc_attn_fwd_partials(v, q, *kv, 0.0, *part)
    torch.cuda.synchronize()
    near("local", part[1], (0,))
    if tr:
        near("received", part[3], (1,))
    v.close()


@pytest.mark.parametrize("cap,top", [(0.6, 2.0 ** 90), (20.0, 2.0 ** 62), (55.0, 2.0 ** 30), (20.0, 2.0 ** -90)])
def test_values_of_any_size_under_a_cap(cap, top, dev):  # noqa: F811
    """The forward of values far from 1 is that of ordinary ones, scaled: exactly, for a
    power of two."""
    cu = np.array([0, 700, 1400], dtype=np.int32)
    hq, hkv, d, n = 4, 2, 64, 1400
    view = F.View(cu, F.fc_plan_per_doc(cu, 1), 1, 0, hq, hkv, d, cap=cap).bind(dev)
    g = torch.Generator(device=dev).manual_seed(2)
    q, k, v = (torch.randn(n, h, d, generator=g, device=dev).bfloat16() for h in (hq, hkv, hkv))
    none = torch.empty(0, hkv, d, dtype=torch.bfloat16, device=dev)
    res = []
    for s in (1.0, top):
        o32, lse = torch.empty(n, hq, d, device=dev), torch.empty(hq, n, device=dev)
        o = torch.empty(n, hq, d, dtype=torch.bfloat16, device=dev)
        ws = torch.empty(max(1, view.workspace_size(F.FC_FUSED)[0]), dtype=torch.uint8, device=dev)
        F.fc_attn_fwd(view, 4 * q, k, v * s, none, none, 0.0, F.FC_FUSED, o, o32, lse, ws)
        res.append((o32, lse))
    torch.cuda.synchronize()
    assert bool(torch.isfinite(res[1][0]).all()) and torch.equal(res[0][1], res[1][1])
    assert torch.equal(res[0][0], res[1][0] / top)
    view.close()
