"""Oracle attention with a score function: capped scores and a distance bias,
forward and backward, with what a bf16 / fp32 implementation may be off by.

Test infrastructure only (see the package docstring).

For query g and key u of one document, u <= g (positions in the document; query
head h on KV head h // (Hq / Hkv)):

* with a window W and S sinks, of these u only those with g - u < W or u < S;
* x = scale <q_gh, k_uj>; s = cap tanh(x / cap) (or x, cap 0) - slope_h (g - u);
* LSE = ln sum_u e^s, P = e^(s - LSE), O = sum_u P v_uj;
* dP = <dO, v>, D = <dO, O>, dX = P (dP - D) (1 - tanh^2(x / cap)),
  dQ = scale sum_u dX k, dK = scale sum_g dX q, dV = sum_g P dO, summed over the
  query heads of a KV head.

Everything in fp64. ``bounds`` (elementwise, same shapes as the outputs) follow
from the roundings an implementation makes: products of bf16 values summed in fp32;
P, dX and the bf16 O rounded to bf16 (2^-8 of the value); 1 - tanh^2 to fp16 (2^-11);
exponentials, reciprocals and fp32 sums (2^-22 or so each); and P, dX and products
below the smallest normal number, 2^-126, taken as 0: TINY for up to 2^20 of them in
a sum, factors of up to 2^20 with them.

Parity: pinned in tests/test_oracle_scores.py by fp64 autograd, by central
differences, and against attention.py where there is no score function.
"""
from __future__ import annotations

import math

import torch

BF16, FP16 = 2.0 ** -8, 2.0 ** -11   # half a step, relative
E = 2.0 ** -23                       # a step of fp32
TINY = 2.0 ** (-126 + 20 + 20)


def attention(doc_q, pos_q, q, doc_k, pos_k, k, v, cap=0.0, slopes=None, dout=None, scale=None,
              delta_from_bf16=False, window=0, sinks=0):
    """(out, bounds): dicts of fp64 tensors o [T, Hq, d], lse [Hq, T] and, with dout,
    dq, dk, dv; doc_*, pos_*: int tensors, each token's document and position in it.
    Rows without a visible key: o 0, lse -inf. bounds["o32"]: of an fp32 O."""
    f64, dev = torch.float64, q.device
    T, hq, d = q.shape
    hkv = k.shape[1]
    G = hq // hkv
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    z = lambda *s: torch.zeros(*s, dtype=f64, device=dev)  # noqa: E731
    out = dict(o=z(T, hq, d), lse=torch.full((hq, T), -math.inf, dtype=f64, device=dev))
    bnd = dict(o=z(T, hq, d), o32=z(T, hq, d), lse=z(hq, T))
    if dout is not None:
        for n, s in (("dq", q.shape), ("dk", k.shape), ("dv", v.shape)):
            out[n], bnd[n] = z(*s), z(*s)
    for n in torch.unique(doc_q).tolist():
        rows, keys = torch.nonzero(doc_q == n).flatten(), torch.nonzero(doc_k == n).flatten()
        dist = pos_q[rows][:, None] - pos_k[keys][None]
        seen = dist >= 0
        if window:
            seen = seen & ((dist < window) | (pos_k[keys] < sinks)[None])
        dist = dist.to(f64)
        for h in range(hq):
            Q, K, V = q[rows, h].to(f64), k[keys, h // G].to(f64), v[keys, h // G].to(f64)
            X = scale * (Q @ K.T)
            err = (d + 2) * E * scale * (Q.abs() @ K.abs().T)   # of the score
            F = torch.ones_like(X)                              # ds/dx
            S = X
            if cap:
                F = 1 / torch.cosh(X / cap) ** 2
                S = cap * torch.tanh(X / cap)
                err = err * F + cap * 4 * E
            if slopes is not None:
                S = S - float(slopes[h]) * dist
                err = err + 2 * E * float(slopes[h]) * dist
            err = err + 2 * E * S.abs()
            S = S.masked_fill(~seen, -math.inf)
            err = err.masked_fill(~seen, 0.0)
            L = torch.logsumexp(S, 1)
            some = torch.isfinite(L)
            P = torch.where(some[:, None], torch.exp(S - torch.where(some, L, 0.0)[:, None]), 0.0)
            O = P @ V
            out["o"][rows, h], out["lse"][h, rows] = O, L
            mean = (P * err).sum(1, keepdim=True)               # of the log of the sum
            rel = err + mean + 8 * E                            # of P, relative
            sums = P @ V.abs()
            o32 = (P * (BF16 + rel)) @ V.abs() + 8 * E * sums
            bnd["o32"][rows, h], bnd["o"][rows, h] = o32, o32 + BF16 * (O.abs() + o32)
            lerr = mean[:, 0] + 4 * E * (torch.where(some, L, 0.0).abs() + 1)
            bnd["lse"][h, rows] = lerr
            if dout is None:
                continue
            dO = dout[rows, h].to(f64)
            dP = dO @ V.T
            D = (dO * O).sum(1, keepdim=True)
            oerr = bnd["o" if delta_from_bf16 else "o32"][rows, h]
            derr = (dO.abs() * oerr).sum(1, keepdim=True) + d * E * (dO.abs() * O.abs()).sum(1, keepdim=True)
            gerr = derr + d * E * (dO.abs() @ V.abs().T)        # of dP - D
            pe = P * (err + lerr[:, None] + 8 * E)              # of P, absolute
            dX = P * F * (dP - D)
            fe = F * FP16 + 8 * E if cap else 0.0
            xe = (dP - D).abs() * (P * fe + F * pe) + P * F * gerr
            xe = xe + BF16 * (dX.abs() + xe) + 2.0 ** -18 * dX.abs()  # rounded, and summed over many
            out["dq"][rows, h] = scale * (dX @ K)
            bnd["dq"][rows, h] = scale * (xe @ K.abs())
            out["dk"][keys, h // G] += scale * (dX.T @ Q)
            bnd["dk"][keys, h // G] += scale * (xe.T @ Q.abs())
            out["dv"][keys, h // G] += P.T @ dO
            bnd["dv"][keys, h // G] += (pe + BF16 * (P + pe) + 2.0 ** -18 * P).T @ dO.abs()
    for n in bnd:
        if n != "lse":
            bnd[n] += TINY
    return out, bnd
