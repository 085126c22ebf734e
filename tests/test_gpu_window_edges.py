"""Windowed views at their limits: KV heads that do not fill the XCDs evenly, ranks
without rows, the largest windows and sinks, positions far into a document under steep
slopes, and calls at once on two streams. Bounds as in test_gpu_window.py."""
import numpy as np
import pytest
import torch

import test_gpu_window as W
from paper_2606_08476_amd import flashcp as F
from test_gpu_parity import dev, say  # noqa: F401
from test_gpu_scores import BF, F32, near

pytestmark = pytest.mark.gpu

W.SHAPES.update({
    "three_g2": dict(lens=[900, 37, 500], cp=3, rank=2, hq=6, hkv=3, d=128),
    "five_g2_d64": dict(lens=[900, 37, 500], cp=3, rank=1, hq=10, hkv=5, d=64),
    "three_g4": dict(lens=[700, 1, 333], cp=2, rank=0, hq=12, hkv=3, d=128),
    "three_g8": dict(lens=[700, 1, 333], cp=2, rank=1, hq=24, hkv=3, d=128),
    "five_g1_d64": dict(lens=[700, 1, 333], cp=2, rank=0, hq=5, hkv=5, d=64),
})


@pytest.mark.parametrize("shape,win,kind", [(s, w, k) for s in ("three_g2", "five_g2_d64", "three_g4", "three_g8",
                                                                "five_g1_d64")
                                            for w, k in (((100, 4), "plain"), ((64, 64), "bias"), ((33, 0), "cap30"),
                                                         ((257, 5), "cap30_bias"))])
def test_heads(shape, win, kind, dev):  # noqa: F811
    W.test_windowed_views(shape, win, kind, dev)


@pytest.mark.parametrize("win", [(1, 2 ** 31 - 1), (5, 700), (700, 2 ** 31 - 1), (2 ** 31 - 1, 3)])
def test_largest_windows_and_sinks(win, dev):  # noqa: F811
    """Sinks that are all of a document: every row sees what it does without a window."""
    W.test_windowed_views("mixed_g4", win, "plain", dev)


def test_a_rank_without_rows(dev):  # noqa: F811
    v = F.View([0, 10, 300], [[0, 0, 0, 10], [1, 0, 0, 290]], 2, 1, 4, 2, 64, window=4, sinks=1).bind(dev)
    e = lambda h, dt=BF: torch.empty(0, h, 64, dtype=dt, device=dev)  # noqa: E731
    q, kv, lse = e(4), [e(2) for _ in range(4)], torch.empty(4, 0, device=dev)
    o, o32 = e(4), e(4, F32)
    for mode in (F.FC_TWO_PASS, F.FC_FUSED):
        F.fc_attn_fwd(v, q, *kv, 0.0, mode, o, o32, lse,
                      torch.empty(max(v.workspace_size(mode)[0], 1), dtype=torch.uint8, device=dev))
    g = [e(4, F32)] + [e(2, F32) for _ in range(4)]
    F.fc_attn_bwd(v, q, *kv, o, lse, e(4), 0.0, *g,
                  torch.empty(max(v.workspace_size()[1], 1), dtype=torch.uint8, device=dev), o_f32=o32)
    torch.cuda.synchronize()


@pytest.mark.parametrize("slopes,cap", [([0.5, 2.0 ** -8, 4.0, 0.03], "bias"), ([1024.0, 128.0, 700.0, 3.0], "bias"),
                                        ([1024.0, 0.25, 2.0 ** -8, 0.0], "cap30_bias")])
@pytest.mark.parametrize("hkv,d", [(1, 128), (4, 64)])
def test_far_into_a_document(slopes, cap, hkv, d, monkeypatch, dev):  # noqa: F811
    """The last tokens of four million, sinks at its start."""
    say(f"[gpu] window far {slopes} {cap} {hkv} {d}")
    n = 4000037
    monkeypatch.setattr(W, "slopes_of", lambda hq: np.array(slopes, dtype=np.float32))
    r = W.Run(dict(lens=[n], cp=2, rank=1, hq=4, hkv=hkv, d=d), (300, 4), cap, dev, tail=130)
    assert (r.tq, r.tr) == (130, 299 + 4)
    want, b = r.oracle(dout=r.do)
    # (a row's share of its biases, counted from the document's start, is off by up to
    # 2^-24 slope n, all scores alike, which the LSE is corrected for; the roundings of
    # scores as large, of the maximum's, the sum's logarithm's and the correction's, are
    # each 2^-24 of that)
    rest = (torch.tensor(slopes, dtype=torch.float64, device=dev) * n * 2.0 ** -46)[:, None]
    for mode in (F.FC_TWO_PASS, F.FC_FUSED):
        o, o32, lse = r.forward(mode)
        near("o", o, want["o"], b["o"])
        near("lse", lse, want["lse"], b["lse"] + rest)
    o, o32, lse = r.forward(F.FC_TWO_PASS)
    g = r.grads()
    F.fc_attn_bwd(r.view, r.q, *r.kv, o, lse, r.do, 0.0, *g, r.u8(r.view.workspace_size()[1]), o_f32=o32)
    torch.cuda.synchronize()
    W.check_grads("bwd", r, g, want, b)


def test_two_calls_at_once(dev):  # noqa: F811
    """Steps on two streams over one view, with workspaces of their own."""
    r = W.Run("split_g4", (2500, 100), "plain", dev)
    v, streams = r.view, [torch.cuda.Stream() for _ in range(2)]

    def step(x):
        (o, o32, lse), g, fws, bws = x
        F.fc_attn_fwd(v, r.q, *r.kv, 0.0, F.FC_TWO_PASS, o, o32, lse, fws)
        F.fc_attn_bwd(v, r.q, *r.kv, o, lse, r.do, 0.0, *g, bws, o_f32=o32)
        return [o, o32, lse, *g]

    new = lambda: (r.outs(), r.grads(), r.u8(v.workspace_size()[0]), r.u8(v.workspace_size()[1]))  # noqa: E731
    want, xs = step(new()), [new() for _ in streams]
    torch.cuda.synchronize()
    for _ in range(4):
        got = []
        for s, x in zip(streams, xs):
            with torch.cuda.stream(s):
                got.append(step(x))
    torch.cuda.synchronize()
    assert all(W.same(want, g) for g in got)


@pytest.mark.parametrize("window", [3, 500])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64)])
def test_capped_rows_of_a_single_key(window, hq, hkv, d, dev):  # noqa: F811
    """A row that sees one key has that key's value for O, whatever its P was rounded to,
    and no gradient in its score: in windows that end in the documents and in ones that
    reach over them. O's only rounding is then the product with 1 / P, in fp32: a step."""
    shape = dict(lens=[1] * 40 + [5, 300, 1, 7], cp=1, rank=0, hq=hq, hkv=hkv, d=d, plan="whole_lpt")
    r = W.Run(shape, (window, 0), "cap30", dev)
    want, b = r.oracle(dout=r.do)
    one = r.pos[0] == 0
    for mode in (F.FC_TWO_PASS, F.FC_FUSED):
        o, o32, lse = r.forward(mode)
        near("o", o, want["o"], b["o"])
        near("lse", lse, want["lse"], b["lse"])
        v = r.kv[1][one].repeat_interleave(hq // hkv, 1).float()
        assert bool(((o32[one] - v).abs() <= 2.0 ** -22 * v.abs()).all())
    o, o32, lse = r.forward(F.FC_TWO_PASS)
    g = r.grads()
    F.fc_attn_bwd(r.view, r.q, *r.kv, o, lse, r.do, 0.0, *g, r.u8(r.view.workspace_size()[1]), o_f32=o32)
    torch.cuda.synchronize()
    W.check_grads("bwd", r, g, want, b)
    # dS = P (dP - D): sums of d products of dO and O, which are the same within fp32
    size = (r.do[one].float().abs() * v.abs()).sum(-1) * (d + 4) * 2.0 ** -23
    k = r.kv[0][one].repeat_interleave(hq // hkv, 1).float().abs()
    assert bool((g[0][one].abs() <= size[..., None] * k).all())
