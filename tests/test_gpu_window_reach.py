"""Windows longer than the slopes' reach: keys that a window lets in and the bias leaves
without weight are not visited. Bounds as in test_gpu_window.py."""
import numpy as np
import pytest
import torch

import test_gpu_window as W
from paper_2606_08476_amd import flashcp as F
from test_gpu_parity import dev, say  # noqa: F401

pytestmark = pytest.mark.gpu

STEEP = {"even": lambda hq: np.full(hq, 0.5), "alibi": lambda hq: 2.0 ** (-8.0 * np.arange(hq) / hq),
         "flat_one": lambda hq: np.where(np.arange(hq) == hq - 1, 0.0, 4.0)}
W.SHAPES.update({
    "far_g4": dict(lens=[3100, 37, 1500], cp=4, rank=3, hq=8, hkv=2, d=128),
    "far_g2_d64": dict(lens=[3100, 37, 1500], cp=3, rank=1, hq=4, hkv=2, d=64),
    "far_g1": dict(lens=[3100, 1, 1500], cp=2, rank=0, hq=3, hkv=3, d=128),
    "far_split_g8": dict(lens=[9001, 1, 70], cp=8, rank=7, hq=8, hkv=1, d=128),
    "far_split_g2_d64": dict(lens=[6001, 1, 77, 300], cp=4, rank=3, hq=4, hkv=2, d=64),
    "far_local_g8_d64": dict(lens=[3100, 129, 1, 70], cp=1, rank=0, hq=16, hkv=2, d=64, plan="whole_lpt"),
})


def norm_bytes(c, r):
    """What a view that looks for keys out of reach takes beside the plain window's."""
    plain = F.View(c.cu, c.plan, c.cp, c.rank, c.hq, c.hkv, c.d, tiles=c.tiles, window=r.win[0], sinks=r.win[1])
    return r.view.workspace_size(F.FC_FUSED)[0] - plain.workspace_size(F.FC_FUSED)[0]


@pytest.mark.parametrize("shape,win,kind,slopes", [
    (s, w, k, n) for i, s in enumerate(("far_g4", "far_g2_d64", "far_g1", "far_split_g8", "far_split_g2_d64",
                                        "far_local_g8_d64"))
    for j, (w, k) in enumerate((((700, 4), "bias"), ((1200, 100), "cap30_bias"), ((2048, 0), "bias")))
    for n in (("even", "alibi", "flat_one")[(i + j) % 3], "even")])
def test_windows_longer_than_the_reach(shape, win, kind, slopes, monkeypatch, dev):  # noqa: F811
    say(f"[gpu] window reach {slopes}")
    monkeypatch.setattr(W, "slopes_of", lambda hq: STEEP[slopes](hq).astype(np.float32))
    r = W.Run(shape, win, kind, dev)
    if slopes == "even":
        assert norm_bytes(r.case, r) == (r.case.hq + 2 * r.case.hkv) * 1024
    W.test_windowed_views(shape, win, kind, dev)


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64), (2, 2, 128)])
@pytest.mark.parametrize("kind", ["bias", "cap30_bias"])
def test_keys_out_of_reach_are_not_read(kind, hq, hkv, d, monkeypatch, dev):  # noqa: F811
    """The last 300 tokens of 3000 under slopes of 1 and windows of 2000 with sinks: of the
    values before token 2400, none of which has a weight, none is read."""
    monkeypatch.setattr(W, "slopes_of", lambda n: np.ones(n, dtype=np.float32))
    r = W.Run(dict(lens=[3000, 5], cp=2, rank=1, hq=hq, hkv=hkv, d=d), (2000, 4), kind, dev, tail=300)
    want, b = r.oracle(dout=r.do)
    # norms: scores within 3 x (a few more than sqrt(d)) of sqrt(d): 2 B + 100 < 1.4427 * 300
    far = (r.doc[1] == 0) & (r.pos[1] < 2400)
    assert bool(far.any())
    r.kv[3][far] = float("nan")
    for mode in (F.FC_TWO_PASS, F.FC_FUSED):
        o, o32, lse = r.forward(mode)
        W.near("o", o, want["o"], b["o"])
        W.near("lse", lse, want["lse"], b["lse"])
    for det in (True, False):
        o, o32, lse = r.forward(F.FC_TWO_PASS)
        g = r.grads()
        F.fc_attn_bwd(r.view, r.q, *r.kv, o, lse, r.do, 0.0, *g, r.u8(r.view.workspace_size()[1]),
                      deterministic=det, o_f32=o32)
        torch.cuda.synchronize()
        W.check_grads("bwd", r, g, want, b)
        assert not bool(g[3][far].any()) and not bool(g[4][far].any())
