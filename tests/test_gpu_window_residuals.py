"""dQ of short windows: the residuals of dS.

dQ = scale sum_u dS k. With dS rounded to bf16 alone each term is off by up to half a step,
2^-8 of the power of two below it: in the norm, with mantissas spread over 1 .. 2, 2^-7 /
sqrt(12) over the root of their mean square, sqrt(7/3): 0.0015 of dQ. In a row of a few
keys, whose every P is above 1/16, dQ's kernel adds the residuals' products (up to 2^-17 of a
dS): what is left is O's rounding of P, at most 2^-8 of a P that is not the row's largest,
through D = <dO, O>: measured on O itself 0.0006 to 0.0008. 0.0012 lies between, and a
half tile of 32 keys whose residuals were left out would show in the rows that see keys
of that half alone."""
import pytest
import torch

import test_gpu_window as W
from paper_2606_08476_amd import flashcp as F
from test_gpu_parity import dev, say  # noqa: F401

pytestmark = pytest.mark.gpu

LIMIT = 0.0012
W.KINDS.update({"plain1": (0.0, False, 1.0), "cap30_1": (30.0, False, 1.0), "cap60_1": (60.0, False, 1.0)})


@pytest.mark.parametrize("kind", ["plain1", "cap30_1", "cap60_1"])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64), (8, 1, 64), (4, 2, 128), (2, 2, 128)])
def test_dq_of_short_windows(hq, hkv, d, kind, dev):  # noqa: F811
    r = W.Run(dict(lens=[1280, 1280], cp=1, rank=0, hq=hq, hkv=hkv, d=d, plan="whole_lpt"), (3, 0), kind, dev)
    want, _ = r.oracle(dout=r.do)
    o, o32, lse = r.forward(F.FC_TWO_PASS)
    g, alone, delta = r.grads(), r.nan(r.tq, hq, d), r.nan(hq, r.tq)
    F.fc_attn_bwd(r.view, r.q, *r.kv, o, lse, r.do, 0.0, *g, r.u8(r.view.workspace_size()[1]), o_f32=o32)
    F.fc_bwd_preprocess(r.view, None, r.do, delta, o_f32=o32)
    F.fc_attn_bwd_dq(r.view, r.q, *r.kv, lse, delta, r.do, 0.0, alone)
    torch.cuda.synchronize()
    half = r.pos[0] // 32 % 2  # of the tiles of 64 keys, which begin with the document
    inside = (r.pos[0] % 32 >= 2)
    for name, dq in (("one launch", g[0]), ("alone", alone)):
        for i in (0, 1):
            rows = inside & (half == i)
            off = float((dq[rows].double() - want["dq"][rows]).norm() / want["dq"][rows].norm())
            say(f"[gpu] dQ residuals {kind} {hq}/{hkv}x{d} {name}, half {i}: {off:.5f}")
            assert off <= LIMIT, (name, i)
