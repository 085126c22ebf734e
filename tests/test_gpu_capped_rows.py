"""Rows of a single key under capped scores without a window, from every forward call and
through the backward.

Such a row's O is its key's value and its score has no gradient. P is rounded to bf16, its
sum is not, so that this holds where P is a power of two but for fp32's roundings: of the
exponent and of what it is counted from (numbers of 32 to 64: 2^-19 each, ln 2 of that in
P), of the exponential (2^-22) and of the division and its product (2^-23): under 2^-18."""
import pytest
import torch

import test_gpu_window as W
from paper_2606_08476_amd import flashcp as F
from test_gpu_parity import dev, say  # noqa: F401
from test_gpu_scores import near

pytestmark = pytest.mark.gpu

OFF = 2.0 ** -18
W.KINDS.update({"cap4": (4.0, False, 6.0)})
ALONE = dict(lens=[1] * 40 + [5, 300, 1, 7], cp=1, rank=0, plan="whole_lpt")
SHAPES = [dict(ALONE, hq=8, hkv=2, d=128), dict(ALONE, hq=4, hkv=4, d=64), dict(ALONE, hq=4, hkv=2, d=128),
          dict(lens=[2, 3, 1, 40, 9] * 9, cp=2, rank=0, hq=8, hkv=2, d=128),
          dict(lens=[9001, 1, 70], cp=8, rank=0, hq=8, hkv=1, d=128),
          dict(lens=[6001, 1, 77, 300], cp=4, rank=0, hq=4, hkv=2, d=64)]


@pytest.mark.parametrize("kind", ["cap4", "cap30", "cap55"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{len(s['lens'])}x{max(s['lens'])}-{s['hq']}-{s['hkv']}-{s['d']}")
def test_rows_of_a_single_key(shape, kind, dev):  # noqa: F811
    say(f"[gpu] capped rows {shape} {kind}")
    hq, hkv, d = shape["hq"], shape["hkv"], shape["d"]
    r = W.Run(shape, (0, 0), kind, dev)
    want, b = r.oracle(dout=r.do)
    one = r.pos[0] == 0
    assert bool(one.any())
    k, v = (t[one].repeat_interleave(hq // hkv, 1).float() for t in r.kv[:2])

    def whole(name, o32):
        over = float(((o32[one] - v).abs() / v.abs().clamp(min=2.0 ** -100)).max())
        say(f"[gpu]   {name}: {over:.1e}")
        assert over <= OFF, name

    for mode in (F.FC_TWO_PASS, F.FC_FUSED):
        o, o32, lse = r.forward(mode)
        near("o", o, want["o"], b["o"])
        near("lse", lse, want["lse"], b["lse"])
        whole(f"mode {mode}", o32)
    part = r.partials()
    whole("local", part[0])
    if r.tr:  # rows that see one received key, whatever they see of their own
        first = r.doc[1][:, None] == r.doc[0]
        seen = (first & (r.pos[1][:, None] <= r.pos[0])).sum(0)
        rows = torch.nonzero(seen == 1).flatten()
        if len(rows):
            at = first[:, rows].int().argmax(0)
            got, val = part[2][rows], r.kv[3][at].repeat_interleave(hq // hkv, 1).float()
            assert bool(((got - val).abs() <= OFF * val.abs()).all())
    o, o32, lse = r.forward(F.FC_TWO_PASS)
    g = r.grads()
    F.fc_attn_bwd(r.view, r.q, *r.kv, o, lse, r.do, 0.0, *g, r.u8(r.view.workspace_size()[1]), o_f32=o32)
    torch.cuda.synchronize()
    W.check_grads("bwd", r, g, want, b)
    # dS = P (dP - D): sums of d products of dO and of V, or O; times 1 - tanh^2 <= 1, scale < 1
    size = (r.do[one].float().abs() * v.abs()).sum(-1) * (OFF + (d + 4) * 2.0 ** -23)
    assert bool((g[0][one].abs() <= size[..., None] * k.abs()).all())


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 2, 64)])
def test_documents_of_few_tokens_are_as_exact_as_uncapped(hq, hkv, d, dev):  # noqa: F811
    """Where the cap hardly bends the scores, O and the gradients of documents of two and
    three tokens are off in the norm by what those of the uncapped view are: the same
    roundings, other draws. (Over some thousand rows and heads the norms of such errors
    differ by a few percent; a quarter is allowed.)"""
    W.KINDS.update({"cap50": (50.0, False, 1.0), "uncapped": (0.0, False, 1.0)})
    off = {}
    for kind in ("uncapped", "cap50"):
        r = W.Run(dict(lens=[2, 3] * 150, cp=1, rank=0, hq=hq, hkv=hkv, d=d, plan="whole_lpt"), (0, 0), kind, dev)
        want, _ = r.oracle(dout=r.do)
        o, o32, lse = r.forward(F.FC_TWO_PASS)
        g = r.grads()
        F.fc_attn_bwd(r.view, r.q, *r.kv, o, lse, r.do, 0.0, *g, r.u8(r.view.workspace_size()[1]), o_f32=o32)
        torch.cuda.synchronize()
        off[kind] = {n: float((t.double() - want[n]).norm() / want[n].norm())
                     for n, t in (("o", o32), ("dq", g[0]), ("dk", g[1]))}
        say(f"[gpu] few tokens {kind}: {off[kind]}")
    for n in ("o", "dq", "dk"):
        assert off["cap50"][n] <= 1.25 * off["uncapped"][n], (n, off)
