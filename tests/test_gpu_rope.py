"""Rotary rows against the fp64 oracle: the rank's own rows, the KV gather, and
gradients, over layouts, rotated parts, types, strides and positions; and one
training step through all of them and attention with a score function.

Tolerances. The angle is off by at most 2^-26 turns (its conversion to fp32), its
sine and cosine by 2 steps of fp32 more: less than 2^-21 of the amplitude each; two
products and a sum add 3 roundings. So y = c a - s b is within 2^-20 A (|a| + |b|) in
fp32, and half a bf16 step of y more (2^-8 |y|) where it is rounded. What is not
rotated is copied or rounded to the bit."""
import numpy as np
import pytest
import torch

import _cases
from oracle import rope as R
from oracle import scores as S
from paper_2606_08476_amd import flashcp as F
from test_gpu_parity import dev, say  # noqa: F401
from test_gpu_scores import near

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
SHORT = [1, 1, 3, 1, 70, 1, 2, 129, 1, 64, 5, 250, 1, 31]


class Rank:
    def __init__(self, dev, lens=(300, 1, 699, 70), cp=2, rank=1, hq=4, hkv=2, d=64, plan="per_doc"):
        self.c = c = _cases.make_case("rows", "tiny", lens=list(lens), cp=cp, rank=rank, hq=hq, hkv=hkv, d=d,
                                      plan=plan)
        self.view = F.View(c.cu, c.plan, cp, rank, hq, hkv, d).bind(dev)
        self.dev, self.hq, self.hkv, self.d = dev, hq, hkv, d
        g = [np.asarray(a, dtype=np.int64) for a in (c.oview.q_gpos, c.oview.recv_gpos)]
        cu = np.asarray(c.cu)
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)  # noqa: E731
        self.gpos = [t(a) for a in g]
        self.doc = [t(np.searchsorted(cu, a, side="right") - 1) for a in g]
        self.pos = [t(a - cu[np.searchsorted(cu, a, side="right") - 1]) for a in g]
        self.gen = torch.Generator(device=dev).manual_seed(sum(lens) + d)

    def randn(self, n, h, dt=BF):
        return torch.randn(n, h, self.d, generator=self.gen, device=self.dev, dtype=dt)

    def nan(self, n, h, dt=BF):
        return torch.full((n, h, self.d), float("nan"), device=self.dev, dtype=dt)

    @property
    def sizes(self):
        return self.gpos[0].numel(), self.gpos[1].numel()


def check(name, got, x, pos, w, inter, amp, back=False):
    """got: x rotated, in its type, where the first 2 len(w) values are concerned, and
    x itself, rounded, elsewhere."""
    m = 2 * len(w)
    want = R.rotate(x, pos, w, inter, amp, back)
    bound = 2.0 ** -20 * R.rotate_bound(x.double().abs(), pos, [0.0] * len(w), inter, amp)
    # (rotate_bound at angle 0 is A |a|: a pair's two values are both needed)
    ia, ib = (slice(0, m, 2), slice(1, m, 2)) if inter else (slice(0, m // 2), slice(m // 2, m))
    s = bound[..., ia] + bound[..., ib]
    bound[..., ia] = s
    bound[..., ib] = s
    if got.dtype == BF:
        bound = bound + 2.0 ** -8 * (want.abs() + bound)
    e = (got.double() - want).abs()[..., :m]
    over = float((e - bound[..., :m]).max()) if e.numel() else 0.0
    say(f"[gpu]   {name}: max {float(e.max()) if e.numel() else 0:.2e}")
    assert over <= 0, (name, over)
    assert torch.equal(got[..., m:], x[..., m:].to(got.dtype)), name


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d,m", [(64, 64), (64, 2), (64, 16), (64, 24), (64, 62), (128, 128), (128, 32), (128, 6),
                                 (128, 112), (128, 126)])
def test_layouts(d, m, inter, dev):  # noqa: F811
    say(f"[gpu] rope d {d} rotated {m} interleaved {inter}")
    r = Rank(dev, d=d)
    (tq, tr), T = r.sizes, int(r.c.cu[-1])
    rope = F.Rope(m, base=500.0, interleaved=inter, amplitude=1.25)
    w = rope.inv_freq.tolist()
    # own rows out of a fused buffer, into tensors of their own
    x = r.randn(tq, r.hq + 2 * r.hkv)
    q, k, v = x.split([r.hq, r.hkv, r.hkv], 1)
    qo, ko, vo = r.nan(tq, r.hq), r.nan(tq, r.hkv), r.nan(tq, r.hkv)
    F.fc_rope_fwd(r.view, rope, q, k, v, qo, ko, vo)
    torch.cuda.synchronize()
    check("q", qo, q, r.pos[0], w, inter, 1.25)
    check("k", ko, k, r.pos[0], w, inter, 1.25)
    assert torch.equal(vo, v)
    # in place, in the fused buffer: the same bits, the values as they were
    y = x.clone()
    q2, k2, v2 = y.split([r.hq, r.hkv, r.hkv], 1)
    F.fc_rope_fwd(r.view, rope, q2, k2, None, q2, k2, None)
    torch.cuda.synchronize()
    assert torch.equal(q2, qo) and torch.equal(k2, ko) and torch.equal(v2, v)
    # the gather: own and received, together and apart
    kp, vp = r.randn(T, r.hkv), r.randn(T, r.hkv)
    out = [r.nan(n, r.hkv) for n in (tq, tq, tr, tr)]
    F.fc_kv_gather_rope(r.view, rope, kp, vp, *out)
    torch.cuda.synchronize()
    for i in (0, 1):
        check(f"gathered k {i}", out[2 * i], kp[r.gpos[i]], r.pos[i], w, inter, 1.25)
        assert torch.equal(out[2 * i + 1], vp[r.gpos[i]])
    apart = [r.nan(n, r.hkv) for n in (tq, tq, tr, tr)]
    F.fc_kv_gather_rope(r.view, rope, kp, vp, *apart[:2], None, None)
    F.fc_kv_gather_rope(r.view, rope, kp, vp, None, None, *apart[2:])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, apart))
    # gradients: to bf16 slices of a fused buffer, to fp32, and in place
    g = [r.randn(n, h, F32) for n, h in ((tq, r.hq), (tq, r.hkv), (tq, r.hkv), (tr, r.hkv), (tr, r.hkv))]
    f = r.nan(tq, r.hq + 2 * r.hkv)
    rec = [r.nan(tr, r.hkv) for _ in range(2)]
    F.fc_rope_bwd(r.view, rope, *g, *f.split([r.hq, r.hkv, r.hkv], 1), *rec)
    wide = [r.nan(*t.shape[:2], F32) for t in g]
    F.fc_rope_bwd(r.view, rope, *g, *wide)
    place = [t.clone() for t in g]
    F.fc_rope_bwd(r.view, rope, *place, *place)
    torch.cuda.synchronize()
    for got in ((*f.split([r.hq, r.hkv, r.hkv], 1), *rec), wide):
        for n, a, b, pos in zip(("dq", "dk_loc", "dv_loc", "dk_recv", "dv_recv"), got, g,
                                (*[r.pos[0]] * 3, *[r.pos[1]] * 2)):
            if n.startswith("dv"):
                assert torch.equal(a, b.to(a.dtype)), n
            else:
                check(f"{n} {a.dtype}", a, b, pos, w, inter, 1.25, back=True)
    assert all(torch.equal(a, b) for a, b in zip(wide, place))


@pytest.mark.parametrize("kw", [
    dict(lens=[1], cp=1, rank=0, hq=1, hkv=1, d=64), dict(lens=[1], cp=1, rank=0, hq=64, hkv=8, d=128),
    dict(lens=SHORT, cp=2, rank=0, hq=2, hkv=2, d=64), dict(lens=SHORT, cp=3, rank=2, hq=16, hkv=2, d=128),
    dict(lens=[1] * 300, cp=2, rank=1, hq=8, hkv=8, d=64, plan="whole_lpt"),
    dict(lens=[4096, 17, 2000], cp=8, rank=5, hq=32, hkv=8, d=128), dict(lens=[700, 1300], cp=3, rank=1, hq=12, hkv=3, d=64),
    dict(lens=[20000], cp=2, rank=1, hq=8, hkv=1, d=128),
])
@pytest.mark.parametrize("packed", [False, True])
def test_documents(kw, packed, dev):  # noqa: F811
    """Positions in documents of every length, and in the packed sequence; row counts
    on, below and above a workgroup's."""
    say(f"[gpu] rope documents {len(kw['lens'])} {kw} packed {packed}")
    r = Rank(dev, **kw)
    (tq, tr), T, m = r.sizes, int(r.c.cu[-1]), r.d // 2
    rope = F.Rope(m, packed_pos=packed)
    w = rope.inv_freq.tolist()
    pos = r.gpos if packed else r.pos
    q, qo = r.randn(tq, r.hq), r.nan(tq, r.hq)
    F.fc_rope_fwd(r.view, rope, q, None, None, qo, None, None)
    kp, vp = r.randn(T, r.hkv), r.randn(T, r.hkv)
    out = [r.nan(n, r.hkv) for n in (tq, tq, tr, tr)]
    F.fc_kv_gather_rope(r.view, rope, kp, vp, *out)
    torch.cuda.synchronize()
    check("q", qo, q, pos[0], w, False, 1.0)
    for i in (0, 1):
        check(f"k {i}", out[2 * i], kp[r.gpos[i]], pos[i], w, False, 1.0)
        assert torch.equal(out[2 * i + 1], vp[r.gpos[i]])
    # no rotation at all: the plain gather and copies
    ref = [r.nan(n, r.hkv) for n in (tq, tq, tr, tr)]
    F.fc_kv_gather(r.view, kp, vp, *ref)
    F.fc_kv_gather_rope(r.view, None, kp, vp, *out)
    F.fc_rope_fwd(r.view, None, q, None, None, qo, None, None)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, ref)) and torch.equal(qo, q)


def test_far_positions(dev):  # noqa: F811
    """A million tokens in, where an fp32 angle would be off by 0.06: a few of the
    last, rotated and rotated back."""
    n, own = 1000003, 40
    cu = np.array([0, n], dtype=np.int32)
    plan = np.array([[0, 1, 0, n - own], [0, 0, n - own, own]], dtype=np.int32)
    v = F.View(cu, plan, 2, 0, 2, 1, 64).bind(dev)
    g = torch.Generator(device=dev).manual_seed(1)
    pos = torch.arange(n - own, n, device=dev)
    for kw in (dict(), dict(scaling="yarn", factor=32.0, context=8192), dict(inv_freq=np.linspace(-8, 8, 32))):
        rope = F.Rope(64, **kw)
        w = rope.inv_freq.tolist()
        x = torch.randn(own, 2, 64, generator=g, device=dev)
        y = torch.empty_like(x)
        F.fc_rope_bwd(v, rope, x, None, None, None, None, y, None, None, None, None)
        torch.cuda.synchronize()
        check(str(kw), y, x, pos, w, False, rope.amplitude, back=True)
    v.close()


def test_edge_values(dev):  # noqa: F811
    """Infinities and NaN stay in their pair; the largest values do not overflow on
    the way; position 0 is the identity."""
    r = Rank(dev, lens=[40], cp=1, rank=0, hq=2, hkv=1, d=64)
    rope = F.Rope(64)
    q = r.randn(40, 2)
    q[3, 0, 5], q[7, 1, 40] = float("inf"), float("nan")
    big = float(torch.finfo(BF).max) / 2
    q[9] = big
    o = r.nan(40, 2)
    F.fc_rope_fwd(r.view, rope, q, None, None, o, None, None)
    torch.cuda.synchronize()
    assert torch.equal(o[0], q[0])
    bad = ~torch.isfinite(o)
    where = {tuple(i) for i in torch.nonzero(bad).tolist()}
    assert where and where <= {(3, 0, 5), (3, 0, 37), (7, 1, 8), (7, 1, 40)}
    # beside them, values that are not rotated stay as they are
    for m in (32, 24, 6):
        for inter in (False, True):
            x = r.randn(40, 2)
            x[:, :, m::2] = float("inf")
            o = r.nan(40, 2)
            F.fc_rope_fwd(r.view, F.Rope(m, interleaved=inter), x, None, None, o, None, None)
            torch.cuda.synchronize()
            assert torch.equal(o[..., m:], x[..., m:]) and torch.isfinite(o[..., :m]).all()


def test_refusals(dev):  # noqa: F811
    r = Rank(dev)
    tq, tr = r.sizes
    rope = F.Rope(64)
    q, qo = r.randn(tq, r.hq), r.nan(tq, r.hq)
    one = lambda *a: F.fc_rope_fwd(r.view, rope, *a)  # noqa: E731
    with pytest.raises(TypeError):
        one(q.float(), None, None, qo, None, None)
    with pytest.raises(TypeError):
        one(q.cpu(), None, None, qo, None, None)
    with pytest.raises(ValueError):
        one(q[:-1], None, None, qo, None, None)
    with pytest.raises(ValueError):
        one(q, None, None, None, None, None)
    with pytest.raises(ValueError):
        one(q.transpose(0, 1).contiguous().transpose(0, 1), None, None, qo, None, None)
    with pytest.raises(TypeError):
        F.fc_rope_bwd(r.view, rope, q.float(), None, None, None, None, qo.half(), None, None, None, None)
    for a, b in ((q, q[:, :].clone()), (q, q)):
        one(a, None, None, b, None, None)   # another tensor, and in place
    buf = torch.empty(tq + 1, r.hq, r.d, dtype=BF, device=dev)
    with pytest.raises(F.FlashCPError) as ei:
        one(buf[:-1], None, None, buf[1:], None, None)
    assert ei.value.code == -1
    with pytest.raises(F.FlashCPError) as ei:
        F.fc_rope_fwd(r.view, F.Rope(128), q, None, None, qo, None, None)
    assert ei.value.code == -1
    torch.cuda.synchronize()


def test_an_empty_rank(dev):  # noqa: F811
    v = F.View(np.array([0, 10], dtype=np.int32), [[0, 0, 0, 10]], 2, 1, 4, 2, 64, cap=5.0,
               slopes=np.ones(4)).bind(dev)
    e = lambda h, dt=BF: torch.empty(0, h, 64, dtype=dt, device=dev)  # noqa: E731
    rope = F.Rope(64)
    F.fc_rope_fwd(v, rope, e(4), e(2), e(2), e(4), e(2), e(2))
    k = torch.zeros(10, 2, 64, dtype=BF, device=dev)
    F.fc_kv_gather_rope(v, rope, k, k.clone(), e(2), e(2), e(2), e(2))
    F.fc_rope_bwd(v, rope, *[e(h, F32) for h in (4, 2, 2, 2, 2)], *[e(h) for h in (4, 2, 2, 2, 2)])
    torch.cuda.synchronize()


def test_captured_and_on_another_stream(dev):  # noqa: F811
    r = Rank(dev, hq=8, hkv=2, d=128)
    tq, tr = r.sizes
    rope = F.Rope(128)
    q, g = r.randn(tq, 8), r.randn(tq, 8, F32)
    kp, vp = r.randn(int(r.c.cu[-1]), 2), r.randn(int(r.c.cu[-1]), 2)
    outs = lambda: [r.nan(tq, 8), *[r.nan(n, 2) for n in (tq, tq, tr, tr)], r.nan(tq, 8)]  # noqa: E731

    def calls(o):
        F.fc_rope_fwd(r.view, rope, q, None, None, o[0], None, None)
        F.fc_kv_gather_rope(r.view, rope, kp, vp, *o[1:5])
        F.fc_rope_bwd(r.view, rope, g, None, None, None, None, o[5], None, None, None, None)

    want, got = outs(), outs()
    calls(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls(got)
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(got)
    for i in range(3):
        for t in got:
            t.fill_(float("nan"))
        rope = F.Rope(64)          # (frequencies went with the captured call)
        calls(outs())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("kind", ["cap", "bias"])
def test_a_training_step(kind, dev):  # noqa: F811
    """Projections in, their gradients out: rows out of the fused buffer, the rotated
    receive, attention with a score function, its backward, gradients rotated back
    into a fused bf16 buffer. The attention is checked against the oracle on the
    rotated bf16 rows the kernels made, the gradients through the rotation with the
    attention's own bounds."""
    lens, cp, rank, hq, hkv, d, m = [900, 37, 1500], 4, 2, 8, 2, 128, 64
    r = Rank(dev, lens=lens, cp=cp, rank=rank, hq=hq, hkv=hkv, d=d)
    (tq, tr), T = r.sizes, sum(lens)
    cap, slopes = (20.0, None) if kind == "cap" else (0.0, (2.0 ** -np.arange(1, hq + 1)).astype(np.float32))
    v = F.View(r.c.cu, r.c.plan, cp, rank, hq, hkv, d, cap=cap, slopes=slopes).bind(dev)
    rope = F.Rope(m, interleaved=kind == "bias", scaling="yarn", factor=4.0, context=512)
    w, amp = rope.inv_freq.tolist(), rope.amplitude
    packed = r.randn(T, hq + 2 * hkv)          # the whole sequence's projections
    packed[:, :hq] *= 3
    own = packed[r.gpos[0]]                    # the rank's own
    q, k, vals = r.nan(tq, hq), r.nan(tq, hkv), r.nan(tq, hkv)
    F.fc_rope_fwd(v, rope, *own.split([hq, hkv, hkv], 1), q, k, vals)
    kr, vr = r.nan(tr, hkv), r.nan(tr, hkv)
    F.fc_kv_gather_rope(v, rope, packed[:, hq:hq + hkv].contiguous(), packed[:, hq + hkv:].contiguous(), None,
                        None, kr, vr)
    o, o32, lse = r.nan(tq, hq), r.nan(tq, hq, F32), torch.empty(hq, tq, device=dev)
    fws, bws, _ = v.workspace_size()
    u8 = lambda n: torch.empty(max(n, 1), dtype=torch.uint8, device=dev)  # noqa: E731
    F.fc_attn_fwd(v, q, k, vals, kr, vr, 0.0, F.FC_TWO_PASS, o, o32, lse, u8(fws))
    do = r.randn(tq, hq)
    g = [r.nan(n, h, F32) for n, h in ((tq, hq), (tq, hkv), (tq, hkv), (tr, hkv), (tr, hkv))]
    F.fc_attn_bwd(v, q, k, vals, kr, vr, o, lse, do, 0.0, *g, u8(bws), o_f32=o32)
    f, rec = r.nan(tq, hq + 2 * hkv), [r.nan(tr, hkv) for _ in range(2)]
    F.fc_rope_bwd(v, rope, *g, *f.split([hq, hkv, hkv], 1), *rec)
    torch.cuda.synchronize()
    inter = kind == "bias"
    check("q", q, own[:, :hq], r.pos[0], w, inter, amp)
    check("k", k, own[:, hq:hq + hkv], r.pos[0], w, inter, amp)
    check("k_recv", kr, packed[r.gpos[1]][:, hq:hq + hkv], r.pos[1], w, inter, amp)
    assert torch.equal(vals, own[:, hq + hkv:]) and torch.equal(vr, packed[r.gpos[1]][:, hq + hkv:])
    want, b = S.attention(r.doc[0], r.pos[0], q, torch.cat(r.doc), torch.cat(r.pos), torch.cat([k, kr]),
                          torch.cat([vals, vr]), cap, slopes, do)
    near("o", o, want["o"], b["o"])
    near("lse", lse, want["lse"], b["lse"])
    for n, got, i, j in (("dq", f[:, :hq], 0, "dq"), ("dk", f[:, hq:hq + hkv], 0, "dk"), ("dk_recv", rec[0], 1, "dk")):
        cut = slice(None) if j == "dq" else slice(0, tq) if i == 0 else slice(tq, None)
        x = R.rotate(want[j][cut], r.pos[i], w, inter, amp, back=True)
        e = R.rotate_bound(b[j][cut], r.pos[i], w, inter, amp)
        near(n, got, x, e + 2.0 ** -8 * (x.abs() + e) + 2.0 ** -19 * x.abs().amax(-1, keepdim=True))
    for n, got, cut in (("dv", f[:, hq + hkv:], slice(0, tq)), ("dv_recv", rec[1], slice(tq, None))):
        near(n, got, want["dv"][cut], b["dv"][cut] + 2.0 ** -8 * (want["dv"][cut].abs() + b["dv"][cut]))


def test_another_device(dev):  # noqa: F811
    """Calls with a view, or tensors, of another device than the current one are refused."""
    class Elsewhere:
        def get_device(self):
            return dev_index + 1
    dev_index = torch.cuda.current_device()
    r = Rank(dev)
    q = r.randn(r.sizes[0], r.hq)
    meta, r.view.meta = r.view.meta, Elsewhere()
    none = [None] * 8
    for call in (lambda: F.fc_rope_fwd(r.view, None, q, None, None, q, None, None),
                 lambda: F.fc_kv_gather_rope(r.view, None, q, q, None, None, None, None),
                 lambda: F.fc_rope_bwd(r.view, None, q, *none[:4], q, *none[:4])):
        with pytest.raises(ValueError, match="device"):
            call()
    r.view.meta = meta
