"""Head norms against the fp64 oracle: the rank's own rows, the KV gather, gradients of
rows and weights, over layouts, types, strides, weights and positions. The oracle's
bounds count an fp32 implementation's roundings (oracle/norm.py)."""
import pytest
import torch

from oracle import norm as N
from paper_2606_08476_amd import flashcp as F
from test_gpu_parity import dev, say  # noqa: F401
from test_gpu_rope import SHORT, Rank

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def near(name, got, want, bound):
    e = (got.double() - want).abs()
    say(f"[gpu]   {name}: max {float(e.max()) if e.numel() else 0:.2e}")
    assert got.shape == want.shape and bool((e <= bound).all()), (name, float((e - bound).max()))


def weights(r, heads, dtype, per_head, offset):
    return (1 - offset + 0.5 * torch.randn(*((heads,) if per_head else ()), r.d, generator=r.gen,
                                          device=r.dev)).to(dtype)


def run_all(r, rope, wq, wk, scale=1.0, **kw):
    """Every call on the rank's rows, checked."""
    (tq, tr), T = r.sizes, int(r.c.cu[-1])
    inter = bool(rope and rope._c.interleaved)
    w, amp = (rope.inv_freq.tolist(), rope.amplitude) if rope else ((), 1.0)
    pos = r.gpos if rope and rope._c.packed_pos else r.pos
    ok = dict(w=w, inter=inter, amp=amp, **kw)
    qn, kn = F.HeadNorm(wq, **kw), F.HeadNorm(wk, **kw)
    x = r.randn(tq, r.hq + 2 * r.hkv) * scale
    q, k, v = x.split([r.hq, r.hkv, r.hkv], 1)
    qo, ko, vo = r.nan(tq, r.hq), r.nan(tq, r.hkv), r.nan(tq, r.hkv)
    F.fc_norm_rope_fwd(r.view, rope, qn, kn, q, k, v, qo, ko, vo)
    kp, vp = r.randn(T, r.hkv) * scale, r.randn(T, r.hkv)
    out = [r.nan(n, r.hkv) for n in (tq, tq, tr, tr)]
    F.fc_kv_gather_norm_rope(r.view, rope, kn, kp, vp, *out)
    # gradients: bf16 slices of a fused buffer; fp32; in place, own keys out of the packed ones
    g = [r.randn(n, h, F32) for n, h in ((tq, r.hq), (tq, r.hkv), (tq, r.hkv), (tr, r.hkv), (tr, r.hkv))]
    ws = torch.empty(max(F.fc_norm_rope_workspace(r.view, qn, kn), 1), dtype=torch.uint8, device=r.dev)
    dw = lambda: [torch.full_like(t, float("nan")) for t in (wq, wk)]  # noqa: E731
    f, rec, d1, d2, d3 = r.nan(tq, r.hq + 2 * r.hkv), [r.nan(tr, r.hkv) for _ in range(2)], dw(), dw(), dw()
    F.fc_norm_rope_bwd(r.view, rope, qn, kn, *g, *f.split([r.hq, r.hkv, r.hkv], 1), *rec, q, k, kp, *d1, ws)
    wide = [r.nan(*t.shape[:2], F32) for t in g]
    F.fc_norm_rope_bwd(r.view, rope, qn, kn, *g, *wide, q, k, kp, *d2, ws)
    place = [t.clone() for t in g]
    F.fc_norm_rope_bwd(r.view, rope, qn, kn, *place, *place, q, None, kp, *d3, ws)
    torch.cuda.synchronize()
    for name, got, src, wt, p in (("q", qo, q, wq, pos[0]), ("k", ko, k, wk, pos[0]),
                                  ("gathered k", out[0], kp[r.gpos[0]], wk, pos[0]),
                                  ("received k", out[2], kp[r.gpos[1]], wk, pos[1])):
        y, b = N.forward(src, wt, p, **ok)
        near(name, got, y, N.rounded(b, y, BF))
    assert torch.equal(vo, v) and torch.equal(out[1], vp[r.gpos[0]]) and torch.equal(out[3], vp[r.gpos[1]])
    dq = N.backward(g[0], q, wq, pos[0], **ok)
    dk = N.backward(g[1], k, wk, pos[0], **ok)
    dp = N.backward(g[1], kp[r.gpos[0]], wk, pos[0], **ok)
    dr = N.backward(g[3], kp[r.gpos[1]], wk, pos[1], **ok)
    for got in ((*f.split([r.hq, r.hkv, r.hkv], 1), *rec), wide, place):
        own = dp if got is place else dk
        for name, t, (dx, b, _, _) in (("dq", got[0], dq), ("dk", got[1], own), ("dk_recv", got[3], dr)):
            near(f"{name} {t.dtype}", t, dx, N.rounded(b, dx, t.dtype))
        assert torch.equal(got[2], g[2].to(got[2].dtype)) and torch.equal(got[4], g[4].to(got[4].dtype))
    for i, (wt, parts) in enumerate(((wq, [dq]), (wk, [dk, dr]), (wq, [dq]), (wk, [dp, dr]))):
        want, b = sum(p[2] for p in parts), sum(p[3] for p in parts)
        if wt.dim() == 1:
            want, b = want.sum(0), b.sum(0)
        near(f"dw {i}", (d1 if i < 2 else d3)[i % 2], want, N.rounded(b, want, wt.dtype))
    assert all(torch.equal(a, b) for a, b in zip(d1, d2)) and torch.equal(d1[0], d3[0])


@pytest.mark.parametrize("centred", [False, True])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d,m", [(64, 64), (64, 2), (64, 16), (64, 24), (64, 0), (128, 128), (128, 32), (128, 6),
                                 (128, 112), (128, 0)])
def test_layouts(d, m, inter, centred, dev):  # noqa: F811
    say(f"[gpu] norm d {d} rotated {m} interleaved {inter} centred {centred}")
    r = Rank(dev, d=d)
    rope = F.Rope(m, base=500.0, interleaved=inter, amplitude=1.25) if m else None
    per_head, offset = inter != centred, 1.0 if centred else 0.0
    dt = BF if inter else F32
    run_all(r, rope, weights(r, r.hq, dt, per_head, offset), weights(r, r.hkv, dt, not per_head, offset),
            offset=offset, centred=centred, eps=1e-5)


@pytest.mark.parametrize("kw", [
    dict(lens=[1], cp=1, rank=0, hq=1, hkv=1, d=64), dict(lens=[1], cp=1, rank=0, hq=64, hkv=8, d=128),
    dict(lens=SHORT, cp=2, rank=0, hq=2, hkv=2, d=64), dict(lens=SHORT, cp=3, rank=2, hq=16, hkv=2, d=128),
    dict(lens=[1] * 300, cp=2, rank=1, hq=8, hkv=8, d=64, plan="whole_lpt"),
    dict(lens=[4096, 17, 2000], cp=8, rank=5, hq=32, hkv=8, d=128), dict(lens=[700, 1300], cp=3, rank=1, hq=12, hkv=3, d=64),
    dict(lens=[600, 90], cp=2, rank=1, hq=40, hkv=5, d=128), dict(lens=[200], cp=2, rank=1, hq=72, hkv=36, d=64),
    dict(lens=[20000], cp=2, rank=1, hq=8, hkv=1, d=128),
])
@pytest.mark.parametrize("per_head", [False, True])
def test_documents(kw, per_head, dev):  # noqa: F811
    """Row counts on, below and above a workgroup's, heads that do not fill one, positions
    in documents and in the packed sequence."""
    say(f"[gpu] norm documents {len(kw['lens'])} {kw} per head {per_head}")
    r = Rank(dev, **kw)
    dt = F32 if per_head else BF
    run_all(r, F.Rope(r.d // 2, packed_pos=per_head), weights(r, r.hq, dt, per_head, 0),
            weights(r, r.hkv, dt, per_head, 0))


@pytest.mark.parametrize("centred", [False, True])
@pytest.mark.parametrize("scale", [2.0 ** -40, 2.0 ** -10, 2.0 ** 20, 2.0 ** 62, 2.0 ** 100, 2.0 ** 124])
def test_sizes_of_values(scale, centred, dev):  # noqa: F811
    """Rows so small that eps is all there is, and so large that their squares leave
    fp32."""
    say(f"[gpu] norm of values of {scale:.0e} centred {centred}")
    r = Rank(dev, lens=(40, 3), cp=1, rank=0)
    run_all(r, F.Rope(64), weights(r, r.hq, F32, False, 0), weights(r, r.hkv, F32, True, 0), scale=scale,
            centred=centred)


def test_edge_rows(dev):  # noqa: F811
    """A row of zeros, a constant row, one value only, and infinities or NaN, which stay in
    their head's row."""
    r = Rank(dev, lens=(40,), cp=1, rank=0)
    q = r.randn(40, r.hq)
    q[1, 0], q[2, 1], q[3, 2] = 0, 3.0, 0
    q[3, 2, 7] = 5.0
    w = weights(r, r.hq, F32, False, 0)
    for centred in (False, True):
        n = F.HeadNorm(w, centred=centred)
        clean, dirty = r.nan(40, r.hq), r.nan(40, r.hq)
        x = q.clone()
        x[9, 0, 5], x[11, 3, 40] = float("inf"), float("nan")
        F.fc_norm_rope_fwd(r.view, None, n, None, q, None, None, clean, None, None)
        F.fc_norm_rope_fwd(r.view, None, n, None, x, None, None, dirty, None, None)
        torch.cuda.synchronize()
        y, b = N.forward(q, w, r.pos[0], centred=centred)
        near("edge rows", clean, y, N.rounded(b, y, BF))
        same = torch.ones(40, r.hq, dtype=torch.bool, device=dev)
        same[9, 0] = same[11, 3] = False
        assert torch.equal(clean[same], dirty[same])
        assert torch.isnan(dirty[11, 3]).all() and torch.isnan(dirty[9, 0, 5])
        # backward: only their own rows, and the weights
        g, dx, ref = r.randn(40, r.hq, F32), r.nan(40, r.hq, F32), r.nan(40, r.hq, F32)
        for src, out in ((q, ref), (x, dx)):
            F.fc_norm_rope_bwd(r.view, None, n, None, g, *[None] * 4, out, *[None] * 4, src, None, None)
        torch.cuda.synchronize()
        assert torch.equal(dx[same], ref[same]) and torch.isfinite(ref).all()


def test_without_weights_and_one_tensor_at_a_time(dev):  # noqa: F811
    r = Rank(dev, hq=8, hkv=2, d=128)
    (tq, tr), T = r.sizes, int(r.c.cu[-1])
    rope, n = F.Rope(128), F.HeadNorm(None, eps=1e-5)
    q, k, v, kp = r.randn(tq, 8), r.randn(tq, 2), r.randn(tq, 2), r.randn(T, 2)
    one = F.HeadNorm(torch.ones(128, device=dev), eps=1e-5)
    a, b = ([r.nan(tq, 8), r.nan(tq, 2), r.nan(tq, 2)] for _ in range(2))
    F.fc_norm_rope_fwd(r.view, rope, n, n, q, k, v, *a)
    F.fc_norm_rope_fwd(r.view, rope, one, None, q, None, None, b[0], None, None)
    F.fc_norm_rope_fwd(r.view, rope, None, one, None, k, v, None, b[1], b[2])
    # no norm at all: the rotation's own rows
    c, d = ([r.nan(tq, 8), r.nan(tq, 2)] for _ in range(2))
    F.fc_norm_rope_fwd(r.view, rope, None, None, q, k, None, *c, None)
    F.fc_rope_fwd(r.view, rope, q, k, None, *d, None)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and all(torch.equal(x, y) for x, y in zip(c, d))
    # gradients: each tensor by itself gives its rows, and its part of the weights'
    g = [r.randn(n_, h, F32) for n_, h in ((tq, 8), (tq, 2), (tr, 2))]
    ws = torch.empty(F.fc_norm_rope_workspace(r.view, one, one), dtype=torch.uint8, device=dev)
    outs = [r.nan(*t.shape[:2]) for t in g]
    dq, dk = (torch.empty(128, device=dev) for _ in range(2))
    F.fc_norm_rope_bwd(r.view, rope, one, one, g[0], g[1], None, g[2], None, outs[0], outs[1], None, outs[2], None,
                       q, k, kp, dq, dk, ws)
    parts, alone = [], [r.nan(*t.shape[:2]) for t in g]
    for i in range(3):
        gi = [None] * 5
        oi = [None] * 5
        j = (0, 1, 3)[i]
        gi[j], oi[j] = g[i], alone[i]
        p = torch.empty(128, device=dev)
        F.fc_norm_rope_bwd(r.view, rope, one, one, *gi, *oi, q, k, kp, *((p, None) if i == 0 else (None, p)), ws)
        parts.append(p)
    zero = torch.full((128,), float("nan"), device=dev)
    F.fc_norm_rope_bwd(r.view, rope, one, one, g[0], *[None] * 4, r.nan(tq, 8), *[None] * 4, q, None, None, None, zero,
                       ws)
    bare = r.nan(tq, 8)
    F.fc_norm_rope_bwd(r.view, rope, n, None, g[0], *[None] * 4, bare, *[None] * 4, q, None, None)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(outs, alone)) and torch.equal(bare, outs[0])
    assert torch.equal(zero, torch.zeros_like(zero))
    # (the sums are taken in other orders: the oracle's bound of either)
    for got, want, parts_of in ((dq, parts[0], [(g[0], q, 0)]), (dk, parts[1] + parts[2], [(g[1], k, 0), (g[2], kp[r.gpos[1]], 1)])):
        b = sum(N.backward(y, x, one.weight, r.pos[i], w=rope.inv_freq.tolist(), eps=1e-5)[3].sum(0) for y, x, i in parts_of)
        near("dw of parts", got, want.double(), 2 * N.rounded(b, want.double(), F32) + 2.0 ** -23 * want.abs())


def test_refusals(dev):  # noqa: F811
    r = Rank(dev)
    tq, tr = r.sizes
    n = F.HeadNorm(torch.ones(64, device=dev))
    q, qo, g = r.randn(tq, r.hq), r.nan(tq, r.hq), r.randn(tq, r.hq, F32)
    one = lambda w, a=q, o=qo: F.fc_norm_rope_fwd(r.view, None, w, None, a, None, None, o, None, None)  # noqa: E731
    for shape in ((32,), (3, 64), (1, 4, 64)):
        with pytest.raises(ValueError):
            one(F.HeadNorm(torch.ones(shape, device=dev)))
    with pytest.raises(ValueError):
        F.HeadNorm(torch.ones(64, 4, device=dev).t())
    with pytest.raises(TypeError):
        F.HeadNorm(torch.ones(64, device=dev, dtype=torch.float16))
    with pytest.raises(TypeError):
        one(n, q.float())
    for bad in (F.HeadNorm(n.weight, eps=0.0), F.HeadNorm(n.weight, eps=float("nan")), F.HeadNorm(n.weight, offset=float("inf"))):
        with pytest.raises(F.FlashCPError) as e:
            one(bad)
        assert e.value.code == -1
    back = lambda *a, **k: F.fc_norm_rope_bwd(r.view, None, n, None, g, *[None] * 4, qo, *[None] * 4, *a, **k)  # noqa: E731
    with pytest.raises(F.FlashCPError) as e:
        back(None, None, None)                        # the rows are needed
    assert e.value.code == -1
    dw = torch.empty(64, device=dev)
    with pytest.raises(F.FlashCPError) as e:
        back(q, None, None, dw_q=dw)                  # no workspace
    assert e.value.code == -5
    ws = torch.empty(F.fc_norm_rope_workspace(r.view, n, None), dtype=torch.uint8, device=dev)
    for bad in (dw.to(BF), dw[:32], torch.empty(4, 64, device=dev)):
        with pytest.raises((TypeError, ValueError)):
            back(q, None, None, dw_q=bad, ws=ws)
    with pytest.raises(ValueError):
        back(q, None, None, dw_k=dw, ws=ws)           # no such norm
    torch.cuda.synchronize()


def test_an_empty_rank(dev):  # noqa: F811
    v = F.View([0, 10], [[0, 0, 0, 10]], 2, 1, 4, 2, 64).bind(dev)
    e = lambda h, dt=BF: torch.empty(0, h, 64, dtype=dt, device=dev)  # noqa: E731
    rope, n = F.Rope(64), F.HeadNorm(torch.ones(64, device=dev))
    F.fc_norm_rope_fwd(v, rope, n, n, e(4), e(2), e(2), e(4), e(2), e(2))
    k = torch.zeros(10, 2, 64, dtype=BF, device=dev)
    F.fc_kv_gather_norm_rope(v, rope, n, k, k.clone(), e(2), e(2), e(2), e(2))
    dq, dk = (torch.full((64,), float("nan"), device=dev) for _ in range(2))
    ws = torch.empty(max(F.fc_norm_rope_workspace(v, n, n), 1), dtype=torch.uint8, device=dev)
    F.fc_norm_rope_bwd(v, rope, n, n, *[e(h, F32) for h in (4, 2, 2, 2, 2)], *[e(h) for h in (4, 2, 2, 2, 2)], e(4),
                       e(2), k, dq, dk, ws)
    torch.cuda.synchronize()
    assert not dq.any() and not dk.any()


def test_captured_and_on_another_stream(dev):  # noqa: F811
    """Two graphs with workspaces of their own, replayed among eager calls: weights are
    read when a call runs."""
    r = Rank(dev, hq=8, hkv=2, d=128)
    (tq, tr), T = r.sizes, int(r.c.cu[-1])
    rope, wq, wk = F.Rope(128), weights(r, 8, BF, False, 0), weights(r, 2, F32, True, 0)
    qn, kn = F.HeadNorm(wq), F.HeadNorm(wk)
    q, kp, vp, gq, gk = r.randn(tq, 8), r.randn(T, 2), r.randn(T, 2), r.randn(tq, 8, F32), r.randn(tr, 2, F32)
    outs = lambda: [r.nan(tq, 8), *[r.nan(n, 2) for n in (tq, tq, tr, tr)], r.nan(tq, 8), r.nan(tr, 2),  # noqa: E731
                    torch.full_like(wq, float("nan")), torch.full_like(wk, float("nan")),
                    torch.empty(F.fc_norm_rope_workspace(r.view, qn, kn), dtype=torch.uint8, device=dev)]

    def calls(o):
        F.fc_norm_rope_fwd(r.view, rope, qn, None, q, None, None, o[0], None, None)
        F.fc_kv_gather_norm_rope(r.view, rope, kn, kp, vp, *o[1:5])
        F.fc_norm_rope_bwd(r.view, rope, qn, kn, gq, None, None, gk, None, o[5], None, None, o[6], None, q, None, kp,
                           o[7], o[8], o[9])

    want, got = outs(), outs()
    calls(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls(got)
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want[:9], got[:9]))
    pairs = []
    for _ in range(2):
        o, graph = outs(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls(o)
        pairs.append((o, graph))
    for i in range(3):
        wq.add_(0.25)
        wk.mul_(1.5)
        for o, _ in pairs:
            for t in o[:9]:
                t.fill_(float("nan"))
        calls(want)
        torch.cuda.synchronize()
        for _, graph in pairs:
            graph.replay()
        calls(want)
        torch.cuda.synchronize()
        for o, _ in pairs:
            assert all(torch.equal(a, b) for a, b in zip(want[:9], o[:9]))


def test_another_device(dev):  # noqa: F811
    class Elsewhere:
        def get_device(self):
            return dev_index + 1
    dev_index = torch.cuda.current_device()
    r = Rank(dev)
    q = r.randn(r.sizes[0], r.hq)
    meta, r.view.meta = r.view.meta, Elsewhere()
    none = [None] * 8
    for call in (lambda: F.fc_norm_rope_fwd(r.view, None, None, None, q, None, None, q, None, None),
                 lambda: F.fc_kv_gather_norm_rope(r.view, None, None, q, q, None, None, None, None),
                 lambda: F.fc_norm_rope_bwd(r.view, None, None, None, q, *none[:4], q, *none[:4], q, None, None)):
        with pytest.raises(ValueError, match="device"):
            call()
    r.view.meta = meta
