"""Attention with capped scores and a distance bias (views with a score function):
every entry point against the fp64 oracle and against the others.

Each output element is held to the oracle's own bound for it (oracle/scores.py:
the roundings of products, P, dX, O and the score function, summed over the keys),
and the 2-norm of the error to 2^-8 of the result's, half of what it would be if
every rounding were as large as it can be (an O that is rounded twice, and
gradients whose P and dX are), or to a quarter of the bounds' norm where these are
wide (a partial pass whose every key is thousands of steep slopes away). Where the same sums run in another order, 2e-5 of
the largest value, as for plain views."""
import numpy as np
import pytest
import torch

import _cases
from oracle import scores as S
from paper_2606_08476_amd import flashcp as F
from test_gpu_parity import dev, say  # noqa: F401

pytestmark = pytest.mark.gpu

NORM_TOL, ORDER_TOL = 2.0 ** -8, 2e-5
BF, F32 = torch.bfloat16, torch.float32

SHORT = [1, 1, 3, 1, 70, 1, 2, 129, 1, 64, 5, 250, 1, 31]
SHAPES = {
    "one_token": dict(lens=[1], cp=1, rank=0, hq=1, hkv=1, d=64),
    "short_g4": dict(lens=SHORT, cp=2, rank=1, hq=8, hkv=2, d=128),
    "short_g1_d64": dict(lens=SHORT, cp=2, rank=0, hq=2, hkv=2, d=64),
    "mixed_g1_d64": dict(lens=[700, 1300, 48], cp=2, rank=0, hq=4, hkv=4, d=64),
    "mixed_g8_d64": dict(lens=[700, 1300, 48], cp=3, rank=1, hq=16, hkv=2, d=64),
    "mixed_g2": dict(lens=[900, 37, 1500], cp=4, rank=2, hq=8, hkv=4, d=128),
    "mixed_g4_bm64": dict(lens=[900, 37, 1500], cp=4, rank=3, hq=8, hkv=2, d=128, tiles=(64, 0, 0, 0)),
    "mixed_g4_bm128": dict(lens=[900, 37, 1500], cp=4, rank=3, hq=8, hkv=2, d=128, tiles=(128, 0, 0, 0)),
    "mixed_g2_d64": dict(lens=[900, 37, 1500], cp=4, rank=2, hq=4, hkv=2, d=64),
    "aligned_g1": dict(lens=[512, 1024, 256], cp=2, rank=0, hq=2, hkv=2, d=128),
    "per_seq_g4_d64": dict(lens=[300, 37, 1500, 11], cp=3, rank=1, hq=8, hkv=2, d=64, plan="per_seq"),
    "local_g8": dict(lens=[640, 129, 1, 70], cp=1, rank=0, hq=8, hkv=1, d=128, plan="whole_lpt"),
    # long key ranges split over workgroups
    "split_g8": dict(lens=[9001, 1, 70], cp=8, rank=7, hq=8, hkv=1, d=128),
    "split_g4": dict(lens=[9001, 1, 70], cp=8, rank=7, hq=4, hkv=1, d=128),
    "split_g2_d64": dict(lens=[6001, 1, 77, 300], cp=4, rank=3, hq=4, hkv=2, d=64),
    "split_g1": dict(lens=[6007, 1, 130, 300], cp=4, rank=3, hq=2, hkv=2, d=128),
}
# cap, slopes, what queries are scaled by (scores well over the cap for the small
# caps, far below it for the largest)
KINDS = {
    "cap30": (30.0, False, 6.0),
    "cap2": (2.0, False, 3.0),
    "cap55": (55.0, False, 30.0),
    "cap56": (56.0, False, 30.0),
    "cap1024": (1024.0, False, 1.0),
    "bias": (0.0, True, 3.0),
    "cap30_bias": (30.0, True, 3.0),
    # every head steep: most keys of longer documents are out of reach, and skipped
    "steep": (0.0, "steep", 1.0),
    "cap30_steep": (30.0, "steep", 1.0),
}
LONG = [s for s in SHAPES if s.startswith(("split", "mixed"))]
CASES = [(s, k) for s in SHAPES for k in KINDS if k in ("cap30", "bias", "cap30_bias") or s in
         ("short_g4", "mixed_g1_d64", "split_g4") or ("steep" in k and s in LONG)]


def slopes_of(hq):
    """Geometric, the first head's 0 and the last head's the steepest a view takes."""
    s = 2.0 ** (-8.0 * np.arange(1, hq + 1) / hq)
    s[0] = 0.0
    if hq > 2:
        s[-1] = F.SLOPE_MAX
    return s.astype(np.float32)


class Run:
    """One case's inputs, bound view and forward, and the oracle's answer."""

    def __init__(self, shape, kind, dev):
        kw = dict(SHAPES[shape])
        kw.setdefault("plan", "per_doc")
        self.case = c = _cases.make_case(shape, "llama8b", seed=3, **kw)
        self.cap, biased, q_std = KINDS[kind]
        self.slopes = None
        if biased:
            # steep: a quarter to 2 per token
            self.slopes = slopes_of(c.hq) if biased is True else np.linspace(0.25, 2.0, c.hq).astype(np.float32)
        x = {n: t.to(dev) for n, t in _cases.inputs(c).items()}
        self.q, self.do = x["q"] * q_std, x["do"]
        self.kv = [x[n].contiguous() for n in ("k_loc", "v_loc", "k_recv", "v_recv")]
        self.view = F.View(c.cu, c.plan, c.cp, c.rank, c.hq, c.hkv, c.d, tiles=c.tiles, cap=self.cap,
                           slopes=self.slopes).bind(dev)
        self.dev = dev
        i = self.view.info
        self.tq, self.tr = i["t_q"], i["t_recv"]
        ov, cu = c.oview, np.asarray(c.cu)
        g = [np.asarray(a, dtype=np.int64) for a in (ov.q_gpos, ov.recv_gpos)]
        doc = [np.searchsorted(cu, a, side="right") - 1 for a in g]
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)  # noqa: E731
        self.doc = [t(a) for a in doc]
        self.pos = [t(a - cu[b]) for a, b in zip(g, doc)]

    def nan(self, *s, dt=F32):
        return torch.full(s, float("nan"), dtype=dt, device=self.dev)

    def forward(self, mode):
        c, v = self.case, self.view
        o, o32 = self.nan(self.tq, c.hq, c.d, dt=BF), self.nan(self.tq, c.hq, c.d)
        lse = self.nan(c.hq, self.tq)
        ws = torch.empty(max(v.workspace_size(mode)[0], 1), dtype=torch.uint8, device=self.dev)
        F.fc_attn_fwd(v, self.q, *self.kv, 0.0, mode, o, o32, lse, ws)
        return o, o32, lse

    def grads(self):
        c = self.case
        return [self.nan(self.tq, c.hq, c.d)] + [self.nan(n, c.hkv, c.d) for n in
                                                 (self.tq, self.tq, self.tr, self.tr)]

    def oracle(self, srcs=(0, 1), dout=None, **kw):
        k = torch.cat([self.kv[2 * i] for i in srcs])
        v = torch.cat([self.kv[2 * i + 1] for i in srcs])
        return S.attention(self.doc[0], self.pos[0], self.q, torch.cat([self.doc[i] for i in srcs]),
                           torch.cat([self.pos[i] for i in srcs]), k, v, self.cap, self.slopes, dout, **kw)


def near(name, got, want, bound):
    """got within bound of want everywhere, and within NORM_TOL of it in norm."""
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fine), f"{name}: finite elsewhere"
    e = torch.where(fine, (got.double() - want).abs(), 0.0)
    over = float((e - bound).max()) if e.numel() else 0.0
    norm = float(torch.where(fine, want, 0.0).norm())
    rel = float(e.norm()) / norm if norm else 0.0
    say(f"[gpu]   {name}: max {float(e.max()) if e.numel() else 0:.2e} rel {rel:.2e} over bound {over:.1e}")
    assert over <= 0, f"{name}: {over:.3e} over its bound"
    # (few values average nothing: theirs is the bound above)
    assert rel <= NORM_TOL or float(e.norm()) <= float(bound.norm()) / 4 or e.numel() < 4096, \
        f"{name}: {rel:.3e} off in norm"


@pytest.mark.parametrize("shape,kind", CASES)
def test_scored_views(shape, kind, dev):  # noqa: F811
    say(f"[gpu] scores {shape} {kind}")
    r = Run(shape, kind, dev)
    c, v, tq, tr = r.case, r.view, r.tq, r.tr
    split = v.export_split()
    if shape.startswith("split"):
        assert split["fwd_chunk"] and len(split["dq_comb"])
    if "steep" in kind and max(SHAPES[shape]["lens"]) > 700:
        plain = F.View(c.cu, c.plan, c.cp, c.rank, c.hq, c.hkv, c.d, tiles=c.tiles)
        assert v.workspace_size()[0] > plain.workspace_size()[0]   # row norms
    want, bnd = r.oracle(dout=r.do)

    # the forward, two passes and one
    o, o32, lse = r.forward(F.FC_TWO_PASS)
    of, of32, lsef = r.forward(F.FC_FUSED)
    torch.cuda.synchronize()
    for n, a, a32, l in (("two-pass", o, o32, lse), ("fused", of, of32, lsef)):
        near(f"{n} o", a, want["o"], bnd["o"])
        near(f"{n} o32", a32, want["o"], bnd["o32"])
        near(f"{n} lse", l, want["lse"], bnd["lse"])

    # the partial passes, each against the oracle, both at once the same bits, and
    # their merge the two-pass forward's
    parts = []
    for src in (0, 1):
        op, lp = r.nan(tq, c.hq, c.d), r.nan(c.hq, tq)
        F.fc_attn_fwd_partial(v, src, r.q, *r.kv[2 * src:2 * src + 2], 0.0, op, lp)
        torch.cuda.synchronize()
        w, b = r.oracle(srcs=(src,))
        near(f"partial {src} o", op, w["o"], b["o32"])
        near(f"partial {src} lse", lp, w["lse"], b["lse"])
        parts += [op, lp]
    both = [r.nan(tq, c.hq, c.d), r.nan(c.hq, tq), r.nan(tq, c.hq, c.d), r.nan(c.hq, tq)]
    F.fc_attn_fwd_partials(v, r.q, *r.kv, 0.0, *both)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(parts, both))
    ob, om, lm = r.nan(tq, c.hq, c.d, dt=BF), r.nan(tq, c.hq, c.d), r.nan(c.hq, tq)
    F.fc_lse_merge(*both, ob, om, lm)
    torch.cuda.synchronize()
    if tr:
        assert torch.equal(ob, o) and torch.equal(om, o32) and torch.equal(lm, lse)

    # the backward: deterministic, from the fp32 O and from the bf16 one
    ws = torch.empty(v.workspace_size()[1], dtype=torch.uint8, device=dev)
    names = ("dq", "dk_loc", "dv_loc", "dk_recv", "dv_recv")
    pieces = lambda t: (t["dq"], t["dk"][:tq], t["dv"][:tq], t["dk"][tq:], t["dv"][tq:])  # noqa: E731
    det = r.grads()
    F.fc_attn_bwd(v, r.q, *r.kv, o, lse, r.do, 0.0, *det, ws, o_f32=o32)
    torch.cuda.synchronize()
    for n, a, w, b in zip(names, det, pieces(want), pieces(bnd)):
        near(n, a, w, b)
    from_bf = r.grads()
    F.fc_attn_bwd(v, r.q, *r.kv, o, lse, r.do, 0.0, *from_bf, ws)
    torch.cuda.synchronize()
    _, bnd16 = r.oracle(dout=r.do, delta_from_bf16=True)
    for n, a, w, b in zip(names, from_bf, pieces(want), pieces(bnd16)):
        assert float(((a.double() - w).abs() - b).max() if a.numel() else 0) <= 0, n

    # in steps, and each kernel alone
    delta = r.nan(c.hq, tq)
    F.fc_bwd_preprocess(v, o, r.do, delta, o_f32=o32)
    wp = torch.empty(max(v.workspace_size()[2], 1), dtype=torch.uint8, device=dev)
    step = r.grads()
    F.fc_attn_bwd_pass(v, r.q, *r.kv, lse, delta, r.do, 0.0, *step, wp)
    alone = r.grads()
    F.fc_attn_bwd_dkdv(v, r.q, *r.kv, lse, delta, r.do, 0.0, *alone[1:], wp)
    F.fc_attn_bwd_dq(v, r.q, *r.kv, lse, delta, r.do, 0.0, alone[0])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(step, det))
    assert all(torch.equal(a, b) for a, b in zip(alone[1:], det[1:]))
    far = lambda a, b: float((a - b).abs().max()) <= ORDER_TOL * max(1.0, float(b.abs().max()))  # noqa: E731
    # (steep: dQ alone has no row norms, and visits every key)
    same = not len(split["dq_comb"]) and "steep" not in kind
    assert torch.equal(alone[0], det[0]) if same else far(alone[0], det[0])

    # without room for row norms, every key is visited: the same to rounding
    if "steep" in kind:
        wo = torch.empty(max(v.workspace_size()[2] - 1024, 1), dtype=torch.uint8, device=dev)
        whole = r.grads()
        F.fc_attn_bwd_pass(v, r.q, *r.kv, lse, delta, r.do, 0.0, *whole, wo)
        torch.cuda.synchronize()
        assert all(far(a, b) for a, b in zip(whole, det) if a.numel())

    # without allocation, and with dQ by atomics
    if v.workspace_size()[1] <= F.NOALLOC_SCRATCH_BYTES:
        na = r.grads()
        F.fc_attn_bwd_noalloc(v, r.q, *r.kv, o, lse, r.do, 0.0, *na, o_f32=o32)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(na, det))
    at = r.grads()
    F.fc_attn_bwd(v, r.q, *r.kv, o, lse, r.do, 0.0, *at, ws, deterministic=False, o_f32=o32)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(at[1:], det[1:]))
    near("dq by atomics", at[0], want["dq"], bnd["dq"])
    v.close()


@pytest.mark.parametrize("kind", ["cap30_bias", "bias"])
def test_far_into_a_document(kind, dev):  # noqa: F811
    """Queries a million tokens into a document: their shares of the biases are tens
    of thousands, of which the keys' shares leave a few."""
    n, own, hq, d = 1000003, 130, 4, 64
    cu = np.array([0, n], dtype=np.int32)
    plan = np.array([[0, 1, 0, n - own], [0, 0, n - own, own]], dtype=np.int32)
    cap, _, q_std = KINDS[kind]
    slopes = np.array([2.0 ** -12, 0.013, 0.1, 1.3], dtype=np.float32)
    v = F.View(cu, plan, 2, 0, hq, 1, d, cap=cap, slopes=slopes).bind(dev)
    i = v.info
    assert (i["t_q"], i["t_recv"]) == (own, n - own)
    g = torch.Generator(device=dev).manual_seed(1)
    e = lambda m, h: torch.randn(m, h, d, generator=g, device=dev, dtype=BF)  # noqa: E731
    q, do, kl, vl, kr, vr = q_std * e(own, hq), e(own, hq), e(own, 1), e(own, 1), e(n - own, 1), e(n - own, 1)
    doc = lambda m: torch.zeros(m, dtype=torch.int64, device=dev)  # noqa: E731
    pos = torch.arange(n, device=dev)
    want, bnd = S.attention(doc(own), pos[n - own:], q, doc(n), torch.cat([pos[n - own:], pos[:n - own]]),
                            torch.cat([kl, kr]), torch.cat([vl, vr]), cap, slopes, do)
    o, o32 = torch.empty(own, hq, d, dtype=BF, device=dev), torch.empty(own, hq, d, device=dev)
    lse = torch.empty(hq, own, device=dev)
    fws, bws, _ = v.workspace_size()
    u8 = lambda m: torch.empty(max(m, 1), dtype=torch.uint8, device=dev)  # noqa: E731
    F.fc_attn_fwd(v, q, kl, vl, kr, vr, 0.0, F.FC_TWO_PASS, o, o32, lse, u8(fws))
    z = lambda m, h: torch.empty(m, h, d, device=dev)  # noqa: E731
    for det in (True, False):
        gr = [z(own, hq), z(own, 1), z(own, 1), z(n - own, 1), z(n - own, 1)]
        F.fc_attn_bwd(v, q, kl, vl, kr, vr, o, lse, do, 0.0, *gr, u8(bws), deterministic=det, o_f32=o32)
        torch.cuda.synchronize()
        near("o", o, want["o"], bnd["o"])
        near("lse", lse, want["lse"], bnd["lse"])
        near("dq", gr[0], want["dq"], bnd["dq"])
        for a, b, name in ((gr[1], gr[3], "dk"), (gr[2], gr[4], "dv")):
            near(name, torch.cat([a, b]), want[name], bnd[name])
    v.close()


def test_no_slope_and_a_wide_cap_are_the_plain_view(dev):  # noqa: F811
    """Slopes of 0, or a cap far over the scores, leave the plain result: x - cap
    tanh(x / cap) is below |x|^3 / (3 cap^2), here 6^3 / (3 * 2^20) = 7e-5."""
    r = Run("mixed_g2", "cap1024", dev)
    c = r.case
    plain = F.View(c.cu, c.plan, c.cp, c.rank, c.hq, c.hkv, c.d).bind(dev)
    flat = F.View(c.cu, c.plan, c.cp, c.rank, c.hq, c.hkv, c.d, slopes=np.zeros(c.hq)).bind(dev)
    wide, res = r.view, []
    for r.view in (plain, flat, wide):
        res.append(r.forward(F.FC_TWO_PASS))
    torch.cuda.synchronize()
    for o, o32, lse in res[1:]:
        # (P's roundings to bf16 may fall on either side: twice half a step of |v| <= 6)
        assert float((o32 - res[0][1]).abs().max()) <= 6 * 2.0 ** -7
        assert float((lse - res[0][2]).abs().max()) <= 2e-3
    r.view = wide


def test_captured_and_on_another_stream(dev):  # noqa: F811
    """A scored forward and backward captured into a graph and replayed between
    eager work, and run on a side stream: the eager bits."""
    for shape in ("mixed_g4_bm64", "split_g4"):
        r = Run(shape, "cap30_bias", dev)
        c, v = r.case, r.view
        o, o32, lse = r.forward(F.FC_TWO_PASS)
        fws, bws, _ = v.workspace_size()
        u8 = lambda m: torch.empty(max(m, 1), dtype=torch.uint8, device=dev)  # noqa: E731
        want = r.grads()
        F.fc_attn_bwd(v, r.q, *r.kv, o, lse, r.do, 0.0, *want, u8(bws), o_f32=o32)
        torch.cuda.synchronize()
        co, co32, cl, cg = torch.empty_like(o), torch.empty_like(o32), torch.empty_like(lse), r.grads()
        w1, w2 = u8(fws), u8(bws)

        def calls():
            F.fc_attn_fwd(v, r.q, *r.kv, 0.0, F.FC_TWO_PASS, co, co32, cl, w1)
            F.fc_attn_bwd(v, r.q, *r.kv, co, cl, r.do, 0.0, *cg, w2, o_f32=co32)

        def same():
            return all(torch.equal(a, b) for a, b in zip((o, o32, lse, *want), (co, co32, cl, *cg)))

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            calls()
        side.synchronize()
        assert same()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls()
        for _ in range(3):
            for t in (co32, cl, *cg):
                t.fill_(float("nan"))
            r.forward(F.FC_FUSED)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert same()
        v.close()


def test_every_rank_together_is_the_whole(dev):  # noqa: F811
    """All ranks of a plan, each with its received keys, give the unsharded result
    (one rank that holds everything) to the order of their sums."""
    lens, cp, hq, hkv, d = [500, 1, 777, 90], 4, 4, 2, 64
    slopes = slopes_of(hq)[::-1].copy() * 0.5
    whole = _cases.make_case("whole", "tiny", lens=lens, cp=1, rank=0, hq=hq, hkv=hkv, d=d, plan="per_doc")
    x = {n: t.to(dev) for n, t in _cases.inputs(whole).items()}
    q, k, v = 4 * x["q"], x["k_pk"], x["v_pk"]

    def run(case):
        view = F.View(case.cu, case.plan, case.cp, case.rank, hq, hkv, d, cap=20.0, slopes=slopes).bind(dev)
        i = view.info
        e = lambda n, h, dt=BF: torch.empty(n, h, d, dtype=dt, device=dev)  # noqa: E731
        kv = e(i["t_q"], hkv), e(i["t_q"], hkv), e(i["t_recv"], hkv), e(i["t_recv"], hkv)
        F.fc_kv_gather(view, k, v, *kv)
        g = torch.from_numpy(np.asarray(case.oview.q_gpos, dtype=np.int64)).to(dev)
        o, o32, lse = e(g.numel(), hq), e(g.numel(), hq, F32), torch.empty(hq, g.numel(), device=dev)
        ws = torch.empty(max(view.workspace_size()[0], 1), dtype=torch.uint8, device=dev)
        F.fc_attn_fwd(view, q[g].contiguous(), *kv, 0.0, F.FC_TWO_PASS, o, o32, lse, ws)
        torch.cuda.synchronize()
        view.close()
        return g, o32, lse

    _, O, L = run(whole)
    pos = torch.cat([torch.arange(n) for n in lens]).to(dev)
    doc = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(lens)).to(dev)
    _, b = S.attention(doc, pos, q, doc, pos, k, v, 20.0, slopes)
    seen = torch.zeros(sum(lens), dtype=torch.int64)
    for plan in ("per_doc", "whole_lpt", "per_seq"):
        for r in range(cp):
            case = _cases.make_case(plan, "tiny", lens=lens, cp=cp, rank=r, hq=hq, hkv=hkv, d=d, plan=plan)
            g, o, l = run(case)
            seen[g.cpu()] += 1
            assert bool(((o - O[g]).abs() <= 2 * b["o32"][g]).all())
            assert bool(((l - L[:, g]).abs() <= 2 * b["lse"][:, g]).all())
    assert bool((seen == 3).all())


@pytest.mark.parametrize("lens,cp,rank,hq,hkv,d,cap", [
    # one long document, heads of very different reach: the far reaching ones first
    ([60000], 8, 7, 32, 32, 64, 0.0), ([60000], 8, 7, 32, 8, 128, 30.0),
    # documents of all lengths: heads in turn
    ([9000, 40, 3000, 700, 1, 5000, 2000, 260], 2, 1, 32, 8, 128, 0.0),
    ([9000, 40, 3000, 700, 1, 5000, 2000, 260], 2, 0, 6, 6, 64, 30.0),
])
def test_out_of_reach(lens, cp, rank, hq, hkv, d, cap, dev):  # noqa: F811
    """Calls with room for row norms, which leave out keys out of reach, against the
    same without (every key): what is left out is 2^-76 of a row, so the results are
    the same but for the order of sums."""
    c = _cases.make_case("reach", "llama8b", lens=lens, cp=cp, rank=rank, hq=hq, hkv=hkv, d=d, plan="per_doc")
    slopes = (2.0 ** (-8.0 * np.arange(1, hq + 1) / hq)).astype(np.float32)
    v = F.View(c.cu, c.plan, cp, rank, hq, hkv, d, cap=cap, slopes=slopes).bind(dev)
    norms = 256 * 4 * (hq + 2 * hkv)
    plain = F.View(c.cu, c.plan, cp, rank, hq, hkv, d)
    assert v.workspace_size(F.FC_FUSED)[0] >= norms + (0 if plain.export_split()["fwd_chunk"] else
                                                       plain.workspace_size(F.FC_FUSED)[0])
    tq, tr = v.info["t_q"], v.info["t_recv"]
    g = torch.Generator(device=dev).manual_seed(7)
    e = lambda n, h: torch.randn(n, h, d, generator=g, device=dev, dtype=BF)  # noqa: E731
    q, do = e(tq, hq), e(tq, hq)
    # (queries of several sizes, one of which reaches far beyond the others)
    q *= torch.tensor([0.25, 1.0, 3.0], device=dev)[torch.arange(tq, device=dev) % 3][:, None, None].to(BF)
    q[tq // 2] *= 20
    kv = e(tq, hkv), e(tq, hkv), e(tr, hkv), e(tr, hkv)
    z = lambda *s, dt=F32: torch.full(s, float("nan"), device=dev, dtype=dt)  # noqa: E731

    def run(short):
        out = []
        for mode in (F.FC_TWO_PASS, F.FC_FUSED):
            o, o32, lse = z(tq, hq, d, dt=BF), z(tq, hq, d), z(hq, tq)
            n = v.workspace_size(mode)[0] - (256 if short else 0)
            F.fc_attn_fwd(v, q, *kv, 0.0, mode, o, o32, lse, torch.empty(n, dtype=torch.uint8, device=dev))
            out += [o32, lse]
        delta = z(hq, tq)
        F.fc_bwd_preprocess(v, None, do, delta, o_f32=out[0])
        n = v.workspace_size()[2] - (256 if short else 0)
        ws = torch.empty(n, dtype=torch.uint8, device=dev)
        for det in (True, False):
            gr = [z(tq, hq, d), z(tq, hkv, d), z(tq, hkv, d), z(tr, hkv, d), z(tr, hkv, d)]
            F.fc_attn_bwd_pass(v, q, *kv, out[1], delta, do, 0.0, *gr, ws, deterministic=det)
            out += gr
        torch.cuda.synchronize()
        return out

    for i, (a, b) in enumerate(zip(run(False), run(True))):
        assert torch.isfinite(a).all() and torch.isfinite(b).all()
        far = float((a - b).abs().max()) if a.numel() else 0.0
        say(f"[gpu]   output {i}: {far:.1e} of {float(b.abs().max()) if b.numel() else 0:.1e}")
        assert far <= ORDER_TOL * max(1.0, float(b.abs().max()) if b.numel() else 0.0), i
    v.close()


def test_nothing_is_out_of_reach_of_a_nan(dev):  # noqa: F811
    """A key that is not a number makes every row that sees it not one, near or far,
    as it does where every key is visited."""
    cu, cp, rank, hq, hkv, d = np.array([0, 9000, 12000], dtype=np.int32), 1, 0, 8, 2, 64
    c = _cases.make_case("nan", "llama8b", lens=[9000, 3000], cp=cp, rank=rank, hq=hq, hkv=hkv, d=d, plan="per_doc")
    slopes = np.full(hq, 0.5, dtype=np.float32)
    v = F.View(c.cu, c.plan, cp, rank, hq, hkv, d, cap=30.0, slopes=slopes).bind(dev)
    tq = v.info["t_q"]
    assert v.workspace_size(F.FC_FUSED)[0] >= 256 * 4 * (hq + 2 * hkv)
    g = torch.Generator(device=dev).manual_seed(7)
    q, k, w = (torch.randn(tq, h, d, generator=g, device=dev, dtype=BF) for h in (hq, hkv, hkv))
    k[20, 1] = float("nan")
    none = torch.empty(0, hkv, d, dtype=BF, device=dev)
    o, o32 = torch.zeros(tq, hq, d, dtype=BF, device=dev), torch.zeros(tq, hq, d, device=dev)
    lse = torch.zeros(hq, tq, device=dev)
    ws = torch.empty(v.workspace_size(F.FC_FUSED)[0], dtype=torch.uint8, device=dev)
    F.fc_attn_fwd(v, q, k, w, none, none, 0.0, F.FC_FUSED, o, o32, lse, ws)
    torch.cuda.synchronize()
    want = torch.zeros(tq, hq, dtype=torch.bool, device=dev)
    want[20:cu[1], hq // hkv:] = True
    assert torch.equal(torch.isnan(o32).all(-1), want) and torch.equal(torch.isnan(o32).any(-1), want)
    # (the LSE of a row with no finite scores says nothing, in any view: inputs are finite)
    assert bool(torch.isfinite(lse.T[~want]).all())
    v.close()


def test_norms_follow_the_inputs(dev):  # noqa: F811
    """A captured forward and backward that leave keys out of reach, replayed after their
    inputs have grown (more keys are then within reach), and the same on two streams at
    once, each with a workspace of its own: the eager bits."""
    r = Run("split_g4", "steep", dev)
    v = r.view
    fws, bws, _ = v.workspace_size()
    assert fws >= 256 * 4 * (r.case.hq + 2 * r.case.hkv)
    u8 = lambda m: torch.empty(m, dtype=torch.uint8, device=dev)  # noqa: E731

    def calls(out, w1, w2):
        o, o32, l, *g = out
        F.fc_attn_fwd(v, r.q, *r.kv, 0.0, F.FC_TWO_PASS, o, o32, l, w1)
        F.fc_attn_bwd(v, r.q, *r.kv, o, l, r.do, 0.0, *g, w2, o_f32=o32)

    def outs():
        return [r.nan(r.tq, r.case.hq, r.case.d, dt=BF), r.nan(r.tq, r.case.hq, r.case.d),
                r.nan(r.case.hq, r.tq), *r.grads()]

    got, w = outs(), (u8(fws), u8(bws))
    calls(got, *w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(got, *w)
    for grow in (1.0, 8.0, 4.0):
        r.q.mul_(grow)
        r.kv[2].mul_(grow)  # (received keys)
        want = outs()
        calls(want, u8(fws), u8(bws))
        torch.cuda.synchronize()
        assert all(bool(torch.isfinite(t).all()) for t in want)
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        side = [torch.cuda.Stream() for _ in range(2)]
        both = [(outs(), u8(fws), u8(bws)) for _ in side]
        torch.cuda.synchronize()
        for s, b in zip(side, both):
            with torch.cuda.stream(s):
                calls(*b)
        torch.cuda.synchronize()
        for b in both:
            assert all(torch.equal(x, y) for x, y in zip(want, b[0]))
    v.close()
