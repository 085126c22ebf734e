"""Attention in sliding windows with sinks (windowed views): every entry point against
the fp64 oracle and against the others, alone and with capped scores and slopes.

Bounds are the oracle's (oracle/scores.py), as for scored views; where the same sums
run in another order, 2e-5 of the largest value, as for plain views."""
import numpy as np
import pytest
import torch

import _cases
from oracle import scores as S
from paper_2606_08476_amd import flashcp as F
from test_gpu_parity import dev, say  # noqa: F401
from test_gpu_scores import BF, F32, ORDER_TOL, SHORT, near, slopes_of

pytestmark = pytest.mark.gpu

SHAPES = {
    "one_token": dict(lens=[1, 1], cp=1, rank=0, hq=1, hkv=1, d=64),
    "short_g4": dict(lens=SHORT, cp=2, rank=1, hq=8, hkv=2, d=128),
    "short_g1_d64": dict(lens=SHORT, cp=2, rank=0, hq=2, hkv=2, d=64),
    "mixed_g1_d64": dict(lens=[700, 1300, 48], cp=2, rank=0, hq=4, hkv=4, d=64),
    "mixed_g8_d64": dict(lens=[700, 1300, 48], cp=3, rank=1, hq=16, hkv=2, d=64),
    "mixed_g2": dict(lens=[900, 37, 1500], cp=4, rank=2, hq=8, hkv=4, d=128),
    "mixed_g4": dict(lens=[900, 37, 1500], cp=4, rank=3, hq=8, hkv=2, d=128),
    "mixed_g4_bm64": dict(lens=[900, 37, 1500], cp=4, rank=0, hq=8, hkv=2, d=128, tiles=(64, 0, 0, 0)),
    "mixed_g4_bm128": dict(lens=[900, 37, 1500], cp=4, rank=3, hq=8, hkv=2, d=128, tiles=(128, 0, 0, 0)),
    "mixed_g2_d64": dict(lens=[900, 37, 1500], cp=4, rank=2, hq=4, hkv=2, d=64),
    "aligned_g1": dict(lens=[512, 1024, 256], cp=2, rank=0, hq=2, hkv=2, d=128),
    "per_seq_g4_d64": dict(lens=[300, 37, 1500, 11], cp=3, rank=1, hq=8, hkv=2, d=64, plan="per_seq"),
    "local_g8": dict(lens=[640, 129, 1, 70], cp=1, rank=0, hq=8, hkv=1, d=128, plan="whole_lpt"),
    "split_g8": dict(lens=[9001, 1, 70], cp=8, rank=7, hq=8, hkv=1, d=128),
    "split_g4": dict(lens=[9001, 1, 70], cp=8, rank=7, hq=4, hkv=1, d=128),
    "split_g2_d64": dict(lens=[6001, 1, 77, 300], cp=4, rank=3, hq=4, hkv=2, d=64),
    "split_g1": dict(lens=[6007, 1, 130, 300], cp=4, rank=3, hq=2, hkv=2, d=128),
}
WINDOWS = [(1, 0), (1, 3), (64, 0), (100, 4), (128, 128), (300, 65), (700, 200)]
SPLIT = [(2000, 0), (2500, 100), (4096, 4)]
# cap, slopes, what queries are scaled by
KINDS = {"plain": (0.0, False, 3.0), "cap30": (30.0, False, 6.0), "cap55": (55.0, False, 30.0),
         "cap56": (56.0, False, 30.0), "bias": (0.0, True, 3.0), "cap30_bias": (30.0, True, 3.0)}
CASES = [(s, w, "plain") for s in SHAPES for w in (SPLIT if s.startswith("split") else WINDOWS)]
CASES += [(s, w, k) for s, w in (("short_g4", (5, 2)), ("mixed_g1_d64", (100, 4)), ("mixed_g8_d64", (300, 65)),
                                 ("mixed_g2", (130, 0)), ("mixed_g4", (700, 200)), ("mixed_g4_bm64", (64, 1)),
                                 ("mixed_g2_d64", (99, 7)), ("aligned_g1", (128, 128)), ("mixed_g4_bm128", (100, 4)),
                                 ("split_g8", (2000, 4)), ("split_g4", (2500, 100)), ("split_g2_d64", (2000, 4)),
                                 ("split_g1", (2500, 0))) for k in KINDS if k != "plain"]


class Run:
    """One case's inputs, bound view and forward, and the oracle's answer."""

    def __init__(self, shape, win, kind, dev, tail=0):
        kw = dict(SHAPES[shape]) if isinstance(shape, str) else dict(shape)
        kw.setdefault("plan", "per_doc")
        self.case = c = _cases.make_case(str(shape), "llama8b", seed=3, **kw)
        self.cap, biased, q_std = KINDS[kind]
        self.slopes = slopes_of(c.hq) if biased else None
        self.win = win
        if tail:
            c.plan = np.array([x for i, n in enumerate(kw["lens"]) for x in
                               ([i, 0, 0, max(n - tail, 0)], [i, 1, max(n - tail, 0), min(n, tail)]) if x[3]],
                              dtype=np.int32)
        self.view = F.View(c.cu, c.plan, c.cp, c.rank, c.hq, c.hkv, c.d, tiles=c.tiles, cap=self.cap,
                           slopes=self.slopes, window=win[0], sinks=win[1]).bind(dev)
        self.dev = dev
        e = self.view.export()
        cu = np.asarray(c.cu)
        g = [e["q_gpos"].astype(np.int64), e["recv_gpos"].astype(np.int64)]
        self.tq, self.tr = len(g[0]), len(g[1])
        doc = [np.searchsorted(cu, a, side="right") - 1 for a in g]
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)  # noqa: E731
        self.doc = [t(a) for a in doc]
        self.pos = [t(a - cu[b]) for a, b in zip(g, doc)]
        gen = torch.Generator(device=dev).manual_seed(sum(kw["lens"]) + win[0])
        r = lambda n, h: torch.randn(n, h, c.d, generator=gen, device=dev, dtype=BF)  # noqa: E731
        self.q, self.do = r(self.tq, c.hq) * q_std, r(self.tq, c.hq)
        self.kv = [r(self.tq, c.hkv), r(self.tq, c.hkv), r(self.tr, c.hkv), r(self.tr, c.hkv)]

    def nan(self, *s, dt=F32):
        return torch.full(s, float("nan"), dtype=dt, device=self.dev)

    def u8(self, n):
        return torch.empty(max(n, 1), dtype=torch.uint8, device=self.dev)

    def outs(self):
        c = self.case
        return self.nan(self.tq, c.hq, c.d, dt=BF), self.nan(self.tq, c.hq, c.d), self.nan(c.hq, self.tq)

    def forward(self, mode, ws=True):
        o, o32, lse = self.outs()
        F.fc_attn_fwd(self.view, self.q, *self.kv, 0.0, mode, o, o32, lse,
                      self.u8(self.view.workspace_size(mode)[0]) if ws else None)
        return o, o32, lse

    def partial(self, src, view=None):
        c = self.case
        op, lp = self.nan(self.tq, c.hq, c.d), self.nan(c.hq, self.tq)
        F.fc_attn_fwd_partial(view or self.view, src, self.q, *self.kv[2 * src:2 * src + 2], 0.0, op, lp)
        return op, lp

    def partials(self, view=None):
        c = self.case
        out = [f(*s) for f in (self.nan,) for s in 2 * [(self.tq, c.hq, c.d), (c.hq, self.tq)]]
        F.fc_attn_fwd_partials(view or self.view, self.q, *self.kv, 0.0, *out)
        return out

    def grads(self):
        c = self.case
        return [self.nan(self.tq, c.hq, c.d)] + [self.nan(n, c.hkv, c.d) for n in
                                                 (self.tq, self.tq, self.tr, self.tr)]

    def oracle(self, srcs=(0, 1), dout=None, **kw):
        k = torch.cat([self.kv[2 * i] for i in srcs])
        v = torch.cat([self.kv[2 * i + 1] for i in srcs])
        return S.attention(self.doc[0], self.pos[0], self.q, torch.cat([self.doc[i] for i in srcs]),
                           torch.cat([self.pos[i] for i in srcs]), k, v, self.cap, self.slopes, dout,
                           window=self.win[0], sinks=self.win[1], **kw)


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def check_grads(name, r, got, want, b):
    tq = r.tq
    for n, t, w, e in (("dq", got[0], want["dq"], b["dq"]), ("dk", got[1], want["dk"][:tq], b["dk"][:tq]),
                       ("dv", got[2], want["dv"][:tq], b["dv"][:tq]), ("dk_recv", got[3], want["dk"][tq:], b["dk"][tq:]),
                       ("dv_recv", got[4], want["dv"][tq:], b["dv"][tq:])):
        near(f"{name} {n}", t, w, e)


def close(a, b):
    """The same sums in another order."""
    for x, y in zip(a, b):
        if x.numel():
            assert float((x - y).abs().max()) <= ORDER_TOL * float(y.abs().max())


@pytest.mark.parametrize("shape,win,kind", CASES)
def test_windowed_views(shape, win, kind, dev):  # noqa: F811
    say(f"[gpu] window {shape} {win} {kind}")
    r = Run(shape, win, kind, dev)
    c, v = r.case, r.view
    want, b = r.oracle(dout=r.do)
    two, one = r.forward(F.FC_TWO_PASS), r.forward(F.FC_FUSED)
    for n, (o, o32, lse) in (("two", two), ("one", one)):
        near(f"{n} o", o, want["o"], b["o"])
        near(f"{n} o32", o32, want["o"], b["o32"])
        near(f"{n} lse", lse, want["lse"], b["lse"])
    # the partial passes: rows that see nothing of a source too; together and apart, over
    # the tables alone: the same bits, and their merge the two-pass forward's
    both = r.partials()
    bare = F.View(c.cu, c.plan, c.cp, c.rank, c.hq, c.hkv, c.d, tiles=c.tiles, cap=r.cap, slopes=r.slopes,
                  window=win[0], sinks=win[1]).bind(dev, slots=False)
    apart = [*r.partial(0), *(r.partial(1) if r.tr else both[2:])]
    tables = [*r.partial(0, bare), *(r.partial(1, bare) if r.tr else both[2:])]
    assert same(both, apart) and same(both, tables) and same(both, r.partials(bare))
    for src, (op, lp) in enumerate((both[:2], both[2:])):
        w, e = r.oracle(srcs=(src,))
        near(f"partial {src} o", op, w["o"], e["o32"])
        near(f"partial {src} lse", lp, w["lse"], e["lse"])
    m = r.outs()
    F.fc_lse_merge(*both, *m)
    torch.cuda.synchronize()
    assert same(m, two)
    # backward: one launch, dK/dV and dQ alone, with less workspace, with atomics, without allocation
    o, o32, lse = two
    ws = r.u8(v.workspace_size()[1])
    g, again = r.grads(), r.grads()
    for out in (g, again):
        F.fc_attn_bwd(v, r.q, *r.kv, o, lse, r.do, 0.0, *out, ws, o_f32=o32)
    torch.cuda.synchronize()
    assert same(g, again)
    check_grads("bwd", r, g, want, b)
    delta = r.nan(c.hq, r.tq)
    F.fc_bwd_preprocess(v, None, r.do, delta, o_f32=o32)
    kv, dq = r.grads(), r.nan(r.tq, c.hq, c.d)
    F.fc_attn_bwd_dkdv(v, r.q, *r.kv, lse, delta, r.do, 0.0, *kv[1:], ws)
    F.fc_attn_bwd_dq(v, r.q, *r.kv, lse, delta, r.do, 0.0, dq)
    at = r.grads()
    F.fc_attn_bwd(v, r.q, *r.kv, o, lse, r.do, 0.0, *at, ws, deterministic=False, o_f32=o32)
    torch.cuda.synchronize()
    assert same(kv[1:], g[1:])
    near("dq alone", dq, want["dq"], b["dq"])
    check_grads("atomic", r, at, want, b)
    close(at[1:], g[1:])
    if v.workspace_size()[1] <= F.NOALLOC_SCRATCH_BYTES:
        na = r.grads()
        F.fc_attn_bwd_noalloc(v, r.q, *r.kv, o, lse, r.do, 0.0, *na, o_f32=o32)
        torch.cuda.synchronize()
        assert same(na, g)
    # unsplit, where the view is split
    if v.export_split()["fwd_chunk"] and shape.startswith("split"):
        u = r.forward(F.FC_FUSED, ws=False)
        near("unsplit o", u[0], want["o"], b["o"])
        near("unsplit lse", u[2], want["lse"], b["lse"])
        part = 2 * v.info["n_bwd_slots"] * c.hkv * 128 * c.d * 4
        short = r.grads()
        F.fc_attn_bwd_pass(v, r.q, *r.kv, lse, delta, r.do, 0.0, *short, r.u8(part))
        torch.cuda.synchronize()
        assert same(short[1:], g[1:]) and torch.equal(short[0], dq)
    bare.close()


def test_split_views_are_among_them(dev):  # noqa: F811
    """Of the cases above: forward chunks and dQ parts with a gap between sinks and window."""
    n = 0
    for shape, win, kind in CASES:
        if shape.startswith("split") and kind == "plain":
            r = Run(shape, win, kind, dev)
            s = r.view.export_split()
            n += bool(s["fwd_chunk"]) and len(s["dq_comb"]) > 0
    assert n >= 6


def test_views_that_see_everything(dev):  # noqa: F811
    """A window that reaches every key, and one that almost does: the full view's bits, and
    nearly so."""
    r = Run("mixed_g4", (100000, 7), "plain", dev)
    c = r.case
    full = F.View(c.cu, c.plan, c.cp, c.rank, c.hq, c.hkv, c.d).bind(dev)
    a = r.forward(F.FC_TWO_PASS)
    o = r.outs()
    F.fc_attn_fwd(full, r.q, *r.kv, 0.0, F.FC_TWO_PASS, *o, r.u8(full.workspace_size()[0]))
    torch.cuda.synchronize()
    assert same(a, o)


@pytest.mark.parametrize("tail", [1, 3, 40])
@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (8, 1, 128), (4, 4, 64)])
def test_last_tokens(tail, hq, hkv, d, dev):  # noqa: F811
    """New tokens at the ends of long and short documents: a decoding step, or a draft's."""
    say(f"[gpu] window last tokens {tail} {hq} {hkv} {d}")
    shape = dict(lens=[20000, 1, 5, 7001, 300, 4100], cp=2, rank=1, hq=hq, hkv=hkv, d=d)
    for win in ((4096, 4), (1, 0), (1000, 70)):
        r = Run(shape, win, "plain", dev, tail=tail)
        want, b = r.oracle(dout=r.do)
        for mode in (F.FC_TWO_PASS, F.FC_FUSED):
            o, o32, lse = r.forward(mode)
            near("o", o, want["o"], b["o"])
            near("lse", lse, want["lse"], b["lse"])
        g = r.grads()
        o, o32, lse = r.forward(F.FC_TWO_PASS)
        F.fc_attn_bwd(r.view, r.q, *r.kv, o, lse, r.do, 0.0, *g, r.u8(r.view.workspace_size()[1]), o_f32=o32)
        torch.cuda.synchronize()
        check_grads("bwd", r, g, want, b)


def test_masked_keys_do_not_matter(dev):  # noqa: F811
    """Keys that a row does not see may hold anything finite, and the largest values there
    are: a row's result has the same bits."""
    r = Run("mixed_g4_bm64", (100, 4), "plain", dev)   # (its rank has the documents' ends)
    a = r.forward(F.FC_FUSED)
    near_rows = (r.doc[0] == 2) & (r.pos[0] >= 1400)   # the last rows of the last document
    for i, src in ((0, 0), (2, 1)):
        far = (r.doc[src] == 2) & (r.pos[src] < 1300) & (r.pos[src] >= 4)
        r.kv[i][far] = 3e4
        r.kv[i + 1][far] = float(torch.finfo(BF).max)
    b = r.forward(F.FC_FUSED)
    torch.cuda.synchronize()
    assert near_rows.any() and same([a[0][near_rows], a[2][:, near_rows]], [b[0][near_rows], b[2][:, near_rows]])


def test_differences(dev):  # noqa: F811
    """Gradients against differences of the forward: along random directions, halves of
    differences of fp64 oracle values as the kernels' own forward rounds too much."""
    r = Run("short_g4", (5, 2), "cap30", dev)
    o, o32, lse = r.forward(F.FC_TWO_PASS)
    g = r.grads()
    F.fc_attn_bwd(r.view, r.q, *r.kv, o, lse, r.do, 0.0, *g, r.u8(r.view.workspace_size()[1]), o_f32=o32)
    gen = torch.Generator(device=dev).manual_seed(1)
    h = 1e-4
    leaves = [r.q, r.kv[0], r.kv[1], r.kv[2], r.kv[3]]
    for i, (x, grad) in enumerate(zip(leaves, g)):
        u = torch.randn(x.shape, generator=gen, device=dev, dtype=torch.float64)
        val = []
        for sgn in (1, -1):
            y = [t.double() for t in leaves]
            y[i] = y[i] + sgn * h * u
            want, _ = S.attention(r.doc[0], r.pos[0], y[0], torch.cat(r.doc), torch.cat(r.pos),
                                  torch.cat([y[1], y[3]]), torch.cat([y[2], y[4]]), r.cap, None, None, window=5, sinks=2)
            val.append(float((want["o"] * r.do.double()).sum()))
        fd = (val[0] - val[1]) / (2 * h)
        # (each gradient's own error, 2^-8 of it at most, averages out along u; the step's
        # third-order term is h^2 of the value)
        tol = 2.0 ** -8 * float((grad.double() * u).norm()) * 4 + 1e-5 * abs(fd)
        assert abs(fd - float((grad.double() * u).sum())) <= tol, (i, fd, tol)


def test_captured_and_on_another_stream(dev):  # noqa: F811
    """A step captured twice, with workspaces of its own each, replayed among eager ones."""
    r = Run("split_g4", (2500, 100), "plain", dev)
    c, v = r.case, r.view

    def buffers():
        return (r.outs(), r.grads(), r.partials(), r.u8(v.workspace_size()[0]), r.u8(v.workspace_size()[1]))

    def step(x):
        (o, o32, lse), g, parts, fws, bws = x
        F.fc_attn_fwd(v, r.q, *r.kv, 0.0, F.FC_TWO_PASS, o, o32, lse, fws)
        F.fc_attn_fwd_partials(v, r.q, *r.kv, 0.0, *parts)
        F.fc_attn_bwd(v, r.q, *r.kv, o, lse, r.do, 0.0, *g, bws, o_f32=o32)
        return [o, o32, lse, *g, *parts]

    want = step(buffers())
    side = torch.cuda.Stream()
    x = buffers()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = step(x)
    torch.cuda.synchronize()
    assert same(want, got)
    graphs = []
    for _ in range(2):
        x, graph = buffers(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step(x)
        graphs.append((graph, got, x))
    eager = buffers()
    for i in range(3):
        r.q.mul_(1.25 if i else 1.0)
        r.kv[3].add_(0.5)
        want = step(eager)
        for _, got, _ in graphs:
            for t in got:
                t.fill_(float("nan"))
        torch.cuda.synchronize()
        for graph, _, _ in graphs:
            graph.replay()
        again = step(buffers())
        torch.cuda.synchronize()
        assert same(want, again)
        for _, got, _ in graphs:
            assert same(want, got)


@pytest.mark.parametrize("cap,window,sinks,hq,hkv,d", [(0.0, 300, 4, 8, 2, 128), (30.0, 64, 0, 4, 4, 64)])
def test_a_training_step(cap, window, sinks, hq, hkv, d, dev):  # noqa: F811
    """Projections in, their gradients out, as a layer runs: queries normalised and
    rotated, the windowed view's receive set gathered with its keys', attention, its
    backward, gradients back through rotation and norm, with those of the weights. Each
    operator is checked on the rows the one before it made."""
    from oracle import norm as N
    lens, cp, rank = [900, 37, 1500], 4, 2
    c = _cases.make_case("step", "llama8b", lens=lens, cp=cp, rank=rank, hq=hq, hkv=hkv, d=d, plan="per_doc")
    v = F.View(c.cu, c.plan, cp, rank, hq, hkv, d, cap=cap, window=window, sinks=sinks).bind(dev)
    e, cu = v.export(), np.asarray(c.cu)
    tok = [torch.from_numpy(e[n].astype(np.int64)).to(dev) for n in ("q_gpos", "recv_gpos")]
    doc = [torch.from_numpy(np.searchsorted(cu, e[n], side="right") - 1).to(dev) for n in ("q_gpos", "recv_gpos")]
    pos = [t - torch.from_numpy(cu.astype(np.int64)).to(dev)[b] for t, b in zip(tok, doc)]
    tq, tr = v.info["t_q"], v.info["t_recv"]
    assert 0 < tr < len(c.oview.recv_gpos)      # less is received than without a window
    gen = torch.Generator(device=dev).manual_seed(window)
    rnd = lambda *s, dt=BF: torch.randn(*s, generator=gen, device=dev, dtype=dt)  # noqa: E731
    rope = F.Rope(d // 2, interleaved=d == 64)
    w = rope.inv_freq.tolist()
    wq, wk = (1 + 0.3 * rnd(d, dt=F32)).to(BF), 0.3 * rnd(hkv, d, dt=F32)
    qn, kn = F.HeadNorm(wq), F.HeadNorm(wk, offset=1.0)
    xq, kp, vp, do = rnd(tq, hq, d), rnd(sum(lens), hkv, d), rnd(sum(lens), hkv, d), rnd(tq, hq, d)
    nan = lambda *s, dt=BF: torch.full(s, float("nan"), device=dev, dtype=dt)  # noqa: E731
    u8 = lambda n: torch.empty(max(n, 1), dtype=torch.uint8, device=dev)  # noqa: E731
    q, kv = nan(tq, hq, d), [nan(n, hkv, d) for n in (tq, tq, tr, tr)]
    F.fc_norm_rope_fwd(v, rope, qn, None, xq, None, None, q, None, None)
    F.fc_kv_gather_norm_rope(v, rope, kn, kp, vp, *kv)
    o, o32, lse = nan(tq, hq, d), nan(tq, hq, d, dt=F32), nan(hq, tq, dt=F32)
    fws, bws, _ = v.workspace_size()
    F.fc_attn_fwd(v, q, *kv, 0.0, F.FC_TWO_PASS, o, o32, lse, u8(fws))
    g = [nan(n, h, d, dt=F32) for n, h in ((tq, hq), (tq, hkv), (tq, hkv), (tr, hkv), (tr, hkv))]
    F.fc_attn_bwd(v, q, *kv, o, lse, do, 0.0, *g, u8(bws), o_f32=o32)
    dx, dwq, dwk = [nan(*t.shape) for t in g], torch.empty_like(wq), torch.empty_like(wk)
    F.fc_norm_rope_bwd(v, rope, qn, kn, *g, *dx, xq, None, kp, dwq, dwk, u8(F.fc_norm_rope_workspace(v, qn, kn)))
    torch.cuda.synchronize()
    ok = dict(w=w, inter=d == 64)
    for n, got, x, wt, p, off in (("q", q, xq, wq, pos[0], 0.0), ("k", kv[0], kp[tok[0]], wk, pos[0], 1.0),
                                  ("k_recv", kv[2], kp[tok[1]], wk, pos[1], 1.0)):
        y, b = N.forward(x, wt, p, offset=off, **ok)
        near(n, got, y, N.rounded(b, y, BF))
    assert torch.equal(kv[1], vp[tok[0]]) and torch.equal(kv[3], vp[tok[1]])
    want, b = S.attention(doc[0], pos[0], q, torch.cat(doc), torch.cat(pos), torch.cat([kv[0], kv[2]]),
                          torch.cat([kv[1], kv[3]]), cap, None, do, window=window, sinks=sinks)
    near("o", o, want["o"], b["o"])
    near("lse", lse, want["lse"], b["lse"])
    for n, got, key, cut in (("dq", g[0], "dq", slice(None)), ("dk", g[1], "dk", slice(0, tq)),
                             ("dv", g[2], "dv", slice(0, tq)), ("dk_recv", g[3], "dk", slice(tq, None)),
                             ("dv_recv", g[4], "dv", slice(tq, None))):
        near(n, got, want[key][cut], b[key][cut])
    parts = []
    for n, got, dy, x, wt, p, off in (("dxq", dx[0], g[0], xq, wq, pos[0], 0.0),
                                      ("dxk", dx[1], g[1], kp[tok[0]], wk, pos[0], 1.0),
                                      ("dxk_recv", dx[3], g[3], kp[tok[1]], wk, pos[1], 1.0)):
        y, e_, dw, be = N.backward(dy, x, wt, p, offset=off, **ok)
        near(n, got, y, N.rounded(e_, y, BF))
        parts.append((dw, be))
    near("dwq", dwq, parts[0][0].sum(0), N.rounded(parts[0][1].sum(0), parts[0][0].sum(0), BF))
    dk, be = parts[1][0] + parts[2][0], parts[1][1] + parts[2][1]
    near("dwk", dwk, dk, N.rounded(be, dk, F32))
