"""Head norms with the rotation and windowed attention, whose speed is followed, as a
training or serving program calls them through ``paper_2606_08476_amd.flashcp``,
beside their plain forms in elementary torch operations.

A case is a packed sequence of documents (recipe, context, length seed), a shard
plan's rank, a head configuration and a ``kind``:

* ``rows``    the rank's own rows out of a fused projection buffer
              [T_q, Hq + 2 Hkv, d]: queries and keys normalised per head and rotated,
              values copied;
* ``gather``  the KV gather with the keys normalised and rotated on the way: own and
              received rows;
* ``grads``   the gradients of rotated, normalised queries and of own and received
              keys back to the projection's rows (bf16 or fp32), those of the values
              rounded only, and those of both norms' weights;
* ``forward`` the one-pass windowed forward over given rows (bf16 O, fp32 LSE);
* ``layer``   one training layer: queries normalised and rotated, the KV gather with
              the keys', two-pass windowed forward, backward preprocess, deterministic
              backward, and the gradients of ``grads``.

A query sees the last ``window`` tokens of its document up to itself and the first
``sinks`` tokens of the document (window 0: every earlier token); a rank receives
the keys that its queries see. Scores are capped by cap * tanh(x / cap) (0: not
capped). With ``centred`` the norms subtract the mean first; ``per_head``: each head
has weights of its own; ``offset``: what is added to the weights. The first ``rot``
values of each head are rotated by the position in the document (0: none). ``tail``
tokens at each document's end are rank 1's (0: every document in 2 cp chunks).
"""
import math

import numpy as np
import torch

own = False

BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def _case(name, kind, recipe, context, len_seed, cp, rank, hq, hkv, d, window=0, sinks=0, tail=0, rot=None,
          inter=False, base=10000.0, centred=False, per_head=False, offset=0.0, eps=1e-6, w_bf16=True, cap=0.0,
          q_std=1.0, bf16=True):
    c = dict(kind=kind, recipe=recipe, context=context, len_seed=len_seed, cp=cp, rank=rank, hq=hq, hkv=hkv, d=d,
             window=window, sinks=sinks, tail=tail, rot=d if rot is None else rot, inter=inter, base=base,
             centred=centred, per_head=per_head, offset=offset, eps=eps, w_bf16=w_bf16, cap=cap, q_std=q_std,
             bf16=bf16)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest call: a 2K sequence on two ranks, launches and latency count
        _case("rows_tiny", "rows", "tiny", 2048, 1, 2, 0, 4, 4, 64),
        # own rows of the headline shape: 64K tokens of mixed documents, 8 ranks
        _case("rows_llama8b", "rows", "mixed", 65536, 2, 8, 3, 32, 8, 128, base=500000.0),
        # a late rank of 256K tokens, 70B heads: own and all earlier keys, weights stored as w - 1
        _case("gather_256k", "gather", "long", 262144, 5, 32, 31, 64, 8, 128, offset=1.0),
        # the headline shape's gradients on their way to the projection
        _case("grads_llama8b", "grads", "mixed", 65536, 2, 8, 3, 32, 8, 128, base=500000.0),
        # centred norms with weights per head, half of a small head rotated, fp32 for a later sum; odd context
        _case("grads_d64_f32", "grads", "mixed", 49999, 6, 4, 2, 16, 8, 64, rot=32, inter=True, centred=True,
              per_head=True, eps=1e-5, w_bf16=False, bf16=False),
        # serving: one new token of each of a batch's long sequences, window and sinks out of the cache
        _case("window_token", "forward", "even", 262144, 16, 2, 1, 32, 8, 128, window=4096, sinks=4, tail=1),
        # evaluation of the headline shape in windows
        _case("window_forward_llama8b", "forward", "mixed", 65536, 2, 8, 3, 32, 8, 128, window=1024, sinks=4,
              q_std=3.0),
        # one document of most of 128K tokens in long windows, its late rank
        _case("window_forward_long", "forward", "long", 131072, 4, 16, 15, 32, 8, 128, window=4096, sinks=64,
              q_std=3.0),
        # one training layer: 2K tokens in short windows, and the headline shape
        _case("window_layer_tiny", "layer", "tiny", 2048, 1, 2, 0, 4, 4, 64, window=256, sinks=4),
        _case("window_layer_llama8b", "layer", "mixed", 65536, 2, 8, 3, 32, 8, 128, window=1024, sinks=4,
              base=500000.0),
        # capped scores in windows without sinks, small heads in pairs, odd context
        _case("window_cap_layer_d64", "layer", "mixed", 32771, 8, 4, 1, 16, 8, 64, window=512, rot=32, inter=True,
              offset=1.0, cap=50.0),
        # the largest: a long document's early and late chunk, long windows
        _case("window_layer_long", "layer", "long", 131072, 4, 8, 1, 32, 8, 128, window=4096, sinks=64),
    ]


HEADS = [(32, 8, 128), (32, 8, 128), (64, 8, 128), (8, 1, 128), (4, 1, 128), (16, 16, 128), (16, 8, 64),
         (16, 2, 64), (4, 4, 64)]
MOST_FLOPS, MOST_BYTES = 3.0e12, 1.1e9  # just under the largest listed cases


def draw(rng):
    while True:
        kind = rng.choice(["rows", "gather", "grads", "forward", "layer", "layer"])
        scores = kind in ("forward", "layer")
        context = int(round(math.exp(rng.uniform(math.log(64), math.log(131072 if scores else 262144)))))
        cp = rng.choice([1, 2, 4, 8, 16, 32])
        hq, hkv, d = rng.choice(HEADS)
        window = 0
        if scores or rng.random() < 0.4:
            window = int(round(math.exp(rng.uniform(math.log(2), math.log(min(context, 16384))))))
        sinks = rng.choice([0, 1, 4, 4, 16, 64, 200]) if window else 0
        tail = rng.choice([1, 1, 5, 33]) if kind == "forward" and rng.random() < 0.3 else 0
        if tail:
            cp = 2
        c = _case(None, kind, rng.choice(["mixed", "mixed", "long", "short", "even"]), context, rng.randrange(1, 64),
                  cp, 1 if tail else rng.randrange(cp), hq, hkv, d, window=window, sinks=sinks, tail=tail,
                  rot=rng.choice([d, d, d // 2, d // 4, 0]), inter=rng.random() < 0.4,
                  base=rng.choice([10000.0, 500000.0]), centred=rng.random() < 0.3, per_head=rng.random() < 0.3,
                  offset=rng.choice([0.0, 1.0]), eps=rng.choice([1e-6, 1e-5]), w_bf16=scores or rng.random() < 0.5,
                  cap=rng.choice([0.0, 0.0, 30.0, 50.0]) if scores else 0.0,
                  q_std=rng.choice([1.0, 3.0]) if kind == "forward" else 1.0, bf16=scores or rng.random() < 0.6)
        if not len(_geometry(c)["q"]):
            continue
        w = work(c)
        # (a layer whose queries see little but themselves has gradients of 0)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES and (
                kind != "layer" or _pairs(c) > 1.5 * len(_geometry(c)["q"])):
            return c


# ------------------------------------------------------------ documents and shards

def _lengths(c):
    rng, C = np.random.default_rng(c["len_seed"]), c["context"]
    if c["recipe"] == "tiny":
        cuts = np.sort(rng.choice(np.arange(1, C), size=2, replace=False))
        return np.diff(np.concatenate([[0], cuts, [C]]))
    if c["recipe"] == "even":  # len_seed documents, as long as each other but for one token
        return np.diff(np.arange(min(c["len_seed"], C) + 1) * C // min(c["len_seed"], C))
    first = [3 * C // 4] if c["recipe"] == "long" else []
    if c["recipe"] == "short":
        n = rng.integers(1, 512, size=C)
    else:
        n = np.clip(np.round(rng.lognormal(math.log(2048), 1.0, size=C // 64 + 1)), 64, C)
    n = np.concatenate([first, n]).astype(np.int64)
    lens = np.diff(np.concatenate([[0], np.minimum(np.cumsum(n), C)]))
    return lens[lens > 0]


def _geometry(c):
    """cu: document bounds; plan: rows (document, rank, offset, length); q, r: packed
    positions of the rank's own and received tokens; their documents, and their
    positions in these."""
    lens, cp = _lengths(c), c["cp"]
    cu = np.concatenate([[0], np.cumsum(lens)])
    if c["tail"]:
        cut = np.stack([np.zeros_like(lens), np.maximum(lens - c["tail"], 0), lens], axis=1)
        owner_of = np.array([0, 1])
    else:
        cut = lens[:, None] * np.arange(2 * cp + 1) // (2 * cp)
        owner_of = np.minimum(np.arange(2 * cp), 2 * cp - 1 - np.arange(2 * cp))
    size = np.diff(cut, axis=1)
    doc, chunk = np.nonzero(size)
    owner = owner_of[chunk]
    plan = np.stack([doc, owner, cut[doc, chunk], size[doc, chunk]], axis=1)
    token_doc = np.repeat(np.arange(len(lens)), lens)
    mine = np.repeat(owner, size[doc, chunk]) == c["rank"]
    pos = np.arange(len(mine))
    far = np.iinfo(np.int64).max // 2
    after = np.minimum.accumulate(np.where(mine, pos, far)[::-1])[::-1]  # the next own token
    got = ~mine & (after < cu[token_doc + 1])
    if c["window"]:
        got &= (after - pos < c["window"]) | (pos - cu[token_doc] < c["sinks"])
    return dict(cu=cu, plan=plan.astype(np.int32), q=pos[mine], r=pos[got], q_doc=token_doc[mine],
                r_doc=token_doc[got], q_pos=pos[mine] - cu[token_doc[mine]], r_pos=pos[got] - cu[token_doc[got]])


def _pairs(c):
    p = _geometry(c)["q_pos"]
    if not c["window"]:
        return int((p + 1).sum())
    w, s = c["window"], c["sinks"]
    return int((np.minimum(p + 1, w) + np.clip(np.minimum(s, p + 1 - w), 0, None)).sum())


def _frequencies(c):
    return c["base"] ** (-np.arange(0, c["rot"], 2) / max(c["rot"], 1))


# ------------------------------------------------------------------------- inputs

def _inputs(c, seed, g, dev):
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    e = lambda n, h, dt=BF: torch.randn(n, h, c["d"], device=dev, dtype=dt, generator=gen)  # noqa: E731
    tq, tr, hq, hkv, kind = len(g["q"]), len(g["r"]), c["hq"], c["hkv"], c["kind"]
    if kind == "forward":
        q = e(tq, hq)
        if c["q_std"] != 1.0:
            q *= c["q_std"]
        return dict(q=q, k_loc=e(tq, hkv), v_loc=e(tq, hkv), k_recv=e(tr, hkv), v_recv=e(tr, hkv))
    # weights about 1, as those of trained models are
    w = lambda h: ((1.0 - c["offset"]) + 0.3 * torch.randn(*((h,) if c["per_head"] else ()), c["d"], device=dev,  # noqa: E731
                                                          generator=gen)).to(BF if c["w_bf16"] else F32)
    x = dict(wq=w(hq), wk=w(hkv))
    if kind in ("rows", "grads", "layer"):
        x["qkv"] = e(tq, hq + 2 * hkv)
    if kind in ("gather", "grads", "layer"):
        x["k"] = e(int(g["cu"][-1]), hkv)
    if kind in ("gather", "layer"):
        x["v"] = e(int(g["cu"][-1]), hkv)
    if kind == "grads":
        x.update(dq=e(tq, hq, F32), dk_loc=e(tq, hkv, F32), dv_loc=e(tq, hkv, F32), dk_recv=e(tr, hkv, F32),
                 dv_recv=e(tr, hkv, F32))
    if kind == "layer":
        x["dout"] = e(tq, hq)
    return x


def prepare(case, seed):
    c, dev = case, torch.device("cuda:0")
    g = _geometry(c)
    t = lambda n: torch.from_numpy(g[n].astype(np.int64)).to(dev)  # noqa: E731
    s = dict(c=c, g=g, x=_inputs(c, seed, g, dev), q_tok=t("q"), r_tok=t("r"), q_pos=t("q_pos"), r_pos=t("r_pos"),
             w=torch.from_numpy(_frequencies(c)).to(dev))
    if own:
        s.update(_handles(c, g, s["x"], dev))
    return s


def _handles(c, g, x, dev):
    """What a program keeps: the bound view, the norms, the rotation, output buffers, workspaces."""
    from paper_2606_08476_amd import flashcp as F
    kind, scores = c["kind"], c["kind"] in ("forward", "layer")
    view = F.View(g["cu"], g["plan"], c["cp"], c["rank"], c["hq"], c["hkv"], c["d"], cap=c["cap"],
                  window=c["window"], sinks=c["sinks"]).bind(dev)
    tq, tr, hq, hkv, d = len(g["q"]), len(g["r"]), c["hq"], c["hkv"], c["d"]
    e = lambda *n, dt=BF: torch.empty(*n, dtype=dt, device=dev)  # noqa: E731
    h = dict(F=F, view=view)
    if kind != "forward":
        norm = lambda w: F.HeadNorm(w, eps=c["eps"], offset=c["offset"], centred=c["centred"])  # noqa: E731
        h.update(qn=norm(x["wq"]), kn=norm(x["wk"]), rope=None)
        if c["rot"]:
            h["rope"] = F.Rope(c["rot"], base=c["base"], interleaved=c["inter"])
    if kind in ("rows", "layer"):
        h.update(q=e(tq, hq, d))
    if kind in ("rows", "gather", "layer"):
        h.update(k_loc=e(tq, hkv, d), v_loc=e(tq, hkv, d))
    if kind in ("gather", "layer"):
        h.update(k_recv=e(tr, hkv, d), v_recv=e(tr, hkv, d))
    if kind in ("grads", "layer"):
        dt = BF if c["bf16"] else F32
        h.update(dqkv=e(tq, hq + 2 * hkv, d, dt=dt), dk_recv=e(tr, hkv, d, dt=dt), dv_recv=e(tr, hkv, d, dt=dt),
                 dwq=torch.empty_like(x["wq"]), dwk=torch.empty_like(x["wk"]),
                 nws=e(max(F.fc_norm_rope_workspace(view, h["qn"], h["kn"]), 1), dt=torch.uint8))
    if scores:
        fwd_b = view.workspace_size(F.FC_FUSED if kind == "forward" else F.FC_TWO_PASS)[0]
        h.update(o=e(tq, hq, d), lse=e(hq, tq, dt=F32), fws=e(max(fwd_b, 1), dt=torch.uint8))
    if kind == "layer":
        h.update(o32=e(tq, hq, d, dt=F32), delta=e(hq, tq, dt=F32),
                 bws=e(max(view.workspace_size()[2], 1), dt=torch.uint8),
                 g32=[e(tq, hq, d, dt=F32)] + [e(n, hkv, d, dt=F32) for n in (tq, tq, tr, tr)])
    return h


# ------------------------------------------------------------------ the operators

GRADS = ("dq", "dk_loc", "dv_loc", "dk_recv", "dv_recv")


def run(state):
    return _own(state) if own else _plain(state)


def _split(c, t):
    return t[:, :c["hq"]], t[:, c["hq"]:c["hq"] + c["hkv"]], t[:, c["hq"] + c["hkv"]:]


def _own(s):
    c, x, F, view, kind = s["c"], s["x"], s["F"], s["view"], s["c"]["kind"]
    if kind == "forward":
        F.fc_attn_fwd(view, x["q"], x["k_loc"], x["v_loc"], x["k_recv"], x["v_recv"], 0.0, F.FC_FUSED, s["o"], None,
                      s["lse"], s["fws"])
        return dict(o=s["o"], lse=s["lse"])
    rope, qn, kn = s["rope"], s["qn"], s["kn"]
    if kind == "rows":
        F.fc_norm_rope_fwd(view, rope, qn, kn, *_split(c, x["qkv"]), s["q"], s["k_loc"], s["v_loc"])
        return dict(q=s["q"], k_loc=s["k_loc"], v_loc=s["v_loc"])
    if kind == "layer":
        F.fc_norm_rope_fwd(view, rope, qn, None, x["qkv"][:, :c["hq"]], None, None, s["q"], None, None)
    if kind in ("gather", "layer"):
        out = dict(k_loc=s["k_loc"], v_loc=s["v_loc"], k_recv=s["k_recv"], v_recv=s["v_recv"])
        F.fc_kv_gather_norm_rope(view, rope, kn, x["k"], x["v"], *out.values())
        if kind == "gather":
            return out
    dx = (*_split(c, s["dqkv"]), s["dk_recv"], s["dv_recv"])
    out = dict(zip(GRADS, dx), dwq=s["dwq"], dwk=s["dwk"])
    q_in, k_in, _ = _split(c, x["qkv"])
    if kind == "grads":
        F.fc_norm_rope_bwd(view, rope, qn, kn, *(x[n] for n in GRADS), *dx, q_in, k_in, x["k"], s["dwq"], s["dwk"],
                           s["nws"])
        return out
    rows = (s["q"], s["k_loc"], s["v_loc"], s["k_recv"], s["v_recv"])
    F.fc_attn_fwd(view, *rows, 0.0, F.FC_TWO_PASS, s["o"], s["o32"], s["lse"], s["fws"])
    F.fc_bwd_preprocess(view, s["o"], x["dout"], s["delta"], o_f32=s["o32"])
    F.fc_attn_bwd_pass(view, *rows, s["lse"], s["delta"], x["dout"], 0.0, *s["g32"], s["bws"])
    # (own keys' rows are the packed tensor's)
    F.fc_norm_rope_bwd(view, rope, qn, kn, *s["g32"], *dx, q_in, None, x["k"], s["dwq"], s["dwk"], s["nws"])
    return dict(o=s["o"], lse=s["lse"], **out)


def _rotate(c, s, x, pos, back=False):
    """x [T, H, d] in 32 bits, its first `rot` values rotated by pos * w (angles in 64 bits)."""
    m = c["rot"]
    if not m:
        return x
    t = pos[:, None].to(F64) * s["w"]
    cos, sin = t.cos().to(F32)[:, None], t.sin().to(F32)[:, None]
    if back:
        sin = -sin
    y = x.clone()
    i, j = (slice(0, m, 2), slice(1, m, 2)) if c["inter"] else (slice(0, m // 2), slice(m // 2, m))
    y[..., i] = x[..., i] * cos - x[..., j] * sin
    y[..., j] = x[..., j] * cos + x[..., i] * sin
    return y


def _normal(c, x):
    """Rows normalised per head, and 1 over what they were divided by."""
    x = x.float()
    if c["centred"]:
        x = x - x.mean(-1, keepdim=True)
    r = (x.square().mean(-1, keepdim=True) + c["eps"]).rsqrt()
    return x * r, r


def _norm_rope(c, s, x, w, pos):
    return _rotate(c, s, _normal(c, x)[0] * (w.float() + c["offset"]), pos).to(BF)


def _norm_rope_back(c, s, dy, x, w, pos):
    """The gradient of x, and the weights' from these rows."""
    n, r = _normal(c, x)
    g = _rotate(c, s, dy, pos, True)
    dw = (g * n).sum(0, dtype=F64)
    a = g * (w.float() + c["offset"])
    dx = a - n * (a * n).mean(-1, keepdim=True)
    if c["centred"]:
        dx = dx - a.mean(-1, keepdim=True)
    return dx * r, dw if c["per_head"] else dw.sum(0)


def _plain(s):
    c, x, kind = s["c"], s["x"], s["c"]["kind"]
    if kind == "forward":
        return _attend(s, x["q"], x["k_loc"], x["v_loc"], x["k_recv"], x["v_recv"])[0]
    out, q_pos, r_pos = {}, s["q_pos"], s["r_pos"]
    if kind == "rows":
        q, k, v = _split(c, x["qkv"])
        return dict(q=_norm_rope(c, s, q, x["wq"], q_pos), k_loc=_norm_rope(c, s, k, x["wk"], q_pos), v_loc=v.clone())
    if kind in ("gather", "layer"):
        for name, tok, pos in (("loc", s["q_tok"], q_pos), ("recv", s["r_tok"], r_pos)):
            out["k_" + name] = _norm_rope(c, s, x["k"][tok], x["wk"], pos)
            out["v_" + name] = x["v"][tok]
        if kind == "gather":
            return out
    grads, k_in = x, _split(c, x["qkv"])[1]
    if kind == "layer":
        q = _norm_rope(c, s, x["qkv"][:, :c["hq"]], x["wq"], q_pos)
        out, grads = _attend(s, q, out["k_loc"], out["v_loc"], out["k_recv"], out["v_recv"])
        k_in = x["k"][s["q_tok"]]
    dq, dwq = _norm_rope_back(c, s, grads["dq"], x["qkv"][:, :c["hq"]], x["wq"], q_pos)
    dk, dwk = _norm_rope_back(c, s, grads["dk_loc"], k_in, x["wk"], q_pos)
    dr, dwr = _norm_rope_back(c, s, grads["dk_recv"], x["k"][s["r_tok"]], x["wk"], r_pos)
    dt = BF if c["bf16"] else F32
    out.update(dq=dq.to(dt), dk_loc=dk.to(dt), dv_loc=grads["dv_loc"].to(dt, copy=True), dk_recv=dr.to(dt),
               dv_recv=grads["dv_recv"].to(dt, copy=True), dwq=dwq.to(x["wq"].dtype), dwk=(dwk + dwr).to(x["wk"].dtype))
    return out


def _attend(s, q_in, k_loc, v_loc, k_recv, v_recv):
    """Attention of the rank's queries over own and received keys, some rows of a
    document at a time over the keys that any of them sees, and (layer) its gradients, in
    32 bits."""
    c, g, x = s["c"], s["g"], s["x"]
    hq, hkv, d, cap, window = c["hq"], c["hkv"], c["d"], c["cap"], c["window"]
    G, scale, dev = hq // hkv, 1.0 / math.sqrt(d), q_in.device
    grads = c["kind"] == "layer"
    tq, tr = len(g["q"]), len(g["r"])
    o = torch.empty(tq, hq, d, dtype=F32, device=dev)
    lse = torch.empty(hq, tq, dtype=F32, device=dev)
    z = lambda n, h: torch.zeros(n, h, d, dtype=F32, device=dev)  # noqa: E731
    dq, dk, dv = (z(tq, hq), z(tq + tr, hkv), z(tq + tr, hkv)) if grads else (None, None, None)
    K, V = torch.cat([k_loc, k_recv]), torch.cat([v_loc, v_recv])
    # keys in the order of their positions; those of a document side by side
    at = np.concatenate([g["q"], g["r"]])
    order = np.argsort(at, kind="stable")
    k_at, order_d = at[order], torch.from_numpy(order).to(dev)
    k_pos = torch.cat([s["q_pos"], s["r_pos"]])[order_d]
    docs, first = np.unique(g["q_doc"], return_index=True)
    last = np.append(first[1:], tq)
    for doc, q0, q1 in zip(docs.tolist(), first.tolist(), last.tolist()):
        start = int(g["cu"][doc])
        lo_doc, sink = np.searchsorted(k_at, [start, start + c["sinks"]]).tolist()
        step = max(1, (1 << 28) // (hq * int(np.searchsorted(k_at, int(g["cu"][doc + 1])) - lo_doc)))
        if window:
            step = min(max(step, 64), max(window // 2, 64))
        for a in range(q0, q1, step):
            b = min(a + step, q1)
            m, p0, p1 = b - a, int(g["q"][a]), int(g["q"][b - 1])
            lo, hi = np.searchsorted(k_at, [max(start, p0 - window + 1) if window else start, p1 + 1]).tolist()
            near = order_d[lo:hi]
            pos = k_pos[lo:hi]
            if window and min(sink, lo) > lo_doc:
                near = torch.cat([order_d[lo_doc:min(sink, lo)], near])
                pos = torch.cat([k_pos[lo_doc:min(sink, lo)], pos])
            n, away = near.numel(), s["q_pos"][a:b, None] - pos
            hidden = away < 0
            if window:
                hidden |= (away >= window) & (pos >= c["sinks"])
            heads = lambda t: t.float().view(m, hkv, G, d).permute(1, 2, 0, 3).reshape(hkv, G * m, d)  # noqa: E731
            k, v = K[near].float().transpose(0, 1).contiguous(), V[near].float().transpose(0, 1).contiguous()
            kt = k.transpose(1, 2).contiguous()
            q = heads(q_in[a:b])
            sc = (q @ kt).mul_(scale)
            if cap:
                th = sc.div_(cap).tanh_()
                sc = th * cap
            sc = sc.view(hkv, G, m, n).masked_fill_(hidden, -math.inf)
            top = sc.amax(-1, keepdim=True)
            p = sc.sub_(top).exp_()
            tot = p.sum(-1, keepdim=True)
            p = p.div_(tot).view(hkv, G * m, n)
            lse[:, a:b] = (top + tot.log()).view(hq, m)
            out = p @ v
            back = lambda t: t.view(hkv, G, m, d).permute(2, 0, 1, 3).reshape(m, hq, d)  # noqa: E731
            o[a:b] = back(out)
            if not grads:
                continue
            do = heads(x["dout"][a:b])
            dv[near] += (p.transpose(1, 2).contiguous() @ do).transpose(0, 1)
            ds = (do @ v.transpose(1, 2).contiguous()).sub_((do * out).sum(-1, keepdim=True)).mul_(p)
            if cap:
                ds = ds.mul_(1 - th * th)
            dq[a:b] = back((ds @ k).mul_(scale))
            dk[near] += (ds.transpose(1, 2).contiguous() @ q).mul_(scale).transpose(0, 1)
    out = dict(o=o.to(BF), lse=lse)
    if not grads:
        return out, None
    return out, dict(dq=dq, dk_loc=dk[:tq], dv_loc=dv[:tq], dk_recv=dk[tq:], dv_recv=dv[tq:])


# ------------------------------------------------------------------ work and definition

def work(case):
    c = case
    g = _geometry(c)
    tq, tk, d = len(g["q"]), len(g["q"]) + len(g["r"]), c["d"]
    rows, own_kv, kv = tq * c["hq"] * d, tq * c["hkv"] * d, tk * c["hkv"] * d
    kind, size = c["kind"], 2 if c["bf16"] else 4
    if kind == "rows":
        return {"bytes": 4 * (rows + 2 * own_kv), "flops": 9.0 * (rows + own_kv)}
    if kind == "gather":
        return {"bytes": 8 * kv, "flops": 9.0 * kv}
    back = {"bytes": 6 * (rows + kv) + 4 * kv + size * (rows + 2 * kv), "flops": 18.0 * (rows + kv)}
    if kind == "grads":
        return back
    pairs = float(_pairs(c)) * c["hq"] * d
    fwd = 2 * (2 * rows + 2 * kv) + 4 * c["hq"] * tq  # q, k, v, o; lse
    if kind == "forward":
        return {"bytes": fwd, "flops": 4 * pairs}
    # and dO; the gradients written
    return {"bytes": fwd + 2 * rows + 2 * (rows + 2 * kv), "flops": 14 * pairs + 27.0 * (rows + kv)}


def exact(case, seed):
    """What run() returns, from the definitions, in 64 bits; gradients of the norms by
    differentiating these. (Rows that an operator of a layer hands to the next are
    bf16.)"""
    c, dev = case, torch.device("cuda:0")
    g = _geometry(c)
    x = {n: t.to(F64) for n, t in _inputs(c, seed, g, dev).items()}
    hq, hkv, d, kind = c["hq"], c["hkv"], c["d"], c["kind"]
    where = {"loc": torch.from_numpy(g["q_pos"]).to(dev), "recv": torch.from_numpy(g["r_pos"]).to(dev)}
    if kind == "forward":
        return _exact_attention(c, g, x, where)[0]
    w = torch.from_numpy(_frequencies(c)).to(dev)

    def turned(t, pos):
        if not c["rot"]:
            return t
        m = c["rot"]
        z = torch.polar(torch.ones((), dtype=F64, device=dev), pos.to(F64)[:, None, None] * w)
        part = t[..., :m].unflatten(-1, (m // 2, 2) if c["inter"] else (2, m // 2))
        if not c["inter"]:
            part = part.transpose(-1, -2)
        y = torch.view_as_real(torch.complex(part[..., 0], part[..., 1]) * z)
        if not c["inter"]:
            y = y.transpose(-1, -2)
        return torch.cat([y.flatten(-2), t[..., m:]], -1)

    def normed(t, weight, pos):
        mean = t.sum(-1, keepdim=True) / d if c["centred"] else 0.0
        spread = ((t - mean) ** 2).sum(-1, keepdim=True) / d + c["eps"]
        return turned((t - mean) / torch.sqrt(spread) * (weight + c["offset"]), pos)

    tok = {"loc": torch.from_numpy(g["q"]).to(dev), "recv": torch.from_numpy(g["r"]).to(dev)}
    if kind == "rows":
        q, k, v = x["qkv"].split([hq, hkv, hkv], 1)
        return dict(q=normed(q, x["wq"], where["loc"]), k_loc=normed(k, x["wk"], where["loc"]), v_loc=v)
    if kind == "gather":
        out = {}
        for n in ("loc", "recv"):
            out["k_" + n], out["v_" + n] = normed(x["k"][tok[n]], x["wk"], where[n]), x["v"][tok[n]]
        return out
    out, grads = {}, x
    q_in, k_in = x["qkv"][:, :hq], x["qkv"][:, hq:hq + hkv] if kind == "grads" else x["k"][tok["loc"]]
    if kind == "layer":
        bf = lambda t: t.to(BF).to(F64)  # noqa: E731
        rows = dict(q=bf(normed(q_in, x["wq"], where["loc"])), dout=x["dout"])
        for n in ("loc", "recv"):
            rows["k_" + n], rows["v_" + n] = bf(normed(x["k"][tok[n]], x["wk"], where[n])), x["v"][tok[n]]
        out, grads = _exact_attention(c, g, rows, where)
    leaf = lambda t: t.detach().clone().requires_grad_()  # noqa: E731
    q, k, r, wq, wk = leaf(q_in), leaf(k_in), leaf(x["k"][tok["recv"]]), leaf(x["wq"]), leaf(x["wk"])
    torch.autograd.backward([normed(q, wq, where["loc"]), normed(k, wk, where["loc"]), normed(r, wk, where["recv"])],
                            [grads["dq"], grads["dk_loc"], grads["dk_recv"]])
    out.update(dq=q.grad, dk_loc=k.grad, dv_loc=grads["dv_loc"], dk_recv=r.grad, dv_recv=grads["dv_recv"],
               dwq=wq.grad, dwk=wk.grad)
    return out


def _exact_attention(c, g, x, where):
    hq, hkv, d, dev = c["hq"], c["hkv"], c["d"], x["q"].device
    qd = torch.from_numpy(g["q_doc"]).to(dev)
    kd = torch.cat([qd, torch.from_numpy(g["r_doc"]).to(dev)])
    kp = torch.cat([where["loc"], where["recv"]])
    k, v = torch.cat([x["k_loc"], x["k_recv"]]), torch.cat([x["v_loc"], x["v_recv"]])
    tq, G = qd.numel(), hq // hkv
    o, lse = torch.zeros_like(x["q"]), torch.zeros(hq, tq, dtype=F64, device=dev)
    dq, dk, dv = torch.zeros_like(x["q"]), torch.zeros_like(k), torch.zeros_like(v)
    for n in torch.unique(qd).tolist():
        rows_all, keys_all = torch.nonzero(qd == n).flatten(), torch.nonzero(kd == n).flatten()
        per = max(1, (1 << 26) // keys_all.numel())
        if c["window"]:
            per = min(per, max(c["window"], 512))
        for r in rows_all.split(per):
            pq = where["loc"][r]
            # keys that some of these rows may see
            pk = kp[keys_all]
            some = pk <= pq.max()
            if c["window"]:
                some &= (pk > pq.min() - c["window"]) | (pk < c["sinks"])
            keys = keys_all[some]
            dist = pq[:, None] - kp[keys][None]
            seen = dist >= 0
            if c["window"]:
                seen = seen & ((dist < c["window"]) | (kp[keys] < c["sinks"])[None])
            for h in range(hq):
                K, V, Q = k[keys, h // G], v[keys, h // G], x["q"][r, h]
                S = Q @ K.T / math.sqrt(d)
                slope = None
                if c["cap"]:
                    slope = 1 / torch.cosh(S / c["cap"]) ** 2
                    S = c["cap"] * torch.tanh(S / c["cap"])
                S = torch.where(seen, S, -math.inf)
                L = torch.logsumexp(S, 1)
                P = torch.exp(S - L[:, None])
                O = P @ V
                o[r, h], lse[h, r] = O, L
                if c["kind"] == "forward":
                    continue
                dO = x["dout"][r, h]
                dX = P * (dO @ V.T - (dO * O).sum(1, keepdim=True)) / math.sqrt(d)
                if slope is not None:
                    dX = dX * slope
                dq[r, h] = dX @ K
                dk[keys, h // G] += dX.T @ Q
                dv[keys, h // G] += P.T @ dO
    out = dict(o=o, lse=lse)
    return out, dict(dq=dq, dk_loc=dk[:tq], dv_loc=dv[:tq], dk_recv=dk[tq:], dv_recv=dv[tq:])
