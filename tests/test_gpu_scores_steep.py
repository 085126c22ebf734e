"""Scored views whose slope times position leaves fp32's range of exponents: steep
slopes (up to the largest a view takes) far into a document (up to the longest a view
takes). A row's own share of its biases is then billions, of which the near keys'
shares leave next to nothing.

Keys more than a few tokens away have no weight left at such slopes (e^-745 is 0 in
64 bits), so the oracle, and its elementwise bounds (oracle/scores.py), are those of
the last keys alone; gradients of all others are exactly 0."""
import numpy as np
import pytest
import torch

from oracle import scores as S
from paper_2606_08476_amd import flashcp as F
from test_gpu_parity import dev, say  # noqa: F401

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
OWN, NEAR = 130, 1024  # own rows at the document's end; received keys the oracle sees


class Far:
    """A rank that holds the last OWN tokens of a document of n, the rest received."""

    def __init__(self, dev, n, hq, hkv, d, slopes, cap, q_std, tiles):
        cu = np.array([0, n], dtype=np.int32)
        plan = np.array([[0, 1, 0, n - OWN], [0, 0, n - OWN, OWN]], dtype=np.int32)
        self.view = F.View(cu, plan, 2, 0, hq, hkv, d, tiles=tiles, cap=cap, slopes=slopes).bind(dev)
        assert (self.view.info["t_q"], self.view.info["t_recv"]) == (OWN, n - OWN)
        self.n, self.hq, self.hkv, self.d, self.dev, self.slopes = n, hq, hkv, d, dev, slopes
        g = torch.Generator(device=dev).manual_seed(n + hq + d)
        e = lambda m, h: torch.randn(m, h, d, generator=g, device=dev, dtype=BF)  # noqa: E731
        self.q, self.do = q_std * e(OWN, hq), e(OWN, hq)
        self.kv = e(OWN, hkv), e(OWN, hkv), e(n - OWN, hkv), e(n - OWN, hkv)
        doc = lambda m: torch.zeros(m, dtype=torch.int64, device=dev)  # noqa: E731
        at = torch.arange(n - OWN - NEAR, n, device=dev)
        k, v = (torch.cat([self.kv[2 + i][-NEAR:], self.kv[i]]) for i in (0, 1))
        self.want, self.bound = S.attention(doc(OWN), at[NEAR:], self.q, doc(OWN + NEAR), at, k, v, cap,
                                            slopes, self.do)
        # (every weight that the oracle leaves out is 0 in 64 bits: a score is at most the
        # product of two norms, here under twice 12 * 12 or the square root of d)
        assert float(np.min(slopes)) * (NEAR - 1) > 800 + 2 * q_std * 4 * d / np.sqrt(d)

    def new(self, *s, dt=F32):
        return torch.full(s, float("nan"), dtype=dt, device=self.dev)

    def rounding(self):
        """What the forward's LSE may be off by beside the oracle's bound. A row's share of
        its biases is counted from the document's start, and off by half a step of it, at
        most 2^-24 slope n; scores are that much off, all alike, and as large, so that
        their own rounding, the maximum's and the sum's logarithm's, and the correction's
        are each 2^-24 of it: four at the most."""
        s = torch.from_numpy(self.slopes).to(self.dev).double()
        return (s * self.n * 2.0 ** -46)[:, None]

    def grads(self):
        m = self.n - OWN
        return [self.new(OWN, self.hq, self.d)] + [self.new(t, self.hkv, self.d) for t in (OWN, OWN, m, m)]

    def ws(self, n):
        return torch.empty(max(n, 1), dtype=torch.uint8, device=self.dev)

    def near(self, name, got, key, old=None):
        """got within the oracle's bound; old: gradients of keys before NEAR, all 0."""
        over = float(((got.double() - self.want[key]).abs() - self.bound[key]).max())
        say(f"[gpu]   {name}: over its bound {over:.1e}")
        assert bool(torch.isfinite(got).all()) and over <= 0, f"{name}: {over:.3e} over its bound"
        if old is not None:
            assert not bool(old.any()), f"{name}: keys without weight"


STEEP = [
    # tokens, heads, head dim, slopes, cap, what queries are scaled by, query tile
    (1500003, 4, 1, 64, [1024.0, 700.0, 128.0, 1024.0], 0.0, 2.0, None),
    (1500003, 2, 1, 128, [1024.0, 128.0], 30.0, 2.0, None),
    (4000037, 8, 2, 128, [1024.0, 128.0, 1000.0, 333.0, 1024.0, 1024.0, 512.0, 256.0], 0.0, 2.0, None),
    (4000037, 4, 1, 64, [1024.0, 512.0, 128.0, 64.0], 30.0, 2.0, (128, 0, 0, 0)),
    # scores that differ by as much as the biases of neighbours: several keys matter
    (4000037, 2, 2, 128, [1024.0, 700.0], 0.0, 800.0, None),
    (4000037, 4, 1, 64, [128.0, 130.0, 150.0, 200.0], 600.0, 150.0, None),
    (1 << 24, 2, 1, 64, [1024.0, 128.0], 0.0, 2.0, None),
    (1 << 24, 2, 1, 64, [128.0, 150.0], 0.0, 150.0, None),
]

# the LSE's own accuracy: products so small that theirs is no part of the bound
SMALL = [(1500003, 2, 1, 64, [1024.0, 512.0], 0.0, 0.01, None), (1 << 24, 2, 1, 64, [1024.0, 64.0], 0.0, 0.01, None),
         (1 << 24, 2, 2, 128, [1024.0, 700.0], 1.0, 0.01, None)]


@pytest.mark.parametrize("n,hq,hkv,d,slopes,cap,q_std,tiles", STEEP)
def test_gradients(n, hq, hkv, d, slopes, cap, q_std, tiles, dev):  # noqa: F811
    """Every way to dQ, dK and dV, from the oracle's own output and LSE: deterministic
    (with and without room for row norms), dQ alone, and by atomics."""
    say(f"[gpu] steep gradients n={n} heads={hq}/{hkv} d={d} cap={cap}")
    f = Far(dev, n, hq, hkv, d, np.array(slopes, dtype=np.float32), cap, q_std, tiles)
    v, o32, lse = f.view, f.want["o"].float(), f.want["lse"].float()
    _, bws, pws = v.workspace_size()
    for det, short in ((True, 0), (True, 256), (False, 0)):
        gr = f.grads()
        F.fc_attn_bwd(v, f.q, *f.kv, None, lse, f.do, 0.0, *gr, f.ws(bws - short), deterministic=det, o_f32=o32)
        torch.cuda.synchronize()
        what = ("dq", "dk", "dv")
        how = f"{'deterministic' if det else 'atomic'}{', every key' if short else ''}"
        f.near(f"{what[0]} {how}", gr[0], "dq")
        for name, own, got in (("dk", gr[1], gr[3]), ("dv", gr[2], gr[4])):
            f.near(f"{name} {how}", torch.cat([got[-NEAR:], own]), name, got[:-NEAR])
    delta, dq = f.new(hq, OWN), f.new(OWN, hq, d)
    F.fc_bwd_preprocess(v, None, f.do, delta, o_f32=o32)
    F.fc_attn_bwd_dq(v, f.q, *f.kv, lse, delta, f.do, 0.0, dq)
    torch.cuda.synchronize()
    f.near("dq alone", dq, "dq")
    v.close()


@pytest.mark.parametrize("n,hq,hkv,d,slopes,cap,q_std,tiles", STEEP + SMALL)
def test_forward(n, hq, hkv, d, slopes, cap, q_std, tiles, dev):  # noqa: F811
    """Both modes, with and without room for row norms, and the partial passes merged."""
    say(f"[gpu] steep forward n={n} heads={hq}/{hkv} d={d} cap={cap}")
    f = Far(dev, n, hq, hkv, d, np.array(slopes, dtype=np.float32), cap, q_std, tiles)
    v = f.view
    for mode in (F.FC_TWO_PASS, F.FC_FUSED):
        for short in (0, 256):
            o, o32, lse = f.new(OWN, hq, d, dt=BF), f.new(OWN, hq, d), f.new(hq, OWN)
            F.fc_attn_fwd(v, f.q, *f.kv, 0.0, mode, o, o32, lse, f.ws(v.workspace_size(mode)[0] - short))
            torch.cuda.synchronize()
            for name, got in (("o", o), ("o32", o32), ("lse", lse)):
                bound = f.bound[name] + (f.rounding() if name == "lse" else 0.0)
                over = float(((got.double() - f.want["lse" if name == "lse" else "o"]).abs() - bound).max())
                say(f"[gpu]   {name} mode {mode}{', every key' if short else ''}: over its bound {over:.1e}")
                assert bool(torch.isfinite(got).all()) and over <= 0, f"{name}: {over:.3e} over its bound"
    part = [f.new(OWN, hq, d), f.new(hq, OWN), f.new(OWN, hq, d), f.new(hq, OWN)]
    F.fc_attn_fwd_partials(v, f.q, *f.kv, 0.0, *part)
    ob, om, lm = f.new(OWN, hq, d, dt=BF), f.new(OWN, hq, d), f.new(hq, OWN)
    F.fc_lse_merge(*part, ob, om, lm)
    torch.cuda.synchronize()
    assert float(((om.double() - f.want["o"]).abs() - f.bound["o32"]).max()) <= 0
    assert float(((lm.double() - f.want["lse"]).abs() - f.bound["lse"] - f.rounding()).max()) <= 0
    v.close()


def test_without_allocation(dev):  # noqa: F811
    """A view whose plain twin fits the static scratch fits it too, however little of its
    work is within reach, and gives the bits of a call with a workspace."""
    n, hq, hkv, d = 16384, 8, 8, 128
    cu = np.array([0, n], dtype=np.int32)
    v = F.View(cu, F.fc_plan_per_doc(cu, 1), 1, 0, hq, hkv, d, slopes=np.full(hq, 0.5)).bind(dev)
    g = torch.Generator(device=dev).manual_seed(3)
    q, do, k, w = (torch.randn(n, h, d, generator=g, device=dev, dtype=BF) for h in (hq, hq, hkv, hkv))
    none = torch.empty(0, hkv, d, dtype=BF, device=dev)
    z = lambda *s, dt=F32: torch.full(s, float("nan"), dtype=dt, device=dev)  # noqa: E731
    u8 = lambda m: torch.empty(max(m, 1), dtype=torch.uint8, device=dev)  # noqa: E731
    fws, bws, _ = v.workspace_size(F.FC_FUSED)
    assert bws <= F.NOALLOC_SCRATCH_BYTES
    o, o32, lse = z(n, hq, d, dt=BF), z(n, hq, d), z(hq, n)
    F.fc_attn_fwd(v, q, k, w, none, none, 0.0, F.FC_FUSED, o, o32, lse, u8(fws))
    a, b = ([z(n, hq, d), z(n, hkv, d), z(n, hkv, d), z(0, hkv, d), z(0, hkv, d)] for _ in range(2))
    F.fc_attn_bwd(v, q, k, w, none, none, o, lse, do, 0.0, *a, u8(bws), o_f32=o32)
    F.fc_attn_bwd_noalloc(v, q, k, w, none, none, o, lse, do, 0.0, *b, o_f32=o32)
    torch.cuda.synchronize()
    assert all(bool(torch.isfinite(t).all()) and torch.equal(t, u) for t, u in zip(a, b))
    v.close()
