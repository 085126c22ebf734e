"""Windowed views on the CPU, by brute force from the definition (a query at position p
of its document sees positions u <= p with p - u < window or u < sinks):

* the receive set is exactly what the rank's queries see and it does not hold, and the
  pair counts are the visible pairs;
* a query tile takes exactly the key tiles of which some row sees a key, whole or cut
  into the forward's chunks and the dQ parts;
* the key-major items, masked as the kernel masks, cover every visible pair once, and
  a wave that is left out, or not masked, rightly is;
* a window that reaches every key gives the view without one."""
import numpy as np
import pytest

from oracle import planner as P
from paper_2606_08476_amd import flashcp as F

BN = 64


def key_tiles(base, end, lo, sink):
    """First keys of the tiles taken of base .. end-1 (fc_view_export_window): those with
    a key from lo on or before sink."""
    return [a for a in range(base, end, BN) if a < sink or min(a + BN, end) > lo]


class Brute:
    def __init__(self, cu, plan, rank, window, sinks):
        cu, plan = np.asarray(cu), np.asarray(plan)
        doc = np.repeat(np.arange(len(cu) - 1), np.diff(cu))
        mine = np.zeros(cu[-1], dtype=bool)
        for d, r, o, n in plan.tolist():
            if r == rank:
                mine[cu[d] + o:cu[d] + o + n] = True
        g = np.arange(cu[-1])
        self.q = g[mine]
        pos = g - cu[doc]
        dist = self.q[:, None] - g[None]
        seen = (doc[self.q][:, None] == doc[None]) & (dist >= 0)
        if window:
            seen &= (dist < window) | (pos < sinks)[None]
        self.recv = g[~mine & seen.any(0)]
        self.local, self.received = seen[:, self.q], seen[:, self.recv]
        assert not seen[:, ~mine].sum() - self.received.sum()


def check_view(cu, plan, cp, rank, hq, hkv, d, window, sinks, tiles=None):
    b = Brute(cu, plan, rank, window, sinks)
    v = F.View(cu, plan, cp, rank, hq, hkv, d, tiles=tiles, window=window, sinks=sinks)
    assert v.window == (window, sinks)
    i, e, L, s, w = v.info, v.export(), v.export_launch(), v.export_split(), v.export_window()
    v.close()
    assert e["q_gpos"].tolist() == b.q.tolist() and e["recv_gpos"].tolist() == b.recv.tolist()
    assert (i["pairs_loc"], i["pairs_recv"]) == (b.local.sum(), b.received.sum())
    tq, tr = i["t_q"], i["t_recv"]
    if w is None:  # every row sees every earlier key of its document
        full = Brute(cu, plan, rank, 0, 0)
        assert np.array_equal(full.local, b.local) and full.recv.tolist() == b.recv.tolist()
        return False, 0
    win, end = w["win"], w["wave_end"]
    see = {0: b.local, 1: b.received}
    # rows' windows: with the causal limits and the sinks, the visible keys
    lim = e["lim"]
    for src, n in ((0, tq), (1, tr)):
        k = np.arange(n)[None]
        doc0 = np.repeat(e["q_cu_docseg"][:-1] if src == 0 else e["recv_cu"][:-1], np.diff(e["q_cu_docseg"]))
        top = (np.arange(tq) + 1 if src == 0 else lim)[:, None]
        want = (k >= doc0[:, None]) & (k < top) & ((k >= win[:, src][:, None]) | (k < win[:, 2 + src][:, None]))
        assert np.array_equal(want, see[src])

    def taken(it):
        q0, q1, r0, r1, l0, l1 = it[:6]
        return ([(1, a) for a in key_tiles(r0, r1, win[q0, 1], win[q0, 3])] +
                [(0, a) for a in key_tiles(l0, l1, win[q0, 0], win[q0, 2])])

    def visible(it):
        q0, q1, r0, r1, l0, l1 = it[:6]
        out = []
        for src, lo, hi in ((1, r0, r1), (0, l0, l1)):
            out += [(src, a) for a in range(lo, hi, BN) if see[src][q0:q1, a:min(a + BN, hi)].any()]
            rest = see[src][q0:q1].copy()
            rest[:, lo:hi] = False
            assert not rest.any() or lo == hi == 0   # (an item of the other source alone)
        return out

    for it in e["fwd_fused"].tolist():
        assert taken(it) == visible(it), it
    for name, src in (("fwd_local", 0), ("fwd_recv", 1)):
        for it in e[name].tolist():
            assert taken(it) == [t for t in visible(it) if t[0] == src], it
    for it in e["fwd_fused"].tolist() + e["fwd_local"].tolist():
        q0, q1, l0, l1, ldiag = it[0], it[1], it[4], it[5], it[6]
        assert all(b.local[q0, a:a + BN].all() or a < win[q1 - 1, 0] for _, a in taken(it)
                   if _ == 0 and a < ldiag and a >= win[q0, 2])
    cost = [len(taken(it)) for it in L["fwd_fused"].tolist()]
    assert cost == sorted(cost, reverse=True)
    # chunks and dQ parts: the same tiles, in the slots' order
    fused = {tuple(it[:2]): it for it in e["fwd_fused"].tolist()}
    c = s["fwd_chunk"]
    if c:
        slot = {x[7]: x for x in s["fwd_units"].tolist()}
        assert sorted(slot) == list(range(len(slot)))
        used = []
        for q0, q1, first, n_r, n_l, *_ in s["fwd_comb"].tolist():
            it = fused.pop((q0, q1))
            got = []
            for k in range(n_r + n_l):
                x = slot[first + k]
                used.append(first + k)
                t = taken(x)
                src = 1 if k < n_r else 0
                lo = it[2] if src else it[4]
                assert t and {a[0] for a in t} == {src} and len({(a[1] - lo) // (c * BN) for a in t}) == 1
                assert all((a[1] - lo) % BN == 0 for a in t)
                got += t
            assert got == taken(it)
        assert not fused and sorted(used) == list(range(len(slot)))
    fused = {tuple(it[:2]): it for it in e["fwd_fused"].tolist()}
    if len(s["dq_items"]):
        slot = {x[7]: x for x in s["dq_items"].tolist() if x[7] >= 0}
        done = {tuple(x[:2]): taken(x) for x in s["dq_items"].tolist() if x[7] < 0}
        for q0, q1, first, n, *_ in s["dq_comb"].tolist():
            done[(q0, q1)] = [t for k in range(n) for t in taken(slot.pop(first + k))]
        assert not slot and done == {k: taken(it) for k, it in fused.items()}
    # key-major items
    cover = {0: np.zeros((tq, tq), dtype=np.int8), 1: np.zeros((tq, tr), dtype=np.int8)}
    always = 2 ** 31 - 1
    for it, qf, we in zip(L["bwd_launch"].tolist(), L["bwd_qfirst"].tolist(), end.tolist()):
        k0, k1, q0, q1, qfull, src, seg, _ = it
        rows = np.arange(q0, q1)[:, None]
        for wv in range(4):
            kw = k0 + 32 * wv
            if kw >= k1:
                continue
            keys = np.arange(kw, min(kw + 32, k1))[None]
            cut, gone = we[wv]
            m = (rows >= keys) if src == 0 else (keys < lim[q0:q1][:, None])
            if cut != always:
                m = m & (keys >= win[q0:q1, src][:, None])
                assert not m[np.arange(q0, q1) >= gone].any()
                assert (win[q0:min(q1, max(q0, cut)), src] <= kw).all()
            else:
                assert gone == always
            assert not m[np.arange(q0, q1) < qf[wv]].any()
            if keys.shape[1] == 32:
                inside = (np.arange(q0, q1) >= qfull) & (np.arange(q0, q1) < cut)
                assert m[inside].all()
            cover[src][q0:q1, kw:min(kw + 32, k1)] += m
    for src in (0, 1):
        assert np.array_equal(cover[src], see[src].astype(np.int8)), src
    return bool(c), int(len(s["dq_comb"]))


def test_random_views():
    rng = np.random.default_rng(5)
    split = np.zeros(2, dtype=int)
    heads = [(4, 1, 128), (8, 1, 128), (16, 2, 64), (4, 4, 64), (32, 8, 128)]
    for k in range(140):
        n = int(rng.integers(1, 6))
        lens = np.exp(rng.uniform(0, np.log(2000 if k % 4 else 5000), size=n)).astype(int) + 1
        cp = int(rng.integers(1, 7))
        cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        plan = [P.plan_per_doc, P.plan_per_seq, P.plan_whole_lpt][int(rng.integers(3))](cu, cp)
        window = int(np.exp(rng.uniform(0, np.log(3000))))
        sinks = int(rng.choice([0, 0, 1, 4, 63, 64, 65, 200, 5000]))
        hq, hkv, d = heads[int(rng.integers(len(heads)))]
        for rank in {0, cp - 1, int(rng.integers(cp))}:
            got = check_view(cu, plan, cp, rank, hq, hkv, d, window, sinks)
            split += np.array(got) > 0
    assert (split > 3).all(), split


@pytest.mark.parametrize("window", [1, 2, 31, 64, 65, 128, 700])
@pytest.mark.parametrize("sinks", [0, 1, 128, 130])
def test_windows_and_tiles(window, sinks):
    cu = np.array([0, 1, 2, 700, 1100, 1164], dtype=np.int32)
    for cp, rank in ((1, 0), (3, 2)):
        for tiles in (None, (128, 0, 0, 0)):
            check_view(cu, P.plan_per_doc(cu, cp), cp, rank, 4, 1, 64, window, sinks, tiles)


def test_last_tokens():
    """A rank of a few tokens at each document's end: what a decoding step sees."""
    for lens, tail in (([3000, 5, 1, 900], 1), ([3000, 5, 900], 5), ([4000], 1)):
        cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        plan = [x for i, n in enumerate(lens) for x in ([i, 0, 0, max(n - tail, 0)], [i, 1, max(n - tail, 0), min(n, tail)])
                if x[3]]
        for window, sinks in ((1, 0), (1, 4), (256, 4), (1024, 0), (2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1)):
            check_view(cu, plan, 2, 1, 8, 1, 128, window, sinks)
            check_view(cu, plan, 2, 0, 8, 1, 128, window, sinks)


def test_a_window_that_reaches_everything_is_none():
    cu = np.array([0, 300, 1000], dtype=np.int32)
    plan = P.plan_per_doc(cu, 2)
    a = F.View(cu, plan, 2, 0, 4, 2, 64)   # (rank 0 has the documents' last tokens)
    for window in (700, 5000):
        b = F.View(cu, plan, 2, 0, 4, 2, 64, window=window, sinks=9)
        assert b.export_window() is None and b.info == a.info and b.window == (window, 9)
        for x, y in ((a.export(), b.export()), (a.export_launch(), b.export_launch())):
            assert all(np.array_equal(x[n], y[n]) for n in x)
    b = F.View(cu, plan, 2, 0, 4, 2, 64, window=699)
    assert b.export_window() is not None
    assert a.window == (0, 0) and a.export_window() is None


def test_refusals():
    cu, plan = np.array([0, 10], dtype=np.int32), [[0, 0, 0, 10]]
    for kw in (dict(window=-1), dict(sinks=3), dict(window=4, sinks=-1)):
        with pytest.raises(F.FlashCPError) as e:
            F.View(cu, plan, 1, 0, 4, 2, 64, **kw)
        assert e.value.code == -1
    assert F.lib().fc_view_get_window(None, None, None) == -1
    assert F.lib().fc_view_export_window(None, None, None, None) == -1
    v = F.View(cu, plan, 1, 0, 4, 2, 64, cap=30.0, slopes=np.ones(4), window=4, sinks=1)
    assert v.window == (4, 1) and v.score[0] == 30.0
    e = F.View([0, 10], plan, 2, 1, 4, 2, 64, window=4)   # no rows
    assert e.info["t_q"] == e.info["t_recv"] == 0 and e.export_window() is None


def test_windowed_views_under_sanitizers(tmp_path):
    """Every attention entry point on windowed views in a host build under AddressSanitizer
    and UndefinedBehaviorSanitizer, with stub launchers that walk the tables."""
    import os
    import shutil
    import subprocess
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    host = os.path.join(root, "paper_2606_08476_amd", "csrc", "host")
    exe = tmp_path / "window_driver"
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(root, "include"),
           *[os.path.join(host, f) for f in ("plan.cpp", "view.cpp", "api.cpp")],
           os.path.join(root, "tests", "sanitize", "window_driver.cpp"), "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert "all checks passed" in r.stdout
