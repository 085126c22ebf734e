"""Host side of scored views and rotary rows, no GPU: the tables and getters of a
view with a score function, frequencies against the oracle's, and every refusal
before anything is launched."""
import ctypes as C
import math
import os

import numpy as np
import pytest

from oracle import rope as R
from paper_2606_08476_amd import flashcp as F


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(F._LIB_PATH):
        from paper_2606_08476_amd import build
        build.build()


CU = np.array([0, 300, 301, 1000], dtype=np.int32)


def _view(**kw):
    return F.View(CU, F.fc_plan_per_doc(CU, 2), 2, 1, 4, 2, 64, **kw)


def _code(fn, *a, **kw):
    with pytest.raises(F.FlashCPError) as ei:
        fn(*a, **kw)
    return ei.value.code


def test_the_score_function_is_kept():
    s = [0.0, 0.5, 1024.0, 2.0 ** -8]
    v = _view(cap=30.0, slopes=s)
    cap, got = v.score
    assert cap == 30.0 and got.tolist() == s
    assert _view(cap=30.0).score == (30.0, None) and _view(cap=1000.0).score == (1000.0, None)
    cap, got = _view(slopes=np.zeros(4)).score
    assert cap == 0.0 and got.tolist() == [0.0] * 4
    assert _view().score == (0.0, None) and _view(cap=0.0).score == (0.0, None)
    # any float sequence, wherever it lies
    raw = np.zeros(4 * 4 + 1, dtype=np.uint8)
    raw[1:] = np.frombuffer(np.array(s, dtype=np.float32).tobytes(), dtype=np.uint8)
    assert _view(slopes=raw[1:].view(np.float32)).score[1].tolist() == s
    assert _view(slopes=np.array(s)[::-1]).score[1].tolist() == s[::-1]
    v.close()
    with pytest.raises(ValueError):
        v.score


def test_a_plain_view_keeps_its_tables():
    """A score function without cap and slopes is none, and a cap alone adds no
    table; tile maps, splits and workspaces are those of the plain view."""
    plain = _view()
    lib = F.lib()
    a, n = np.ascontiguousarray(CU), 3
    plan = np.ascontiguousarray(F.fc_plan_per_doc(CU, 2), dtype=np.int32)
    h = C.c_void_p()
    none = F.Score(0.0, None)
    for score in (None, C.byref(none)):
        assert lib.fc_view_create_scored(a.ctypes.data_as(F.I32P), n, plan.ctypes.data_as(C.POINTER(F.Shard)),
                                         len(plan), 2, 1, 4, 2, 64, None, score, C.byref(h)) == 0
        info = F.ViewInfo()
        assert lib.fc_view_get_info(h, C.byref(info)) == 0 and info.as_dict() == plain.info
        lib.fc_view_destroy(h)
    capped, biased = _view(cap=5.0), _view(slopes=np.ones(4))
    assert capped.info == plain.info
    assert biased.info["table_bytes"] > plain.info["table_bytes"]
    for v in (capped, biased):
        # (a bias steep enough for most keys to be out of reach takes row norms too)
        more = 256 * 4 * (4 + 2 * 2) if v is biased else 0
        assert v.workspace_size() == tuple(n + more for n in plain.workspace_size())
        for x, y in ((v.export(), plain.export()), (v.export_launch(), plain.export_launch())):
            assert all(np.array_equal(x[k], y[k]) for k in x)
    assert _view(slopes=np.zeros(4)).workspace_size() == plain.workspace_size()
    # an empty rank
    cu = np.array([0, 10], dtype=np.int32)
    v = F.View(cu, [[0, 0, 0, 10]], 2, 1, 4, 4, 64, cap=5.0, slopes=np.ones(4))
    assert v.info["t_q"] == 0


def test_score_refusals():
    for cap in (-1.0, math.nan, math.inf, 2.0 ** -7, 1025.0, -math.inf):
        assert _code(_view, cap=cap) == -1
    _view(cap=F.CAP_MIN).close()
    _view(cap=F.CAP_MAX).close()
    for bad in (-0.1, math.nan, math.inf, 1025.0):
        assert _code(_view, slopes=[0.1, 0.1, bad, 0.1]) == -1
    for s in ([0.1] * 3, [0.1] * 5, 0.1, [[0.1] * 4]):
        with pytest.raises(ValueError):
            _view(slopes=s)
    # distances are counted in fp32: 2^24 tokens are the longest document
    big = np.array([0, (1 << 24) + 1], dtype=np.int32)
    plan = [[0, 0, 0, (1 << 24) + 1]]
    assert _code(F.View, big, plan, 1, 0, 4, 4, 64, slopes=np.ones(4)) == -4
    assert F.lib().fc_view_get_score(None, None, None, None) == -1
    assert F.lib().fc_view_create_scored(None, 1, None, 0, 1, 0, 4, 4, 64, None, None, None) == -1


@pytest.mark.parametrize("kw", [
    dict(), dict(base=500000.0), dict(scaling="linear", factor=3.0), dict(scaling="base", factor=8.0),
    dict(scaling="bands", factor=8.0, context=8192.0), dict(scaling="bands", factor=2.0, context=100.0, low=0.5, high=7.0),
    dict(scaling="yarn", factor=32.0, context=4096.0), dict(scaling="yarn", factor=1.0, context=50.0),
    dict(scaling="yarn", factor=4.0, context=2048.0, low=2.0, high=64.0),
])
@pytest.mark.parametrize("m", [4, 24, 64, 128])
def test_frequencies(m, kw):
    w, amp = F.fc_rope_freqs(m, **kw)
    kw = dict(kw)
    w2, amp2 = R.frequencies(m, **kw)
    # (a power, a logarithm and a few products in 64 bits)
    assert np.allclose(w, w2, rtol=1e-13, atol=0) and amp == np.float32(amp2)
    r = F.Rope(m, **kw)
    assert np.array_equal(r.inv_freq, w) and r.amplitude == amp


def test_frequency_refusals():
    ok = dict(dim=64, base=10000.0, scaling="yarn", factor=2.0, context=100.0)
    F.fc_rope_freqs(**ok)
    for bad in (dict(dim=0), dict(dim=7), dict(dim=130), dict(base=1.0), dict(base=math.nan), dict(base=math.inf),
                dict(factor=0.5), dict(factor=math.nan), dict(low=0.0), dict(low=32.0), dict(high=math.inf),
                dict(context=0.0), dict(context=math.nan), dict(dim=2, scaling="base")):
        assert _code(F.fc_rope_freqs, **dict(ok, **bad)) == -1, bad
    with pytest.raises(ValueError):
        F.fc_rope_freqs(64, scaling="other")
    with pytest.raises(ValueError):
        F.Rope(64, inv_freq=np.ones(31))
    w = (C.c_double * 64)()
    a = C.c_float()
    assert F.lib().fc_rope_freqs(64, 10000.0, 5, 1.0, 1.0, 4.0, 0.0, w, C.byref(a)) == -1
    assert F.lib().fc_rope_freqs(64, 10000.0, 0, 1.0, 1.0, 4.0, 0.0, None, C.byref(a)) == -1
    assert F.lib().fc_rope_freqs(64, 10000.0, 0, 1.0, 1.0, 4.0, 0.0, w, None) == -1


def _rows(i=256, o=1 << 20, si=0, so=0):
    return F._ROWS.pack(i, si, o, so)


def test_rows_rejected_before_launch():
    """Nothing is dereferenced or launched: an unbound view is refused first, a bound
    one's arguments after it (the view is bound to an address by hand)."""
    lib = F.lib()
    v = _view()
    h, rope = v.handle, F.Rope(64)
    q, k, w = _rows(), _rows(1 << 22, 1 << 23), _rows(1 << 24, 1 << 25)
    assert lib.fc_rope_fwd(h, rope._p, q, k, w, None) == -5
    assert lib.fc_rope_bwd(h, rope._p, 1, q, k, None, None, None, None) == -5
    assert lib.fc_kv_gather_rope(h, rope._p, 256, 256, 1000, 256, 256, 256, 256, None) == -5
    assert lib.fc_rope_fwd(None, rope._p, q, k, w, None) == -1
    v.close()


def test_bound_rows_refusals_under_sanitizers(tmp_path):
    """The same entry points on a bound view, in a host build without a GPU (stub
    launchers that check their tables), under AddressSanitizer and
    UndefinedBehaviorSanitizer: refusals, overlaps, in-place rows, row blocks."""
    import shutil
    import subprocess
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    host = os.path.join(root, "paper_2606_08476_amd", "csrc", "host")
    exe = tmp_path / "rows_driver"
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(root, "include"),
           *[os.path.join(host, f) for f in ("plan.cpp", "view.cpp", "api.cpp", "rope.cpp")],
           os.path.join(root, "tests", "sanitize", "rows_driver.cpp"), "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert "all checks passed" in r.stdout
