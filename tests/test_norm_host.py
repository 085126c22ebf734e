"""Head norms without a GPU: the entry points on bound views in a host build under
AddressSanitizer and UndefinedBehaviorSanitizer, with stub launchers that check every
table, row share and partial row; and the binding's refusals."""
import os
import shutil
import subprocess

import pytest
import torch

from paper_2606_08476_amd import flashcp as F

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_entry_points_under_sanitizers(tmp_path):
    host = os.path.join(ROOT, "paper_2606_08476_amd", "csrc", "host")
    exe = tmp_path / "norm_driver"
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"),
           *[os.path.join(host, f) for f in ("plan.cpp", "view.cpp", "api.cpp", "rope.cpp", "norm.cpp")],
           os.path.join(ROOT, "tests", "sanitize", "norm_driver.cpp"), "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert "all checks passed" in r.stdout


def test_binding_refusals():
    with pytest.raises(TypeError):
        F.HeadNorm(torch.ones(64))           # host memory
    with pytest.raises(TypeError):
        F.HeadNorm([1.0] * 64)
    n = F.HeadNorm(None, eps=1e-5, offset=1.0, centred=True)
    assert (n.weight, n.offset, n.centred) == (None, 1.0, True)
    v = F.View([0, 10], [[0, 0, 0, 10]], 1, 0, 4, 2, 64)
    assert F.fc_norm_rope_workspace(v, n, None) > 0 and F.fc_norm_rope_workspace(v, None, None) == 0
    with pytest.raises(F.FlashCPError) as e:
        F.fc_norm_rope_workspace(v, F.HeadNorm(eps=0.0), None)
    assert e.value.code == -1
    with pytest.raises(ValueError):
        F.fc_norm_rope_bwd(v, None, n, n, *[None] * 13, dw_q=torch.ones(64))
    v.close()
