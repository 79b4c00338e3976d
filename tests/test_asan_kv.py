"""The calls over a paged cache and the verification of drafts under AddressSanitizer (CPU): tests/asan/kv_checks.cpp in the
place of host_checks.cpp, in a build of its own."""
import os
import re
import shutil
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.join(HERE, "asan"))


@pytest.mark.skipif(not os.path.exists("/opt/rocm/llvm/bin/clang++"), reason="needs the ROCm clang")
def test_cache_calls_under_asan(tmp_path, monkeypatch):
    import build_and_run
    src = tmp_path / "src"
    src.mkdir()
    shutil.copy(os.path.join(HERE, "asan", "fake_hip_runtime.cpp"), src)
    shutil.copy(os.path.join(HERE, "asan", "kv_checks.cpp"), src / "host_checks.cpp")
    monkeypatch.setattr(build_and_run, "HERE", str(src))
    exe = build_and_run.build(str(tmp_path / "out"))
    r = subprocess.run([exe], capture_output=True, text=True,
                       env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1:halt_on_error=1"))
    assert r.returncode == 0, r.stdout + r.stderr[-4000:]
    m = re.search(r"kv checks ok: (\d+) checks, (\d+) launches", r.stdout)
    assert m and int(m.group(1)) > 20000 and int(m.group(2)) > 2500
