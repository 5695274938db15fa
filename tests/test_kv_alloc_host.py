"""The cache calls return a status where the library's host memory runs out (tests/kv_alloc_check.cpp, built here)."""
import os
import shutil
import subprocess

import pytest

from paper_2408_04323_amd._native import LIB_PATH

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NO_MEMORY = -5


def test_no_exception_leaves_a_cache_call(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path / "kv_alloc_check")
    subprocess.run([cxx, "-O1", "-g", "-std=c++17", "-rdynamic", "-I", os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "tests", "kv_alloc_check.cpp"), "-o", exe, "-ldl"], check=True)
    env = dict(os.environ, HIP_VISIBLE_DEVICES="-1", ROCR_VISIBLE_DEVICES="-1")  # no launch may come of it
    r = subprocess.run([exe, LIB_PATH], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, (r.returncode, r.stdout, r.stderr[-500:])
    lines = [line.split(" ", 3) for line in r.stdout.splitlines()]
    assert [x[0] for x in lines] == ["scoot_kv_assign", "scoot_kv_write", "scoot_kv_attention"]
    for name, thrown, status, message in lines:
        assert int(thrown) > 0 and int(status) == NO_MEMORY and "allocation" in message, (name, thrown, status, message)
