"""What the attention kernel's waves tell each other goes through words that a barrier orders (tests/kv_waves_check.cpp, built
here with threads as waves)."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2408_04323_amd", "csrc")


@pytest.mark.parametrize("sanitize", [[], ["-fsanitize=thread"]], ids=["values", "races"])
def test_waves_agree_without_races(tmp_path, sanitize):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path / "kv_waves_check")
    subprocess.run([cxx, "-O1", "-g", "-std=c++17", "-Wno-unknown-pragmas", *sanitize, "-I", CSRC, os.path.join(ROOT, "tests", "kv_waves_check.cpp"),
                    "-o", exe, "-lpthread"], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "WARNING: ThreadSanitizer" not in r.stderr, (r.stdout, r.stderr[-2000:])


def test_the_kernel_has_no_other_way_to_the_words():
    """The words are handed on and never indexed outside of kv_waves.h."""
    text = open(os.path.join(CSRC, "kv_attn.h")).read()
    assert "any_of_waves<" in text and "most_of_waves<" in text
    assert not re.search(r"\bflag\s*\[|\bwords\s*\[", text)
