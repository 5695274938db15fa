"""Which form of the attention kernel the cases of tests/kv_cases.py take, by the library's own plan (tests/kv_plan_check.cpp,
built here against its internal header): every form has cases whose values are compared on the GPU, also when the plan's
thresholds change."""
import os
import shutil
import subprocess

import pytest

import kv_cases

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path_factory.mktemp("plan") / "kv_plan_check")
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2408_04323_amd", "csrc"),
                    os.path.join(ROOT, "tests", "kv_plan_check.cpp"), "-o", exe], check=True)

    def ask(lines):
        out = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(lines)
        return [tuple(x if i == 0 else int(x) for i, x in enumerate(line.split())) for line in out]
    return ask


def test_the_cases_take_the_forms_that_they_are_for(plan):
    names = list(kv_cases.CASES)
    for name, (kind, waves, buffers, parts, _) in zip(names, plan([kv_cases.plan_line(kv_cases.CASES[n]) for n in names])):
        assert (kind, waves, buffers, parts > 1) == kv_cases.CASES[name]["form"], (name, parts)


def test_every_form_has_a_case():
    have = {(c["d"], c["kind"], c["cache"] == "f8") + c["form"] for c in kv_cases.CASES.values()}
    for d in kv_cases.DIMS:
        for kind in kv_cases.TYPES:
            for f8 in (False, True):
                wide = d * (1 if f8 else 2) > 256
                want = {("few", w, 0) for w in ({4} if wide else {4, 8})} | {("tiles", 4, 4 if d == 192 and f8 else 2)}
                for form in want:
                    for parts in (False, True):
                        assert (d, kind, f8) + form + (parts,) in have, (d, kind, f8, form, parts)


def test_parts_of_few_rows(plan):
    """No launch that joins parts for few keys: one part up to 768 keys (four waves) and 1024 (eight), then none of less than
    128, few workgroups more than compute units unless they are more anyway, and never more parts than can be asked for."""
    asked = [(seqs, heads, dim, size, keys) for seqs in (1, 3, 16, 40, 300) for heads in (1, 8) for dim in (64, 128, 192, 256)
             for size in (1, 2) for keys in (1, 129, 513, 768, 769, 1024, 1025, 1500, 2047, 4000, 4097, 9000, 65536, 2 ** 30)]
    got = plan([f"{s} {h} {h} {d} {b} {s} 1 {k} 0" for s, h, d, b, k in asked])
    for (seqs, heads, dim, size, keys), (kind, waves, _, parts, part) in zip(asked, got):
        at = (seqs, heads, dim, size, keys, waves, parts, part)
        assert kind == "few" and parts >= 1 and part % 128 == 0, at
        assert (parts - 1) * part < keys and parts * part + 128 > keys, at
        if keys <= (1024 if waves == 8 else 768):
            assert parts == 1, at
        if parts > 1:
            assert keys - (parts - 1) * part >= 128 and part >= 256, at
            assert seqs * heads * parts <= (256 if seqs * heads <= 256 else 2048), at
