"""Drafted tokens at the largest extents that the calls take, where no GPU is needed (tests/draft_limits_check.cpp)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2504_12526_amd", "csrc")


def _check(tmp_path, include):
    exe = os.path.join(str(tmp_path), "draft_limits_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", include, "-o", exe, os.path.join(ROOT, "tests", "draft_limits_check.cpp")], check=True)
    return subprocess.run([exe], capture_output=True, text=True, timeout=60)


def test_shares_of_the_longest_sequences_and_one_workspace_for_smaller_calls(tmp_path):
    r = _check(tmp_path, CSRC)
    assert r.returncode == 0 and ": ok" in r.stdout, r.stdout


@pytest.mark.parametrize("old,new,says", [
    ("for (int qb = 1; qb <= 2; ++qb) {", "for (int qb = 2; qb <= 2; ++qb) {", "workspace"),
    ("if (max_kv <= kWholeTokens) return 0;", "if (max_kv <= kManyWholeTokens) return 0;", "workspace"),
    ("return x.tiles * ((x.steps + wk - 1) / wk); }", "return x.tiles * x.steps; }", "shortest"),
    ("hi = rounds / (workgroups - tiles) + 1;", "hi = rounds / workgroups + 1;", "room"),
    ("uint32_t lo = rounds / workgroups,", "uint32_t lo = rounds / workgroups + 3,", "shortest"),
])
def test_a_planted_mistake_is_caught(tmp_path, old, new, says):
    """Planted in a copy of the header, on the CPU."""
    text = open(os.path.join(CSRC, "mom_draft.h")).read()
    assert text.count(old) == 1, old
    shutil.copy(os.path.join(CSRC, "mom_mx.h"), str(tmp_path))
    with open(os.path.join(str(tmp_path), "mom_draft.h"), "w") as f:
        f.write(text.replace(old, new))
    r = _check(tmp_path, str(tmp_path))
    assert r.returncode != 0 and says in r.stdout, r.stdout
