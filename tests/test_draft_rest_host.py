"""What refusals leave where no GPU is needed: powers, weights and rests (tests/draft_rest_check.cpp)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2504_12526_amd", "csrc")


def _check(tmp_path, include):
    exe = os.path.join(str(tmp_path), "draft_rest_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", include, "-o", exe, os.path.join(ROOT, "tests", "draft_rest_check.cpp")], check=True)
    return subprocess.run([exe], capture_output=True, text=True, timeout=60)


def test_powers_weights_and_rests(tmp_path):
    r = _check(tmp_path, CSRC)
    assert r.returncode == 0 and ": ok" in r.stdout, r.stdout


@pytest.mark.parametrize("old,new,says", [
    ("double y = fma(f, kStep * kStep * kStep / 6, kStep * kStep / 2);", "double y = kStep * kStep / 2;", "power"),
    ("f = fma(d, k, kMagic - moved);", "f = d * k - (moved - kMagic);", "far power"),
    ("c12 = c11 * kLn2 / 12, c13 = c12 * kLn2 / 13;", "c12 = 0, c13 = 0;", "power of two"),
    ("return d > -s.limit ? ldexp(root * x.rest, (int32_t)x.whole >> kPowerBits) : 0.0;", "return ldexp(root * x.rest, (int32_t)x.whole >> kPowerBits);", "weight of a flat row"),
    ("+ (j << (20 - kPowerBits))) << 32", "+ (x.whole << (20 - kPowerBits))) << 32", "weight"),
    ("t * (1100.0 * 0.6", "t * (10.0 * 0.6", "weight of what is far below"),
    ("    if (n.low < low) n.low = nextafterf(n.low, INFINITY);\n", "", "near"),
    ("return x >= n.low ? y.two * y.rest : 0.0;", "return y.two * y.rest;", "near weight of what is masked"),
    ("l.drafted, l.k) * l.draft_inverse;", "l.drafted, l.k) * l.target_inverse;", "rest"),
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
