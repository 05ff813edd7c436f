"""min-p's cut (csrc/min_p_cut.h), the same code compiled for the host: the smallest logit that is kept, found in a bounded number of steps."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("min_p_cut") / "check")
    clang = shutil.which("amdclang++") or "/opt/rocm/llvm/bin/clang++"
    subprocess.check_call([clang, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(HERE, "wave_on_host"), "-o", exe, os.path.join(HERE, "min_p_cut_check.cpp")])
    return exe


@pytest.mark.parametrize("top,temperature,min_p", [(0.0866413191, 0.0650000051, 0.263699979), (1.79451227, 0.782053828, 0.100800216), (0.0, 1.0, 1.0), (-0.0, 1.0, 0.5),
                                                   (3e38, 1e30, 1e-30), (-3.4e38, 3e38, 0.01), (1e-45, 1e-45, 0.5), (5.0, 1e-30, 0.1), (1.0, 1e30, 1.0), (2.0, 1.0, 1e-45)])
def test_cuts_at_the_ends_and_next_to_zero(check, top, temperature, min_p):
    r = subprocess.run([check, repr(top), repr(temperature), repr(min_p)], capture_output=True, text=True, timeout=20)
    assert r.returncode == 0, r.stdout


@pytest.mark.parametrize("seed", [1, 2])
def test_any_cut(check, seed):
    r = subprocess.run([check, "random", "200000", str(seed)], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stdout
