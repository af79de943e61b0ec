"""Loads of tokens that the layer for a few tokens holds in LDS, and of its hidden rows, stay in their rows and find their channels, at every width (on the host; no
GPU)."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1705_01598_amd", "csrc")


def _walk(tmp_path, header, *arguments):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    (tmp_path / "few_places.hpp").write_text(header)
    exe = str(tmp_path / "few_places")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-I" + str(tmp_path), os.path.join(ROOT, "tests", "few_places.cpp"), "-o", exe], check=True)
    return subprocess.run([exe, *arguments], capture_output=True, text=True)


def test_loads_stay_in_their_rows(tmp_path):
    r = _walk(tmp_path, open(os.path.join(CSRC, "few_places.hpp")).read())
    assert r.returncode == 0 and r.stdout.startswith("ok:"), r.stdout


def test_the_walk_finds_a_load_that_leaves_its_row(tmp_path):
    """Loads that ignore the row's end: the second of two steps that are requested at once lies behind it."""
    header = open(os.path.join(CSRC, "few_places.hpp")).read()
    broken = header.replace("return i < depth ? i : 0u;", "return i + 0 * depth;")
    assert broken != header
    r = _walk(tmp_path, broken, "tokens")
    assert r.returncode == 1 and r.stdout.startswith("width 1, 2 steps"), r.stdout
    r = _walk(tmp_path, broken)
    assert r.returncode == 1 and r.stdout.startswith("hidden rows of 1, pieces of 4"), r.stdout


def test_the_kernels_load_by_these_rules():
    text = open(os.path.join(CSRC, "few.hpp")).read()
    assert "load_vec<T, N, true>(row + start_in(i, depth))" in text
    # columns in filled rows go by the row's end too, but where a step is there as a whole
    ready = text[text.index("template <typename E, int P, bool FILLED = false> struct Ready"):]
    assert re.search(r"kReach = FILLED && REACH != Reach::kAll \? Reach::kEnd : REACH;\s+.*load_reach<kReach, E, N, ALIGNED \|\| FILLED>", ready[:ready.index("};\n//")])
