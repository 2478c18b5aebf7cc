"""The rule that picks the feed-forward block's tiles, on the host (no GPU): tests/native/ffn_form_check.cpp
compiles csrc/ffn_form.h for the host."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_00993_amd", "csrc")
FEW8, FEW32, MID, WIDE = range(4)


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("g++ not found")
    exe = str(tmp_path_factory.mktemp("ffn_form") / "ffn_form_check")
    cmd = [cxx, "-O1", "-std=c++17", "-Wall", f"-I{CSRC}", os.path.join(ROOT, "tests", "native", "ffn_form_check.cpp"), "-o",
           exe]
    p = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert p.returncode == 0, f"build failed:\n{' '.join(cmd)}\n{p.stdout}"
    return exe


def _ask(check, *args):
    r = subprocess.run([check, *map(str, args)], stdout=subprocess.PIPE, text=True, timeout=60)
    assert r.returncode == 0
    return [int(v) for v in r.stdout.split()]


def products(check, rows, groups, H, I):
    """(tiles, rows of one) of the four products."""
    return [tuple(_ask(check, "form", kind, rows, groups, n, k)[:2])
            for kind, n, k in ((0, I, H), (1, H, I), (2, I, H), (3, H, 2 * I))]


def test_launches_cover_their_rows(check):
    r = subprocess.run([check], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), r.stdout[:2000]


def test_gpu_cases_reach_every_form(check):
    from tests.test_gpu_ffn_forms import CASES, WEIGHTS, rows_of

    seen = [set() for _ in range(4)]
    for name, (where, H, I) in CASES.items():
        got = products(check, rows_of(CASES[name]), 1 if isinstance(where, int) else len(where) - 1, H, I)
        named = {"few8": FEW8, "few32": FEW32, "mid": MID, "wide": WIDE}[name.split("-")[0]]
        assert named in {t for t, _ in got}, (name, got)
        for kind, (t, rows) in enumerate(got):
            seen[kind].add(t)
            if t == MID:
                seen[kind].add(("mid", rows))
    for kind in range(4):
        assert {FEW8, FEW32, MID, WIDE} <= seen[kind], (kind, seen[kind])
        assert ("mid", 160) in seen[kind] and any(("mid", r) in seen[kind] for r in (32, 64, 96, 128)), (kind, seen[kind])
    for name, (rows, groups, m, n) in WEIGHTS.items():
        (parts,) = _ask(check, "parts", rows, groups, m, n)
        assert (parts > 1) == name.startswith("parts"), (name, parts)


def test_workspace_is_what_the_parts_need(check):
    from paper_2609_00993_amd import moepd as M

    for rows, groups, m, n in ((9000, 1, 272, 264), (300, 3, 272, 264), (16000, 1, 512, 512), (0, 1, 8, 8), (1, 1024, 8, 8)):
        (parts,) = _ask(check, "parts", rows, groups, m, n)
        st, need = M.moe_ffn_weight_workspace(rows, groups, m, n)
        assert st == M.MOE_OK and need == (4 * parts * groups * m * n if parts > 1 else 0) and need <= 1 << 27
