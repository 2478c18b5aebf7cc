"""The MX FP4 products' tiles on the host (no GPU): tests/native/mx4_form_check.cpp
compiles csrc/mx4_form.h for the host."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_00993_amd", "csrc")


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("g++ not found")
    exe = str(tmp_path_factory.mktemp("mx4_form") / "mx4_form_check")
    cmd = [cxx, "-O1", "-std=c++17", "-Wall", f"-I{CSRC}", os.path.join(ROOT, "tests", "native", "mx4_form_check.cpp"),
           "-o", exe]
    p = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert p.returncode == 0, f"build failed:\n{' '.join(cmd)}\n{p.stdout}"
    return exe


def test_lane_offsets_fit(check):
    r = subprocess.run([check], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), r.stdout[:2000]


def _form(check, case):
    """(ring, 32-row blocks, panels, waves) of a case's launch."""
    width = -(-case.N // 256) * 256 if case.out == "fp4" else case.N
    r = subprocess.run([check, "form"] + [str(int(v)) for v in (case.gated, width, case.rows, len(case.group_rows),
                                                                -(-case.K // 256), case.rows)],
                       stdout=subprocess.PIPE, text=True, timeout=60)
    ring, blocks, panels, waves = (int(v) for v in r.stdout.split())
    return bool(ring), blocks, panels, waves


def _ring_blocks(rows):
    """The heights, in 32-row blocks, of the ring tiles that share a group's rows."""
    if not rows:
        return set()
    per = -(-rows // -(-rows // 128))
    return {-(-min(per, rows - at) // 32) for at in range(0, rows, per)}


def test_gpu_cases_reach_every_form(check):
    """tests/test_gpu_mx4_forms.py compares every kernel of the products with the oracle: ring tiles
    of every height at one slice and at numbers of slices that leave the ring at each slot and
    parity, odd widths, strides, gaps and clamped offsets; streaming tiles of both heights and panel
    counts, of one to eight waves with slices shared evenly and not."""
    from tests.test_gpu_mx4_forms import CASES, KINDS

    forms = [(c, *_form(check, c)) for c in CASES]
    for c, ring, *_ in forms:
        assert ring == c.name.startswith("ring"), c.name
    for gated, out in KINDS:
        mine = [f for f in forms if f[0].gated == gated and f[0].out == out]
        ring = [f[0] for f in mine if f[1]]
        slices = {-(-c.K // 256) for c in ring if len(c.group_rows) == 20}
        assert {1, 2, 3, 4, 5, 7} <= slices
        for n in slices:
            heights = set().union(*(_ring_blocks(r) for c in ring if -(-c.K // 256) == n for r in c.group_rows))
            assert heights == {1, 2, 3, 4}, (gated, out, n)
        assert any(len(c.group_rows) > 128 for c in ring) and any(c.groups is None for c in ring)
        assert any(c.before for c in ring) and any(c.clamp for c in ring)
        if out != "fp4":
            assert any(c.N % 32 for c in ring) and any(c.stride % 4 and c.pad for c in ring)
        stream = [f for f in mine if not f[1]]
        assert {(b, p) for _, _, b, p, _ in stream} == {(b, p) for b in (1, 2) for p in ((2,) if gated else (1, 2))}
        assert len({w for *_, w in stream}) >= 3, (gated, out)
        assert any(-(-f[0].K // 256) % f[4] for f in stream if f[4] > 1)
    plain = [f for f in forms if not f[1]]
    for gated in (False, True):
        assert {f[4] for f in plain if f[0].gated == gated} == {1, 2, 4, 8}
        # a wave that takes slices alone, two buffers of them in turn
        assert any(f[4] == 1 and -(-f[0].K // 256) >= 3 for f in plain if f[0].gated == gated)
