"""Registers, LDS and spills of the built kernels of the feed-forward block, the token rows and AdamW (no GPU):
what their launches count on."""

import os
import re
import subprocess
import tempfile

from tests.kernel_resources import READELF, VGPR_UNIT, VGPRS_PER_LANE, _code_objects, kernels, resources

OBJDUMP = os.path.join(os.path.dirname(READELF), "llvm-objdump")

LDS = 160 * 1024
MINE = ("ffn_block", "rows_", "adamw_")


def test_no_kernel_spills():
    got = {n: r for n, r in resources().items() if n.startswith(MINE)}
    # products: six of mid, wide and of each few height; weights' gradients (float32, bf16, bf16 added) and their join by type; float32: four and weights'
    assert sum(n.startswith("ffn_block") for n in got) == 6 * 4 + 3 + 2 + 5, sorted(got)
    # gather by size, combine by two types, its gradient by three, each plain and past the caches; the gate's by type
    assert sum(n.startswith("rows_") for n in got) == 4 + 8 + 16 + 2, sorted(got)
    assert sum(n.startswith("adamw_") for n in got) == 4, sorted(got)
    for name, r in got.items():
        assert (r["vgpr_spill_count"], r["sgpr_spill_count"], r["private_segment_fixed_size"]) == (0, 0, 0), name


def test_ring_tiles_fit_a_cu():
    for name, (vgprs, lds) in kernels().items():
        if name.startswith(("ffn_block_mid", "ffn_block_wide", "ffn_block_few")):
            waves = 2 if name.startswith("ffn_block_few") and name.endswith(", 8>") else 1  # to a SIMD
            assert lds <= LDS and vgprs * waves <= VGPRS_PER_LANE, (name, vgprs, lds)


def test_two_weight_tiles_share_a_cu():
    got = {n: v for n, v in kernels().items() if n.startswith("ffn_block_weights")}
    assert len(got) == 3
    for name, (vgprs, lds) in got.items():
        assert 2 * lds <= LDS and 2 * vgprs <= VGPRS_PER_LANE, (name, vgprs, lds)


def test_row_kernels_leave_room_for_four_waves_to_a_simd():
    for name, (vgprs, lds) in kernels().items():
        if name.startswith(("rows_", "adamw_")):
            assert vgprs <= VGPRS_PER_LANE // 4 // VGPR_UNIT * VGPR_UNIT and lds == 0, (name, vgprs, lds)


def _listings(prefix):
    """{kernel: its instructions as built} of the gfx950 code objects in the library."""
    got = {}
    for elf in _code_objects():
        with tempfile.NamedTemporaryFile(suffix=".co") as f:
            f.write(elf)
            f.flush()
            text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", f.name], stdout=subprocess.PIPE, text=True, check=True).stdout
        for name, body in re.findall(r"^[0-9a-f]+ <(\w+)>:\n(.*?)(?=^[0-9a-f]+ <|\Z)", text, re.M | re.S):
            if prefix in name:
                got[name] = [line.split("//")[0].strip() for line in body.split("\n") if line.strip()]
    return got


def test_few_tiles_read_a_slot_before_it_is_filled_again():
    """A wave's own ring has no barrier: each block's LDS reads are waited for before the next transfer into LDS is
    issued, and come after the wait for the transfers of their block."""
    got = _listings("ffn_block_few")
    assert len(got) == 12
    for name, lines in got.items():
        reading, landed, transfers = False, False, 0
        for line in lines:
            if line.startswith("ds_read"):
                assert landed, (name, line)
                reading = True
            elif line.startswith("s_waitcnt"):
                reading = reading and "lgkmcnt(0)" not in line
                landed = landed or "vmcnt" in line
            elif line.startswith("buffer_load") and line.endswith("lds"):
                assert not reading, (name, line)
                transfers += 1
                landed = False
        assert transfers > 0, name
