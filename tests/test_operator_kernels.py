"""Registers, LDS and spills of the built MX FP4 and balance-loss kernels (no GPU): what
their launches count on."""

from tests.kernel_resources import VGPR_UNIT, VGPRS_PER_LANE, kernels, resources

LDS = 160 * 1024


def _mine():
    return {n: r for n, r in resources().items() if n.startswith(("mx4_", "balance_"))}


def test_no_kernel_spills():
    got = _mine()
    assert len(got) == 2 + 1 + 2 + 5 + 14 + 3 * 10 + 3, sorted(got)  # quantize, pack, dequantize, ring, streaming, balance
    for name, r in got.items():
        assert (r["vgpr_spill_count"], r["sgpr_spill_count"], r["private_segment_fixed_size"]) == (0, 0, 0), name


def test_two_ring_workgroups_share_a_cu():
    """Four waves each, one to a SIMD: half a SIMD's registers and half the LDS."""
    ring = {n: v for n, v in kernels().items() if n.startswith("mx4_ring_kernel")}
    assert len(ring) == 5
    for name, (vgprs, lds) in ring.items():
        assert 2 * vgprs <= VGPRS_PER_LANE and 2 * lds <= LDS, (name, vgprs, lds)


def test_streaming_waves_to_a_simd():
    """Two with 64-row tiles, three with 32 rows and two panels, four with one panel."""
    got = kernels()
    for gated, outs in (("false", (0, 1)), ("true", (0, 1, 2))):
        for out in outs:
            for blocks, panels, waves in ((2, 2, 2), (2, 1, 2), (1, 2, 3), (1, 1, 4)):
                if gated == "true" and panels == 1:
                    continue
                vgprs, lds = got[f"mx4_stream_kernel<{blocks}, {panels}, {gated}, {out}>"]
                assert vgprs <= VGPRS_PER_LANE // waves // VGPR_UNIT * VGPR_UNIT and lds == 0, (blocks, panels, gated, out)


def test_balance_workgroups_fit():
    """The largest, 1024 experts in one launch, within a CU's LDS; the pieces two to a CU."""
    for name, (vgprs, lds) in kernels().items():
        if name.startswith("balance_"):
            assert (2 if name.startswith("balance_pieces") else 1) * lds <= LDS, (name, lds)
            assert vgprs <= VGPRS_PER_LANE // (4 if name.startswith(("balance_small", "balance_join", "balance_total")) else 2), name
