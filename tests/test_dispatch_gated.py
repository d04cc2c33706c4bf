"""Which kernels slope_gated_fwd takes (host only, no GPU), and that the shapes of its GPU tests reach all of them."""
import pytest

from paper_2405_16325_amd import binding as sl
from tests.test_gpu_gated import BESIDE, LARGE, SHAPES

SMALL_BATCH, SLABS, TILE, GENERAL, ROW_SPLIT, REST, TWO_TILES = range(7)


def plan(b, d_ff, d_in, r=0, **more):
    return sl.slope_gated_fwd_plan(b, d_in, d_ff, r, **more)


def test_regimes():
    assert plan(1, 2048, 768)["product"] == SMALL_BATCH
    assert plan(1, 24576, 9216)["product"] == ROW_SPLIT
    assert plan(1, 24576, 9216, kept=8)["product"] == ROW_SPLIT
    assert plan(1, 24576, 9216, kept=8, with_workspace=False)["product"] == TILE         # the small-batch kernels leave sums of what is kept
    assert plan(128, 200, 4096)["product"] == SLABS and plan(128, 200, 4096, with_workspace=False)["product"] == TILE
    assert plan(300, 1000, 1000) == {"product": GENERAL, "rows": 64, "tokens": 64, "slabs": 1, "xl": 0, "padded": 0}
    p = plan(1000, 1000, 1000)
    assert (p["product"], p["padded"]) == (TILE, 1024) and plan(1000, 1000, 1000, with_workspace=False)["product"] == GENERAL
    p = plan(16384, 24576, 9216)
    assert (p["product"], p["rows"], p["tokens"]) == (TILE, 256, 256)


def test_workgroups_of_64_rows_where_they_save_a_thin_round():
    for d_ff, d_in, rows in ((24576, 9216, 64), (20480, 5120, 64), (18432, 9216, 48), (12288, 9216, 48), (27648, 10240, 48)):
        assert plan(1, d_ff, d_in)["rows"] == rows, (d_ff, d_in)
    assert plan(1, 2048, 16384) == {"product": ROW_SPLIT, "rows": 48, "tokens": 16, "slabs": 8, "xl": 0, "padded": 0}


def test_codes_from_no_tile_of_192_rows():
    """A wavefront's rows of a tile that writes 8-bit blocks are whole blocks of 32 elements."""
    tall = set()
    for b in (40, 100, 128, 300, 777, 1000, 2048, 5000):
        for d_ff in (96, 1000, 2176, 4352, 13648, 24576):
            for d_in in (128, 2112, 2560, 4352):
                p = plan(b, d_ff, d_in, kept=8)
                assert p["rows"] in (64, 128, 256) or p["product"] == SLABS
                tall.add(plan(b, d_ff, d_in, kept=16)["rows"])
    assert 192 in tall


@pytest.mark.parametrize("bad", [dict(b=0), dict(d_ff=12), dict(d_in=4), dict(d_ff=(1 << 22) + 8)])
def test_refusals(bad):
    args = dict(b=4, d_ff=64, d_in=64)
    args.update(bad)
    with pytest.raises(sl.SlopeError):
        plan(**args)
    with pytest.raises(sl.SlopeError):
        plan(4, 64, 64, 33)


def forms():
    """(product, rows, tokens, split, X L inside, whether the contraction ends inside what the kernel takes at a time)"""
    found = set()
    cases = [(b, f, i, r) for b, f, i in SHAPES for r in (0, 32, 160)] + LARGE
    for b, f, i, r in cases:
        for kept in (0, 8, 16):
            for ws in (True, False):
                if not ws and (r or kept):
                    continue
                p = plan(b, f, i, r, kept=kept, with_workspace=ws)
                whole = 256 if p["rows"] * p["tokens"] >= 192 * 128 else 128
                k = p["padded"] or i
                tail = k % whole != 0 if p["product"] != GENERAL else (i % 64 != 0) + (i % 128 != 0)
                split = p["slabs"] > 1 and p["product"] in (SLABS, ROW_SPLIT)
                found.add((p["product"], p["rows"], p["tokens"], split, p["xl"], int(tail)))
                if p["product"] in (SMALL_BATCH, ROW_SPLIT):
                    found.add((p["product"], p["rows"], p["tokens"], split, "kept" if kept else "h"))
    return found


def test_the_gpu_tests_reach_every_form():
    found = forms()
    for rows in (32, 48, 64):
        for xl in (0, 1):
            for tail in (0, 1):
                assert (SMALL_BATCH, rows, 16, False, xl, tail) in found, (rows, xl, tail)
    for rows in (32, 48):
        for xl in (0, 1):
            assert any((SMALL_BATCH, rows, 32, False, xl, tail) in found for tail in (0, 1)), (rows, xl)
    for tokens in (16, 32):
        assert (ROW_SPLIT, 48, tokens, True, 0, 0) in found
        for rows in (32, 48):
            assert (SMALL_BATCH, rows, tokens, False, "kept") in found
        assert (ROW_SPLIT, 48, tokens, True, "kept") in found
    assert (SMALL_BATCH, 64, 16, False, "kept") in found and (ROW_SPLIT, 48, 16, False, "kept") in found and (ROW_SPLIT, 64, 16, False, "kept") in found
    assert (ROW_SPLIT, 48, 16, False, 0, 0) in found and (ROW_SPLIT, 64, 16, False, 0, 0) in found
    for rows, tokens in ((128, 64), (128, 128), (192, 64), (256, 64), (256, 128)):
        for tail in (0, 1):
            assert (SLABS, rows, tokens, True, 0, tail) in found, (rows, tokens, tail)
    for rows, tokens in ((128, 64), (128, 96), (128, 128), (192, 64), (192, 96), (192, 128), (192, 192), (192, 256), (256, 128), (256, 192), (256, 256)):
        for tail in (0, 1):
            assert (TILE, rows, tokens, False, 0, tail) in found, (rows, tokens, tail)
    assert (TILE, 64, 64, False, 0, 0) in found
    for edge, tails in ((64, (1, 2)), (128, (1, 2))):
        for tail in tails:
            assert (GENERAL, edge, edge, False, 0, tail) in found, (edge, tail)
    assert (REST, 256, 256, False, 0, 0) in found and (REST, 256, 256, False, 0, 1) in found


def test_the_gpu_tests_reach_padded_copies():
    found = set()
    for b, f, i, r in [(b, f, i, r) for b, f, i in SHAPES for r in (0, 32, 160)] + LARGE:
        p = plan(b, f, i, r)
        if p["padded"]:
            assert p["padded"] % 64 == 0 and 0 < p["padded"] - i < 64
            found.add((p["product"], r > 0))
    assert {(TILE, False), (TILE, True), (SLABS, False), (SLABS, True)} <= found


def test_the_adapter_beside_the_product():
    """Where only h is wanted; what is kept needs the projections before they are finished."""
    found = set()
    for b, f, i, r in BESIDE:
        p = plan(b, f, i, r)
        found.add((p["product"], p["rows"], p["tokens"], f % 16 != 0))
        assert p["xl"] == 2, (b, f, i, r)
        assert plan(b, f, i, r, kept=8)["xl"] != 2 and plan(b, f, i, r, kept=16)["xl"] != 2 and plan(b, f, i, 0)["xl"] == 0
    for rows, tokens in ((32, 16), (48, 16), (64, 16), (32, 32), (48, 32)):
        assert {(SMALL_BATCH, rows, tokens, odd) for odd in (False, True)} & found, (rows, tokens)
    assert {(SLABS, rows, tokens) for rows, tokens in ((128, 64), (128, 128), (192, 64), (256, 64), (256, 128))} <= {k[:3] for k in found}
    assert {k[3] for k in found if k[0] == SLABS} == {k[3] for k in found if k[0] == SMALL_BATCH} == {False, True}


def test_whole_rounds_of_the_largest_tiles_and_others_behind():
    p = plan(512, 24576, 9216)
    assert p == {"product": TWO_TILES, "rows": 256, "tokens": 128, "slabs": 32768, "xl": 0, "padded": 0}
    assert plan(2048, 6912, 2560)["product"] == TILE
    found = set()
    for b, f, i, r in LARGE:
        for kept in (0, 8, 16):
            p = plan(b, f, i, r, kept=kept)
            if p["product"] == TWO_TILES:
                assert p["slabs"] % 256 == 0 and 0 < p["slabs"] < 2 * f
                columns, rows = -(-b // 256), p["slabs"] // 256
                assert columns * rows <= 256 * -(-columns * rows // 256) < columns * (rows + 1)      # as many as whole rounds have
                found |= {(p["rows"], kept), ("adapter", r > 0), ("block", f % 32 == 0), ("padded", p["padded"] > 0)}
    assert {(rows, kept) for rows in (64, 128) for kept in (0, 8, 16)} <= found and (256, 0) in found
    assert {(what, yes) for what in ("adapter", "block", "padded") for yes in (False, True)} <= found


def test_tiles_left_over_after_whole_rounds():
    """256 x 256 tiles of a wide grid, more than whole rounds of 256 by up to half a round: 128 x 128 or 256 x 128 ones."""
    quarter = half = 0
    for b, f, i, _ in LARGE:
        p = plan(b, f, i)
        if (p["product"], p["rows"], p["tokens"]) != (TILE, 256, 256):
            continue
        left = (-(-2 * f // 256)) * (-(-b // 256)) % 256
        quarter |= (0 < left <= 64 and i >= 2048) << (i % 256 != 0)
        half |= (64 < left <= 128 and i >= 6144) << (i % 256 != 0)
    assert quarter == 3 and half == 3
