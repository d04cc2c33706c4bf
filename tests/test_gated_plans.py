"""slope_gated_fwd_plan says what slope_gated_fwd launches: where last tokens are left over from whole tiles, the others may run as whole rounds of
256 x 256 tiles and another tile, three launches; tokens beyond what a launch's grid holds run in several."""
import random

import pytest
import torch

from paper_2405_16325_amd import binding as sl
from tests.graph_util import kernels

SMALL_BATCH, SLABS, TILE, GENERAL, ROW_SPLIT, REST, TWO_TILES, TWO_TILES_AND_REST = range(8)
# (b, d_ff, d_in, r)
THREE = [(8223, 1176, 9280, 0), (4636, 2056, 11456, 0), (5388, 1800, 10752, 64), (1542, 9360, 10688, 0)]


def plan(b, d_ff, d_in, r=0, **more):
    return sl.slope_gated_fwd_plan(b, d_in, d_ff, r, **more)


def test_tokens_left_over_behind_two_kinds_of_tiles():
    for b, d_ff, d_in, r in THREE + [(4632, 2112, 15872, 0)]:
        p = plan(b, d_ff, d_in, r)
        assert p["product"] == TWO_TILES_AND_REST and p["slabs"] % 256 == 0 and 0 < p["slabs"] < 2 * d_ff
        assert plan(b, d_ff, d_in, r, kept=8)["product"] not in (REST, TWO_TILES_AND_REST)
    assert plan(4632, 2112, 15872) == {"product": TWO_TILES_AND_REST, "rows": 128, "tokens": 96, "slabs": 3584, "xl": 0, "padded": 0}
    assert {(plan(*s)["rows"], plan(*s)["tokens"]) for s in THREE} == {(192, 64), (128, 96), (256, 192)}


def test_the_tokens_of_whole_tiles_run_as_a_batch_of_their_own():
    rng, seen = random.Random(7), set()
    cases = [(128 * int(2 ** rng.uniform(0, 7)) + rng.randint(1, 32), 8 * int(2 ** rng.uniform(6, 12)), 64 * int(2 ** rng.uniform(1, 9))) for _ in range(40000)]
    for b, d_ff, d_in in cases + [s[:3] for s in THREE]:
        p = plan(b, d_ff, d_in)
        if p["product"] not in (REST, TWO_TILES_AND_REST):
            continue
        seen.add(p["product"])
        rest = b % 128
        assert p["product"] == TWO_TILES_AND_REST or p["slabs"] == rest
        whole = plan(b - rest, d_ff, d_in, with_workspace=False)            # (a batch by itself might be split over the contraction)
        assert whole["product"] == (TILE if p["product"] == REST else TWO_TILES), (b, d_ff, d_in)
        assert (whole["rows"], whole["tokens"]) == (p["rows"], p["tokens"]), (b, d_ff, d_in)
        assert p["product"] == REST or whole["slabs"] == p["slabs"], (b, d_ff, d_in)
    assert seen == {REST, TWO_TILES_AND_REST}


def test_more_tokens_than_a_launch_holds():
    d_ff = 1 << 20                                                          # 4096 tokens a launch
    for b in (4096, 8192, 4352, 1 << 20):
        assert plan(b, d_ff, 64) == plan(4096, d_ff, 64)


def launches(ran):
    """[(rows, tokens)] of the product's kernels, [None] for a small-batch kernel"""
    found = []
    for name, n in ran:
        if name in ("spmm_kernel", "spmm_ring_kernel"):
            found.append(n[:2])
        elif name == "spmm_split_kernel":
            found.append((256, 256))
        elif name == "spmm_generic_kernel":
            found.append((32 * n[1], 32 * n[1]))
        elif name in ("spmm_stream_lds_kernel", "spmm_rows_kernel"):
            found.append(None)
    return found


@pytest.mark.gpu
@pytest.mark.parametrize("b,d_ff,d_in,r", THREE + [(512, 24576, 9216, 0), (1561, 1280, 3712, 0), (523, 6592, 128, 0), (1000, 1000, 1000, 0), (300, 1000, 1000, 0)])
def test_the_kernels_that_run_are_those_of_the_plan(b, d_ff, d_in, r):
    from tests.test_gpu_gated import Layer, check_h
    print(f"gated_fwd launches b={b} d_ff={d_ff} d_in={d_in} r={r}", flush=True)
    layer, p = Layer(b, d_ff, d_in, r, seed=b), plan(b, d_ff, d_in, r)
    h = torch.empty(b, d_ff, dtype=sl.BF16, device="cuda")
    ws = torch.empty(max(256, sl.slope_workspace_bytes(sl.SLOPE_CALL_GATED_FWD, b, d_in, d_ff, r)), dtype=torch.uint8, device="cuda")
    ran = launches(kernels(lambda: sl.slope_gated_fwd(layer.x, layer.vals, layer.meta, L=layer.l, R=layer.r, out=(h, None, None, None), workspace=ws)))
    want = [(p["rows"], p["tokens"])]
    if p["product"] in (TWO_TILES, TWO_TILES_AND_REST):
        want = [(256, 256)] + want
    if p["product"] in (REST, TWO_TILES_AND_REST):
        want += [None]
    assert ran == want, p
    h.zero_()
    sl.slope_gated_fwd(layer.x, layer.vals, layer.meta, L=layer.l, R=layer.r, out=(h, None, None, None), workspace=ws)
    check_h(h, layer.gu, layer.off, "silu", "h")
