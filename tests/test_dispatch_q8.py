"""Host logic: which kernels slope_spmm_fwd_q8 picks for a shape (slope_spmm_fwd_q8_plan, no GPU needed).  The choices are estimates
of time over the shape alone; pinned here is that the shapes of the GPU tests reach every kernel in every form."""
import pytest

from paper_2405_16325_amd import binding as sl
from tests import test_gpu_spmm_q8 as gpu

STREAM, TILE, GENERAL = range(3)
KSTEP = 128


def form(p):
    return "rows left" if p["rows0"] else "slabs" if p["slabs"] > 1 else "whole"


def test_the_gpu_tests_tiles_are_every_tile_in_every_form():
    reached = set()
    for b, d_out, d_in in gpu.TILES:
        p = sl.slope_spmm_fwd_q8_plan(b, d_in, d_out)
        assert p["product"] == TILE and p["padded"] == 0, (b, d_out, d_in)
        reached.add((p["rows"], p["tokens"], form(p), d_in % KSTEP != 0))
    want = {(rows, tokens, f, tail) for rows, tokens in ((128, 32), (128, 64), (128, 128), (256, 256)) for f in ("whole", "slabs")
            for tail in (False, True)}
    want |= {(128, tokens, "rows left", tail) for tokens in (64, 128) for tail in (False, True)}
    assert reached == want


def test_the_gpu_tests_ordinary_shapes_reach_all_kinds():
    plans = [sl.slope_spmm_fwd_q8_plan(b, d_in, d_out) for b, d_out, d_in in gpu.SHAPES]
    assert {p["product"] for p in plans} == {STREAM, TILE, GENERAL}
    assert {p["tokens"] for p in plans if p["product"] == STREAM} == {4, 8}
    assert any(p["padded"] for p in plans)


def test_the_gpu_tests_few_tokens_are_in_slabs():
    plans = [(sl.slope_spmm_fwd_q8_plan(b, d_in, d_out), d_in) for b, d_out, d_in in gpu.STREAM_SLABS]
    assert all(p["product"] == STREAM and p["slabs"] > 1 for p, _ in plans)
    assert {(p["tokens"], d_in % 256 != 0) for p, d_in in plans} == {(t, tail) for t in (4, 8) for tail in (False, True)}
    assert min(p["slabs"] for p, _ in plans) == 2 and max(p["slabs"] for p, _ in plans) >= 8
    assert any(-(-d_in // 256) % p["slabs"] for p, d_in in plans)                      # a short last slab


def test_the_gpu_tests_padded_copies_feed_every_kernel():
    plans = [sl.slope_spmm_fwd_q8_plan(b, d_in, d_out) for b, d_out, d_in in gpu.PADDED]
    assert all(p["padded"] for p in plans)
    assert {(p["rows"], p["tokens"]) for p in plans} == {(32, 4), (32, 8), (128, 32), (128, 64), (128, 128), (256, 256)}
    assert {form(p) for p in plans} == {"whole", "slabs", "rows left"}


@pytest.mark.parametrize("b,d_in,d_out", [(1, 9216, 36864), (4, 5120, 5120), (8, 9216, 9216), (777, 5120, 20480), (128, 4096, 512), (33, 1000, 1000)])
def test_without_a_workspace_nothing_is_split_or_copied(b, d_in, d_out):
    p = sl.slope_spmm_fwd_q8_plan(b, d_in, d_out, False)
    assert p["slabs"] == 1 and p["padded"] == 0
    if sl.slope_workspace_bytes(sl.SLOPE_CALL_SPMM_FWD_Q8, b, d_in, d_out) == 0:
        assert p == sl.slope_spmm_fwd_q8_plan(b, d_in, d_out)


def test_refusals():
    with pytest.raises(sl.SlopeError):
        sl.slope_spmm_fwd_q8_plan(0, 64, 64)
    with pytest.raises(sl.SlopeError):
        sl.slope_spmm_fwd_q8_plan(1, 64, 12)
    assert sl.lib().slope_spmm_fwd_q8_plan(1, 64, 64, 1, None) == sl.SLOPE_ERR_NULL


# A dimension of a grid holds fewer than 2^32 work items, here 2^24 workgroups of 256; a launch beyond that runs a part of them
# without an error.  Rows: the most that stay below it by the streaming kernel and by 128 x 32 tiles, and what lies around them.
@pytest.mark.parametrize("b,d_in,d_out", [(b, d_in, m + 8 * off) for b, d_in, m in ((1, 32, 2 ** 29 - 32), (8, 64, 2 ** 29 - 32), (40, 64, 2 ** 30 - 128),
                                                                              (64, 128, 2 ** 30 - 128), (96, 64, 2 ** 29), (16, 64, 2 ** 30))
                                          for off in (-2 ** 20, -9, -1, 0, 1, 3, 4, 9, 16, 17)])
@pytest.mark.parametrize("with_workspace", [False, True])
def test_no_grid_passes_what_a_launch_holds(b, d_in, d_out, with_workspace):
    p = sl.slope_spmm_fwd_q8_plan(b, d_in, d_out, with_workspace)
    assert p["groups"] < 2 ** 24, p


def test_the_last_shapes_of_the_streaming_kernel():
    assert sl.slope_spmm_fwd_q8_plan(1, 32, 2 ** 29 - 32)["product"] == STREAM
    assert sl.slope_spmm_fwd_q8_plan(1, 32, 2 ** 29 - 24)["product"] != STREAM
