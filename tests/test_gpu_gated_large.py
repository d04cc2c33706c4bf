"""The gated product where shapes alone do not reach a path: batches of more tokens than the last-level cache holds, whose 256 x 256 tiles fetch ahead;
codes that pass the caches, rows of them that start 8 bytes off and end in half a piece; tokens that run in several launches; every tile in every
form of the call, alone and behind whole rounds of the largest (which shapes reach what: test_the_shapes_do_reach_it and those behind it, on the host)."""
import random

import pytest
import torch

from paper_2405_16325_amd import binding as sl
from tests import test_gpu_gated as tg
from tests.test_gated_plans import REST, THREE, TILE, TWO_TILES, plan

CACHE = 256 << 20
# (b, d_ff, d_in): contractions of whole quads of k-steps and not; 33 and 18 rows of 64 tiles, of which a quarter and half a round are left over
AHEAD = [(16384, 4104, 9216), (16384, 2184, 9216), (16384, 2184, 9280)]
# (b, d_ff, d_in, r, what is kept): beside the shapes of test_gpu_gated
MORE = [(1541, 1864, 128, 0, 0), (1802, 1720, 128, 32, 0), (1599, 1960, 128, 0, 16), (1697, 1824, 128, 160, 16), (2321, 1896, 128, 0, 0), (1972, 2264, 128, 32, 0),
        (8198, 200, 5888, 32, 0), (7776, 1176, 1152, 0, 0), (1926, 4712, 1280, 160, 0), (1774, 5296, 1024, 0, 8), (3078, 2848, 1408, 160, 8),
        (3540, 2688, 1408, 0, 16), (2520, 3624, 1216, 32, 16), (2897, 3392, 2048, 0, 0), (2177, 4384, 1728, 64, 0), (5294, 1808, 1920, 0, 8),
        (2497, 3936, 1920, 160, 8), (3474, 2792, 1792, 0, 16), (4993, 1848, 1728, 64, 16), (11129, 2256, 768, 0, 0), (2035, 4856, 1216, 64, 0),
        (3221, 2912, 1728, 0, 16), (5301, 1800, 1536, 160, 16), (1574, 5912, 3776, 0, 0), (3797, 2720, 3776, 160, 0), (4703, 2088, 3776, 160, 16),
        (5421, 3392, 1280, 0, 0), (2988, 6192, 1536, 64, 0), (4144, 4512, 1216, 0, 16), (4195, 4424, 1280, 32, 16), (7842, 1584, 2176, 0, 0),
        (2696, 4440, 2432, 32, 0), (2615, 4632, 2176, 0, 16), (3478, 3464, 2432, 64, 16), (3451, 5696, 2048, 0, 0), (1762, 6824, 1536, 0, 8),
        (4243, 4576, 2048, 0, 16), (2409, 5440, 6400, 0, 0), (1031, 11504, 4608, 64, 0), (4113, 3016, 6144, 0, 8), (1630, 7176, 4864, 32, 8),
        (1149, 11184, 4608, 0, 16), (4983, 2464, 5376, 32, 16), (2169, 2080, 128, 64, 16), (2005, 9256, 1216, 0, 16)]


# ------------------------------------------------------------------------------------------------------------------ on the host
def test_the_shapes_do_reach_it():
    for b, d_ff, d_in in AHEAD:
        assert 2 * b * d_in > CACHE and 8 * b * d_ff > CACHE and d_ff % 16 == 8
        for kept in (0, 8, 16):
            p = plan(b, d_ff, d_in, kept=kept)
            assert (p["product"], p["rows"], p["tokens"]) == (TILE, 256, 256)
    left = {(-(-(-(-d_ff // 16) * 32) // 256) * -(-b // 256) % 256, d_in % 256 != 0) for b, d_ff, d_in in AHEAD}
    assert left == {(64, False), (128, False), (128, True)}
    b, d_ff, d_in = CUT
    most = (1 << 21) // ((-(-d_ff // 16) * 32 + 63) // 64) * 64 // 256 * 256
    assert most < b < 2 * most


def form(b, d_ff, d_in, r, kept, **more):
    p = plan(b, d_ff, d_in, r, kept=kept, **more)
    return p["product"], p["rows"], p["tokens"], kept, r > 0


def test_every_tile_in_every_form_that_a_call_reaches():
    shapes = [(b, f, i, r) for b, f, i in tg.SHAPES for r in (0, 32, 160)] + tg.LARGE + tg.BESIDE
    reached = {form(*s, kept) for s in shapes for kept in (0, 8, 16)} | {form(*s[:3], 0, 0, with_workspace=False) for s in shapes}
    reached |= {form(*s, 0) for s in THREE} | {form(*s) for s in MORE}
    rng = random.Random(5)
    for _ in range(100000):
        b, d_ff, d_in = int(2 ** rng.uniform(0, 13.5)), 8 * int(2 ** rng.uniform(0, 11.5)), rng.choice([8, 64, 64, 256]) * int(2 ** rng.uniform(0, 6))
        if b * d_ff * d_in > 2e11:
            continue
        case = b, d_ff, d_in, rng.choice([0, 32, 64, 160]), rng.choice([0, 8, 16])
        assert form(*case) in reached, (case, form(*case))
    for rows, tokens in ((128, 64), (128, 96), (128, 128), (256, 128), (256, 192), (256, 256)):
        for adapter in (False, True):
            assert {(TILE, rows, tokens, kept, adapter) for kept in (0, 8, 16)} <= reached
    for rows, tokens in ((192, 64), (192, 96), (192, 128), (192, 192)):
        for adapter in (False, True):
            assert (TWO_TILES, rows, tokens, 0, adapter) in reached
    assert any(f[0] == REST and f[4] for f in reached) and any(f[0] == REST and not f[4] for f in reached)


# ---------------------------------------------------------------------------------------------------------------- on the device
class Rows:
    """Operands of a large batch, and the projections of some of its tokens in 64 bits."""

    def __init__(self, b, d_ff, d_in):
        gen = torch.Generator(device="cuda").manual_seed(b + d_ff)
        gauss = lambda shape, std: torch.randn(shape, generator=gen, device="cuda").mul_(std).to(sl.BF16)       # noqa: E731
        self.x = gauss((b, d_in), 1.0)
        self.vals, self.meta, _ = sl.slope_prune_rows(gauss((2 * d_ff, d_in), d_in ** -0.5))
        self.at, self.d_ff = tg.far_rows(b), d_ff
        x, w = tg.double(self.x[self.at]), tg.dense_of(self.vals, self.meta).t().contiguous()
        self.gu = x @ w
        self.off = (d_in / 2 + 8) * 2.0 ** -24 * (x.abs() @ w.abs_())

    def check(self, h, gu, q, scale):
        at, d_ff = self.at, self.d_ff
        tg.check_h(h[at], self.gu, self.off, "silu", "h")
        if gu is not None:
            tg.check_kept(gu[at], self.gu, self.off, "gu")
        if q is not None:
            tg.check_blocks(tg.codes(q)[at].view(-1, d_ff), scale[at].view(2 * len(at), -1), self.gu.view(-1, d_ff), self.off.view(-1, d_ff), "codes")


@pytest.mark.gpu
@pytest.mark.parametrize("b,d_ff,d_in", AHEAD)
def test_batches_that_the_last_level_cache_does_not_hold(b, d_ff, d_in):
    print(f"gated_fwd large b={b} d_ff={d_ff} d_in={d_in}", flush=True)
    p = Rows(b, d_ff, d_in)
    plain = sl.slope_gated_fwd(p.x, p.vals, p.meta)
    both = sl.slope_gated_fwd(p.x, p.vals, p.meta, want_gu=True, want_q8=True)
    codes = sl.slope_gated_fwd(p.x, p.vals, p.meta, want_q8=True)
    wide = sl.slope_gated_fwd(p.x, p.vals, p.meta, want_gu=True)
    for out in (plain, both, codes, wide):
        p.check(*out)
    assert torch.equal(tg.codes(both[2]), tg.codes(codes[2])) and torch.equal(both[3], codes[3])
    for other in (both, codes, wide):                                       # every token: the same sums in the same order
        assert torch.equal(plain[0], other[0])
    assert torch.equal(both[1], wide[1])


CUT = (4100, (1 << 20) + 8, 128)


@pytest.mark.gpu
def test_tokens_of_more_than_one_launch():
    """4.3e9 elements of h, twice as many projections."""
    print("gated_fwd in several launches", flush=True)
    b, d_ff, d_in = CUT
    p = Rows(b, d_ff, d_in)
    p.at = torch.cat([p.at[:2], torch.arange(3838, 3842, device="cuda"), p.at[-2:]])          # both sides of the cut, 3840
    x, w = tg.double(p.x[p.at]), tg.dense_of(p.vals, p.meta).t().contiguous()
    p.gu, p.off = x @ w, (d_in / 2 + 8) * 2.0 ** -24 * (x.abs() @ w.abs_())
    del x, w
    p.check(*sl.slope_gated_fwd(p.x, p.vals, p.meta))
    p.check(*sl.slope_gated_fwd(p.x, p.vals, p.meta, want_gu=True, want_q8=True))


@pytest.mark.gpu
@pytest.mark.parametrize("b,d_ff,d_in,r,kept", MORE)
def test_every_tile_in_every_form(b, d_ff, d_in, r, kept):
    print(f"gated_fwd forms b={b} d_ff={d_ff} d_in={d_in} r={r} kept={kept}", flush=True)
    p = tg.Layer(b, d_ff, d_in, r, seed=b + d_ff + d_in)
    h, gu, q, scale = sl.slope_gated_fwd(p.x, p.vals, p.meta, L=p.l, R=p.r, want_gu=kept == 16, want_q8=kept == 8)
    tg.check_h(h, p.gu, p.off, "silu", "h")
    if kept == 16:
        tg.check_kept(gu, p.gu, p.off, "gu")
    if kept == 8:
        tg.check_blocks(q.view(2 * b, d_ff), scale.view(2 * b, -1), p.gu.view(2 * b, d_ff), p.off.view(2 * b, d_ff), "codes")
