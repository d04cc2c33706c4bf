"""The gated feed-forward layer and activations kept in 8 bits: HIP path vs the oracle in 64 bits.

Bounds of an element, u = 2^-8 being half a step of bf16:
  - a projection before it is rounded: fp32 sums of K / 2 products (r more with an adapter) are off by at most (K / 2 + r + 8) 2^-24 of the
    terms' magnitudes, S; with an adapter X L is rounded to bf16 on the way, u of |X L| |R|.  E is the sum of both.
  - g and u as they are kept: u of the value, and E; in 8 bits 2^-4 of the value or 2^-10 of the scale, and 1.1 E (the rounding of a
    value that is E off may go the other way, by no more than that).
  - h = act(g) u: |act'| <= 1.13, so 1.13 E_g |u| + |act(g)| E_u + E_g E_u; the exponential's argument and result, the reciprocal and two
    products are off by (|g| + 8) 2^-22 of the value together (gelu: its argument is 1.6 (g + 0.045 g^3)); one rounding, u.
  - the gradient, from given g and u: the same for du = dh act(g); dg = dh u act'(g), where the terms of act' = s + g s (1 - s) ... may
    cancel: the relative part is taken of |dh u| (1 + |g|).
  - the logistic function is 1 / (1 + e^-x), and the reciprocal instruction gives zero for results below fp32's normal numbers: s is off by
    up to 2^-126, so a by 2^-126 |g| and act' by 2^-126 (1 + 1.6 |g| (1 + 0.135 g^2)).
"""
import numpy as np
import pytest
import torch

from oracle import slope_oracle as so
from oracle import surroundings_oracle as oo
from paper_2405_16325_amd import binding as sl
from paper_2405_16325_amd import inputs
from tests.graph_util import kernels
from tests.parity_util import check_product

pytestmark = pytest.mark.gpu
ACTS = {"silu": sl.SLOPE_ACT_SILU, "gelu": sl.SLOPE_ACT_GELU, "relu": sl.SLOPE_ACT_RELU}
HALF, FLUSH = 2.0 ** -8, 2.0 ** -126


def say(msg):
    print(msg, flush=True)


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def codes_of(t):
    return t.view(torch.uint8).cpu().numpy()


def double(t):
    return t.detach().float().double()


def dense_of(vals, meta):
    """Packed 2:4 -> fp64[rows, cols], on the device."""
    rows, half = vals.shape
    m = meta.to(torch.int64)
    at = torch.stack([m & 3, m >> 2 & 3, (m >> 4 & 3) + 4, (m >> 6) + 4], dim=-1) + 8 * torch.arange(m.shape[1], device="cuda")[:, None]
    return torch.zeros(rows, 2 * half, dtype=torch.float64, device="cuda").scatter_(1, at.view(rows, half), double(vals))


class Layer:
    """Operands of a gated layer and its projections in 64 bits, with what fp32 sums may be off (on the device: some are large)."""

    def __init__(self, b, d_ff, d_in, r=0, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def gauss(shape, std):
            return torch.randn(shape, generator=gen, device="cuda").mul_(std).to(sl.BF16)

        self.b, self.d_ff, self.d_in = b, d_ff, d_in
        self.x = gauss((b, d_in), 1.0)
        self.vals, self.meta, _ = sl.slope_prune_rows(gauss((2 * d_ff, d_in), d_in ** -0.5))
        x, w = double(self.x), dense_of(self.vals, self.meta).t().contiguous()
        self.gu = x @ w
        self.off = (d_in / 2 + r + 8) * 2.0 ** -24 * (x.abs() @ w.abs_())
        self.l = self.r = None
        if r:
            self.l, self.r = gauss((d_in, r), 0.05), gauss((r, 2 * d_ff), 0.2)
            ld, rd = double(self.l), double(self.r)
            t = x @ ld
            self.gu = self.gu + t @ rd
            t_off = HALF * t.abs() + (d_in + 8) * 2.0 ** -24 * (x.abs() @ ld.abs())
            self.off += t_off @ rd.abs() + (d_in / 2 + r + 8) * 2.0 ** -24 * (t.abs() @ rd.abs())


def activation(g, act):
    """(act(g), act'(g)) in 64 bits, as the oracle has them (test_the_reference_on_the_device)."""
    if act == "relu":
        return g.clamp(min=0), (g > 0).double()
    if act == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s + g * s * (1 - s)
    c = 2 * (2 / np.pi) ** 0.5
    s = 1 / (1 + torch.exp(-c * (g + 0.044715 * g ** 3)))
    return g * s, s + g * s * (1 - s) * c * (1 + 3 * 0.044715 * g ** 2)


def restored(codes, bytes_):
    """Values of 8-bit blocks, fp64."""
    value = torch.from_numpy(oo.e4m3_value(np.arange(256))).cuda()[codes.view(torch.uint8).long()]
    return value * scale_of(bytes_, codes.shape[1])


def scale_of(bytes_, d):
    power = torch.from_numpy(np.append(2.0 ** (np.arange(255) - 127.0), np.nan)).cuda()[bytes_.long()]
    return power.repeat_interleave(32, dim=1)[:, :d]


def relative(g, act):
    z = g.abs() if act == "silu" else 1.6 * (g.abs() + 0.045 * g.abs() ** 3)
    return (z + 8) * 2.0 ** -22


def within(got, want, bound, what):
    bad = ~((double(got) - want).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist())


def check_h(got, gu, off, act, what):
    d_ff = got.shape[1]
    g, u, eg, eu = gu[:, :d_ff], gu[:, d_ff:], off[:, :d_ff], off[:, d_ff:]
    a = activation(g, act)[0]
    want = a * u
    bound = 1.13 * eg * (u.abs() + eu) + a.abs() * eu + (HALF + relative(g, act)) * want.abs() + FLUSH * (g * u).abs() + 1e-38
    within(got, want, bound * 1.01, what)


def check_kept(got, want, off, what):
    within(got, want, HALF * (want.abs() + off) + off + 1e-38, what)


def check_blocks(codes, bytes_, want, off, what):
    """codes e4m3[rows, d], bytes u8[rows, blocks] of values want, which may be `off` off."""
    d = codes.shape[1]
    within(restored(codes, bytes_), want, torch.maximum(2.0 ** -4 * (want.abs() + off), 2.0 ** -10 * scale_of(bytes_, d)) + 1.1 * off, what)
    pad = (0, bytes_.shape[1] * 32 - d)                                     # the smallest scale that holds the block
    least = torch.nn.functional.pad((want.abs() - off).clamp(min=0), pad).view(len(codes), -1, 32).amax(2)
    most = torch.nn.functional.pad(want.abs() + off, pad).view(len(codes), -1, 32).amax(2)
    s = torch.pow(2.0, bytes_.double() - 127)
    assert (least <= 448 * s * 1.0001).all() and ((most * 1.0001 > 224 * s) | (bytes_ == 1)).all(), what


def test_the_reference_on_the_device():
    p = Layer(5, 40, 64, 32, seed=1)
    x, w = f64(p.x), so.bf16_to_f64(so.unpack_2to4(sl.bf16_to_host(p.vals), p.meta.cpu().numpy()))
    assert np.allclose(p.gu.cpu().numpy(), x @ w.T + x @ f64(p.l) @ f64(p.r), rtol=0, atol=1e-12)
    for act in ACTS:
        for mine, theirs in zip(activation(p.gu, act), oo.activation(p.gu.cpu().numpy(), act)):
            assert np.allclose(mine.cpu().numpy(), theirs, rtol=1e-12, atol=1e-14)
    q, s = sl.slope_checkpoint_q8(p.x)
    assert (restored(q, s).cpu().numpy() == oo.restored(codes_of(q), s.cpu().numpy())).all()


# one token to many; d_ff a multiple of 256, of 64, of 16, of 8 only, less than a block; contractions of whole quads, pairs, odd steps, parts
SHAPES = [(1, 8, 8), (1, 256, 128), (1, 64, 1024), (2, 1000, 768), (7, 40, 264), (16, 512, 2048), (17, 136, 704), (31, 2048, 256), (32, 72, 64), (33, 128, 384),
          (40, 520, 1024), (64, 256, 2304), (100, 1000, 1000), (128, 200, 4096), (129, 1024, 1088), (200, 344, 192), (257, 24, 320),
          (300, 768, 640), (512, 136, 8), (520, 256, 520), (700, 1032, 448), (1000, 1000, 1000), (1030, 2048, 128), (2100, 320, 256)]
# what the small ones do not reach: the other numbers of rows of the small-batch kernel, its row-split form with and without slices, every
# tile and every split, an odd k-step at the end of each, tokens and tiles that are left over (test_dispatch_gated.py)
LARGE = [(1568, 5056, 768, 32), (785, 9984, 832, 0), (35, 2600, 10048, 0), (65, 1688, 15360, 32), (130, 1040, 12096, 0), (98, 8504, 192, 0), (131, 8368, 192, 32), (197, 8200, 256, 64), (199, 8224, 128, 0),
         (385, 11080, 256, 0), (386, 10936, 128, 32), (1, 8, 192, 0), (1, 8, 192, 32), (1, 3912, 192, 32), (1, 6872, 128, 32), (1, 7104, 704, 32), (1, 6656, 320, 0), (17, 8, 128, 32), (19, 8, 192, 32),
         (1, 4056, 128, 0), (1, 4128, 192, 0), (1, 6848, 128, 0), (5, 6656, 320, 32), (17, 4304, 128, 0), (20, 5120, 192, 32), (1, 12288, 1024, 0),
         (3, 2056, 17408, 0), (2, 24576, 1024, 0), (13, 20488, 1024, 32), (300, 2056, 2056, 0), (1000, 520, 2200, 32), (2048, 264, 520, 0), (200, 8, 4104, 0), (400, 520, 8200, 32), (1999, 1000, 1096, 64), (16, 2048, 16384, 64), (20, 2048, 16384, 0), (31, 4104, 16384, 32), (9, 12296, 2048, 96),
         (1, 4272, 128, 32), (17, 4544, 128, 32), (35, 8, 2816, 32), (40, 8, 2624, 0), (4344, 8, 6144, 0), (3546, 8, 8000, 32),
         (34, 4584, 7424, 0), (33, 4208, 7616, 32), (131, 2880, 5120, 32), (133, 2752, 4672, 0), (5526, 136, 128, 32), (145, 5480, 192, 0),
         (195, 5568, 128, 32), (198, 6248, 192, 0), (259, 5504, 256, 160), (258, 5576, 128, 0), (654, 5384, 256, 32), (522, 6592, 128, 0),
         (783, 6696, 256, 0), (770, 6720, 128, 64), (131, 5448, 64, 32), (142, 5504, 8, 0), (1560, 1280, 3584, 32), (1561, 1280, 3712, 0),
         (1026, 7232, 768, 0), (2054, 3904, 576, 64), (1024, 8320, 2048, 32), (1000, 8312, 2112, 0), (1024, 10752, 6144, 0), (1020, 10752, 6208, 32),
         (962, 8200, 640, 32), (423, 16520, 664, 0), (435, 17696, 768, 32), (11211, 680, 768, 0), (608, 16568, 1264, 32), (8235, 968, 2048, 32), (8287, 976, 2112, 0)]


# X L beside the product and the adapter added with the sums (test_dispatch_gated.py)
BESIDE = [(1, 8, 1088, 96), (9, 40, 1152, 96), (16, 520, 2048, 32), (17, 6992, 1152, 64), (18, 6792, 1152, 96), (1, 4600, 1216, 64), (3, 4944, 1280, 128),
          (18, 5680, 1408, 32), (17, 4664, 1856, 32), (2, 15936, 1728, 32), (3, 6424, 2176, 128), (33, 16, 1920, 64), (37, 8, 1856, 128), (100, 200, 4096, 160), (321, 16, 12224, 160),
          (400, 8, 9088, 160), (436, 72, 7936, 192), (33, 2592, 10304, 96), (37, 1720, 15680, 192), (485, 112, 15168, 192), (137, 808, 15232, 192)]


@pytest.mark.parametrize("b,d_ff,d_in,r", BESIDE)
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_forward_with_the_adapter_beside(b, d_ff, d_in, r, act):
    check_forward(b, d_ff, d_in, act, r)


@pytest.mark.parametrize("b,d_ff,d_in", SHAPES)
@pytest.mark.parametrize("act,r", [("silu", 0), ("gelu", 32), ("relu", 160)])
def test_forward(b, d_ff, d_in, act, r):
    check_forward(b, d_ff, d_in, act, r)


@pytest.mark.parametrize("b,d_ff,d_in,r", LARGE)
def test_forward_of_every_kernel(b, d_ff, d_in, r):
    check_forward(b, d_ff, d_in, "silu", r)


def check_forward(b, d_ff, d_in, act, r):
    say(f"gated_fwd b={b} d_ff={d_ff} d_in={d_in} act={act} r={r}")
    p = Layer(b, d_ff, d_in, r, seed=b + d_ff + d_in)
    args = dict(act=ACTS[act], L=p.l, R=p.r)
    h, none_gu, none_q, none_s = sl.slope_gated_fwd(p.x, p.vals, p.meta, **args)
    assert none_gu is None and none_q is None and none_s is None
    again = sl.slope_gated_fwd(p.x, p.vals, p.meta, **args)[0]
    kept, gu, q, scale = sl.slope_gated_fwd(p.x, p.vals, p.meta, want_gu=True, want_q8=True, **args)
    wide, gu_only, _, _ = sl.slope_gated_fwd(p.x, p.vals, p.meta, want_gu=True, **args)
    torch.cuda.synchronize()
    check_h(wide, p.gu, p.off, act, "h of the call that keeps bf16")
    check_kept(gu_only, p.gu, p.off, "gu without codes")
    check_h(h, p.gu, p.off, act, "h")
    check_h(kept, p.gu, p.off, act, "h of the call that keeps")
    assert torch.equal(h, again)
    check_kept(gu, p.gu, p.off, "gu")
    check_blocks(q.view(2 * b, d_ff), scale.view(2 * b, -1), p.gu.view(2 * b, d_ff), p.off.view(2 * b, d_ff), "codes")
    if r == 0:
        alone = sl.slope_gated_fwd(p.x, p.vals, p.meta, act=ACTS[act], workspace=None)[0]
        check_h(alone, p.gu, p.off, act, "h without scratch")
        if b <= 32:                                                         # kept by the tile kernels then
            _, gu, q, scale = sl.slope_gated_fwd(p.x, p.vals, p.meta, act=ACTS[act], want_gu=True, want_q8=True, workspace=None)
            check_kept(gu, p.gu, p.off, "gu without scratch")
            check_blocks(q.view(2 * b, d_ff), scale.view(2 * b, -1), p.gu.view(2 * b, d_ff), p.off.view(2 * b, d_ff), "codes without scratch")


@pytest.mark.parametrize("b,d_ff,d_in,r", [(1, 1000, 768, 32), (20, 264, 448, 0), (70, 72, 1024, 64), (300, 328, 640, 0), (515, 1000, 256, 96), (260, 264, 264, 32)])
def test_nothing_outside_is_written_and_parts_agree(b, d_ff, d_in, r):
    say(f"gated_fwd guards b={b} d_ff={d_ff} d_in={d_in} r={r}")
    p = Layer(b, d_ff, d_in, r, seed=3)
    pad = 4096
    blocks = (d_ff + 31) // 32
    sizes = {"h": (b * d_ff, sl.BF16), "gu": (2 * b * d_ff, sl.BF16), "q": (2 * b * d_ff, torch.uint8), "s": (2 * b * blocks, torch.uint8)}
    whole = {k: torch.full((n + 2 * pad,), 7, dtype=t, device="cuda") for k, (n, t) in sizes.items()}
    cut = {k: whole[k][pad:pad + n] for k, (n, _) in sizes.items()}
    out = (cut["h"].view(b, d_ff), cut["gu"].view(b, 2 * d_ff), cut["q"].view(sl.E4M3).view(b, 2 * d_ff), cut["s"].view(b, 2, blocks))
    sl.slope_gated_fwd(p.x, p.vals, p.meta, L=p.l, R=p.r, out=out)
    only = sl.slope_gated_fwd(p.x, p.vals, p.meta, L=p.l, R=p.r, want_gu=True)
    codes = sl.slope_gated_fwd(p.x, p.vals, p.meta, L=p.l, R=p.r, want_q8=True)
    torch.cuda.synchronize()
    for k, (n, _) in sizes.items():
        assert (whole[k][:pad] == 7).all() and (whole[k][pad + n:] == 7).all(), k
    assert torch.equal(codes[0], out[0]) and torch.equal(codes[3], out[3])
    check_h(only[0], p.gu, p.off, "silu", "h")
    check_kept(only[1], p.gu, p.off, "gu")
    assert torch.equal(codes[2].view(torch.uint8), out[2].view(torch.uint8))


@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("b,d_ff", [(1, 8), (3, 40), (5, 256), (333, 1000), (64, 2048), (1025, 72)])
def test_gradient(b, d_ff, act, q8):
    say(f"gated_bwd b={b} d_ff={d_ff} act={act} q8={q8}")
    gu = sl.bf16_to_device(inputs.gaussian_bf16((b, 2 * d_ff), 3.0, b + d_ff, 1))
    dh = sl.bf16_to_device(inputs.gaussian_bf16((b, d_ff), 1e-3, b + d_ff, 2))
    if q8:
        q, scale = sl.slope_checkpoint_q8(gu.view(2 * b, d_ff))
        v = restored(q, scale).view(b, 2 * d_ff)
        dgu, h = sl.slope_gated_bwd(dh, ACTS[act], q8=q.view(b, 2 * d_ff), scale=scale.view(b, 2, -1))
    else:
        v = double(gu)
        dgu, h = sl.slope_gated_bwd(dh, ACTS[act], gu=gu)
    torch.cuda.synchronize()
    check_gradient(dgu, h, double(dh), v, act)


def check_gradient(dgu, h, dh, v, act):
    d_ff = h.shape[1]
    g, u = v[:, :d_ff], v[:, d_ff:]
    check_h(h, v, torch.zeros_like(v), act, "h")
    a, d = activation(g, act)
    want = torch.cat([dh * u * d, dh * a], 1)
    rel, flushed = relative(g, act), FLUSH * dh.abs()
    bound = HALF * want.abs() + 1e-38 + torch.cat([rel * (dh * u).abs() * (1 + g.abs()) + flushed * u.abs() * (1 + 1.6 * g.abs() * (1 + 0.135 * g * g)),
                                                   rel * (dh * a).abs() + flushed * g.abs()], 1)
    within(dgu, want, bound * 1.01, "dgu")


@pytest.mark.parametrize("act", list(ACTS))
def test_gradient_far_from_zero_and_in_place(act):
    """Gates from -300 to 300 and beyond, where exponentials leave fp32's range; dGU over GU, H over dH; without H."""
    say(f"gated_bwd far {act}")
    b, d_ff = 9, 64
    g = np.linspace(-300, 300, b * d_ff).reshape(b, d_ff)
    g[0, :8] = [0.0, -0.0, 1e30, -1e30, 3e38, -3e38, 1e-38, -1e-38]
    gu = torch.from_numpy(np.concatenate([g, np.ones_like(g)], 1)).to(sl.BF16).cuda()
    dh = torch.full((b, d_ff), 0.5, dtype=sl.BF16, device="cuda")
    v = f64(gu)
    plain = sl.slope_gated_bwd(dh, ACTS[act], gu=gu)
    alone, none = sl.slope_gated_bwd(dh, ACTS[act], gu=gu, want_h=False)
    assert none is None and torch.equal(alone, plain[0])
    d = f64(dh)
    sl.slope_gated_bwd(dh, ACTS[act], gu=gu, out=(gu, dh))
    torch.cuda.synchronize()
    assert torch.equal(gu, plain[0]) and torch.equal(dh, plain[1])
    with np.errstate(over="ignore", invalid="ignore"):
        want_h = np.where(v[:, :d_ff] < -80, 0.0, oo.gated(np.clip(v, -80, None), act))
        d_act = np.where(v[:, :d_ff] < -80, 0.0, np.where(v[:, :d_ff] > 80, 1.0, oo.activation(np.clip(v[:, :d_ff], -80, 80), act)[1]))
    want_h[0, [2, 4]] = v[0, [2, 4]]                                       # (the cube leaves the range of 64 bits)
    got_h, got = f64(plain[1]), f64(plain[0])
    assert (np.abs(got_h - want_h) <= 1.1 * HALF * np.abs(want_h) + 1e-25).all()
    assert (np.abs(got[:, :d_ff] - d * d_act) <= 1.1 * HALF * d * np.abs(d_act) + 2e-6).all()
    assert (np.abs(got[:, d_ff:] - d * want_h) <= 1.1 * HALF * np.abs(d * want_h) + 1e-25).all()


@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("act", list(ACTS))
def test_nan_and_infinity_reach_the_results(act, q8):
    b, d_ff = 4, 96
    g = torch.ones(b, 2 * d_ff)
    g[0, 3], g[1, 40], g[2, d_ff + 70] = float("nan"), float("inf"), float("nan")
    gu = g.to(sl.BF16).cuda()
    dh = torch.ones(b, d_ff, dtype=sl.BF16, device="cuda")
    kw = dict(gu=gu)
    if q8:
        q, s = sl.slope_checkpoint_q8(gu.view(2 * b, d_ff))
        kw = dict(q8=q.view(b, 2 * d_ff), scale=s.view(b, 2, -1))
    dgu, h = sl.slope_gated_bwd(dh, ACTS[act], **kw)
    touched = torch.zeros(b, d_ff, dtype=torch.bool)
    for row, col in ((0, 3), (1, 40), (2, 70)):
        if q8:
            touched[row, col // 32 * 32:col // 32 * 32 + 32] = True        # the block
        else:
            touched[row, col] = True
    assert (torch.isfinite(h.cpu()) == ~touched).all()
    assert torch.isfinite(dgu.cpu().view(b, 2, d_ff)[~touched[:, None].expand(b, 2, d_ff)]).all()


def test_forward_of_tokens_that_are_not_finite():
    """A token with a NaN spoils its own row and no other; its blocks read NaN."""
    p = Layer(40, 136, 256, 0, seed=5)
    x = p.x.clone()
    x[7, 100], x[23, 0] = float("nan"), float("inf")
    h, gu, q, scale = sl.slope_gated_fwd(x, p.vals, p.meta, want_gu=True, want_q8=True)
    clean = sl.slope_gated_fwd(p.x, p.vals, p.meta, want_gu=True, want_q8=True)
    rows = [i for i in range(40) if i not in (7, 23)]
    assert torch.equal(h[rows], clean[0][rows]) and torch.equal(gu[rows], clean[1][rows]) and torch.equal(scale[rows], clean[3][rows])
    back = sl.slope_restore_q8(q.view(80, 136), scale.view(80, -1)).view(40, 272)
    assert not torch.isfinite(h[7]).all()
    lost = ~torch.isfinite(gu).view(40, 2, 136)
    for i in (7, 23):
        assert lost[i].any()
        for half in range(2):
            for c in range(5):
                block = slice(c * 32, min(136, (c + 1) * 32))
                assert torch.isnan(back.view(40, 2, 136)[i, half, block]).all() == bool(lost[i, half, block].any())


# ------------------------------------------------------------------------------------------------ 8-bit blocks of an activation
@pytest.mark.parametrize("rows,d", [(1, 8), (1, 32), (3, 40), (5, 256), (64, 1000), (333, 2048), (1, 36864), (1025, 72), (2, 8200)])
def test_checkpoint_is_the_oracles_bit_for_bit(rows, d):
    say(f"checkpoint_q8 {rows} x {d}")
    bits = inputs.gaussian_bf16((rows, d), 1.0, rows + d, 1)
    wide = so.bf16_to_f64(bits) * 2.0 ** np.random.default_rng(d).integers(-60, 60, (rows, d)).clip(-3, 3)
    x = torch.from_numpy(wide).to(sl.BF16)
    q, scale = sl.slope_checkpoint_q8(x.cuda())
    back = sl.slope_restore_q8(q, scale)
    codes, bytes_ = oo.checkpoint(f64(x))
    assert (scale.cpu().numpy() == bytes_).all() and (codes_of(q) == codes).all()
    assert (f64(back) == oo.restored(codes, bytes_)).all()


def test_checkpoint_at_the_ends_of_the_range():
    x = torch.zeros(8, 48, dtype=sl.BF16)
    x[1, 5] = 2.0 ** -133
    x[2, 0], x[2, 40] = 3.3895313892515355e38, -2.0 ** -126
    x[3, 31], x[3, 32] = float("inf"), 1.0
    x[4, 47] = float("nan")
    x[5, :] = -0.0
    x[6, :32] = torch.arange(32) * 14.0                                     # up to 434, ties among them
    x[7, 0], x[7, 1], x[7, 33] = 448.0 * 2.0 ** -126, 2.0 ** -133, 1.9375 * 2.0 ** 127
    q, scale = sl.slope_checkpoint_q8(x.cuda())
    back = f64(sl.slope_restore_q8(q, scale))
    codes, bytes_ = oo.checkpoint(f64(x))
    assert (scale.cpu().numpy() == bytes_).all()
    fine = np.repeat(bytes_ != 255, 32, axis=1)[:, :48]
    assert (codes_of(q)[fine] == codes[fine]).all()
    want = oo.restored(codes, bytes_)
    assert (np.isnan(back) == ~fine).all() and (back[fine] == want[fine]).all()


def test_restore_reads_every_code_and_byte():
    """All 256 codes under all 256 bytes: code * 2^(byte - 127), rounded to bf16 where that is below its range or above it."""
    codes = torch.arange(256, dtype=torch.uint8).repeat(256, 1)
    bytes_ = torch.arange(256, dtype=torch.uint8)[:, None].expand(256, 8).contiguous()
    got = f64(sl.slope_restore_q8(codes.cuda().view(sl.E4M3), bytes_.cuda()))
    want = oo.restored(codes.numpy(), bytes_.numpy())
    normal = np.abs(want) >= 2.0 ** -126
    inside = normal & (np.abs(want) < 3.39e38)
    assert (got[inside] == want[inside]).all() and (np.isnan(got) == np.isnan(want)).all()
    small = ~normal & ~np.isnan(want)
    assert (np.abs(got[small] - want[small]) <= 2.0 ** -134).all()          # half a step of bf16's smallest
    assert np.isinf(got[np.abs(want) >= 3.4e38]).all()


# ------------------------------------------------------------------------------------------- the weight gradient from 8-bit blocks
@pytest.mark.parametrize("b,d_out,d_in", [(1, 8, 8), (3, 64, 40), (64, 256, 256), (100, 72, 1000), (200, 1000, 264), (333, 512, 2048),
                                          (700, 1032, 448), (1000, 1000, 1000), (2050, 256, 512), (65, 4160, 96), (130, 2304, 2304), (1536, 4096, 4128)])
def test_weight_gradient(b, d_out, d_in):
    say(f"wgrad_masked_q8 b={b} d_out={d_out} d_in={d_in}")
    t = inputs.layer_inputs(b, d_out, d_in, seed=b + d_out)
    _, meta, _ = so.prune_rows_packed(t["W"])
    q, scale = sl.slope_checkpoint_q8(sl.bf16_to_device(t["X"]))
    dy, m = sl.bf16_to_device(t["dY"]), torch.from_numpy(meta).cuda()
    x = oo.restored(codes_of(q), scale.cpu().numpy())
    buf = torch.full((d_out * d_in // 2 + 8192,), 7.0, dtype=sl.BF16, device="cuda")
    out = buf[4096:4096 + d_out * d_in // 2].view(d_out, d_in // 2)
    sl.slope_wgrad_masked_q8(dy, q, scale, m, out=out)
    again = sl.slope_wgrad_masked_q8(dy, q, scale, m)
    torch.cuda.synchronize()
    assert torch.equal(out, again) and (buf[:4096] == 7).all() and (buf[4096 + d_out * d_in // 2:] == 7).all()
    xb = inputs.f32_to_bf16_bits(x.astype(np.float32))                      # exact: codes stand for bf16 numbers
    assert (so.bf16_to_f64(xb) == x).all()
    check_product(sl.bf16_to_host(out), so.wgrad_masked(t["dY"], xb, meta), "dW")


# X restored on the way by groups of wavefronts, by those of a tile that load; first, as stored, token-contiguous; dY's copy; tiles cut along the
# tokens; layers whose rows are no multiple of 32
FORMS = [(1024, 1000, 1000, ["wgrad_groups"]), (512, 2264, 696, ["wgrad_groups"]), (513, 2264, 696, ["dense_tn 64 128"]), (912, 1024, 2048, ["dense_tn 64 128"]),
         (1025, 1000, 1000, ["dense_tn 64 64"]), (1500, 200, 2200, ["dense_tn 64 64"]), (300, 2048, 2048, ["dense_tn 128 128"]), (1100, 1032, 1992, ["dense_tn 128 128"]),
         (65, 2048, 2040, ["dense_tn 128 128"]), (33, 4160, 1032, ["dense_tn 192 128"]), (130, 2560, 2568, ["dense_tn 256 128"]), (16384, 1024, 1024, ["dense_tn 256 128", "skinny_sum"]), (2047, 2040, 2056, ["dense_tn 192 128"]),
         (700, 4160, 2112, ["restore", "dense_tn 192 192"]), (8192, 2560, 2568, ["restore", "dense_tn 256 128"]),
         (4053, 3008, 392, ["dense_tn 256 128", "skinny_sum"]), (4854, 2704, 144, ["dense_tn 192 128", "skinny_sum"]), (3591, 136, 2112, ["dense_tn 128 128", "skinny_sum"]),
         (2068, 2736, 72, ["dense_tn 64 128", "skinny_sum"]), (1421, 64, 64, ["dense_tn 64 64", "skinny_sum"]), (16384, 256, 256, ["dense_tn 64 64", "skinny_sum"]),
         (1155, 3752, 2352, ["restore", "dense_tn 256 192"]),
         (16384, 4096, 768, ["restore_transposed", "dense_tn_split", "tail_finish"]), (18181, 3280, 1184, ["restore_transposed", "dense_tn_split", "tail_finish"]),
         (2048, 5120, 5120, ["restore_transposed", "dense_tn_split"]),
         (999, 4096, 16384, ["restore_transposed", "transpose_pad", "dense_tn_split"]),
         (1033, 9216, 9216, ["restore_transposed", "dense_tn_split", "dense_tn_split", "tail_finish"]),
         (1024, 4096, 16640, ["restore_transposed", "transpose_pad", "dense_tn_split", "dense_tn_split", "tail_finish"])]


@pytest.mark.parametrize("b,d_out,d_in,names", FORMS)
def test_weight_gradient_of_every_form(b, d_out, d_in, names):
    """Some rows of dW against 64 bits; which kernels ran."""
    say(f"wgrad_masked_q8 forms b={b} d_out={d_out} d_in={d_in}")
    gen = torch.Generator(device="cuda").manual_seed(b)
    x = torch.randn(b, d_in, generator=gen, device="cuda").to(sl.BF16)
    dy = torch.randn(b, d_out, generator=gen, device="cuda").mul_(1e-3).to(sl.BF16)
    _, meta, _ = sl.slope_prune_rows(torch.randn(d_out, d_in, generator=gen, device="cuda").to(sl.BF16))
    q, scale = sl.slope_checkpoint_q8(x)
    need = sl.slope_workspace_bytes(sl.SLOPE_CALL_WGRAD_MASKED_Q8, b, d_in, d_out)
    assert (need > 0) == (len(names) > 1)
    ws = torch.empty(max(256, need), dtype=torch.uint8, device="cuda")
    out = torch.zeros(d_out, d_in // 2, dtype=sl.BF16, device="cuda")
    ran = kernels(lambda: sl.slope_wgrad_masked_q8(dy, q, scale, meta, out=out, workspace=ws))
    assert [k.replace("_kernel", "") + (" %d %d" % n[:2] if k == "dense_tn_kernel" else "") for k, n in ran] == names
    sl.slope_wgrad_masked_q8(dy, q, scale, meta, out=out, workspace=ws)
    rows = torch.randperm(d_out, generator=torch.Generator().manual_seed(1))[:96].sort().values.cuda()
    want = dy[:, rows].double().t().contiguous() @ sl.slope_restore_q8(q, scale).double()
    mask = torch.from_numpy(so.meta_to_mask(meta[rows].cpu().numpy())).cuda()
    check_product(sl.bf16_to_host(out[rows]), want[mask].view(len(rows), -1).cpu().numpy(), "dW")


# ----------------------------------------------------------------------------------------------------------- as they are used
def test_one_training_step_of_a_layer_against_the_oracle():
    """Forward that keeps 8 bits, the gradient from the codes, both products of the backward pass, all by the library."""
    b, d_ff, d_in = 300, 520, 256
    p = Layer(b, d_ff, d_in, 0, seed=11)
    vals_t, meta_t, _ = sl.slope_double_prune(p.vals, p.meta)
    xq, xs = sl.slope_checkpoint_q8(p.x)
    h, _, q, scale = sl.slope_gated_fwd(p.x, p.vals, p.meta, want_q8=True)
    dh_bits = inputs.gaussian_bf16((b, d_ff), 1e-3, 11, 3)
    dgu, again = sl.slope_gated_bwd(sl.bf16_to_device(dh_bits), q8=q, scale=scale)
    dx = sl.slope_spmm_bwd_x(dgu, vals_t, meta_t)
    dw = sl.slope_wgrad_masked_q8(dgu, xq, xs, p.meta)
    torch.cuda.synchronize()
    check_gradient(dgu, again, double(sl.bf16_to_device(dh_bits)), restored(q.view(2 * b, d_ff), scale.view(2 * b, -1)).view(b, 2 * d_ff), "silu")
    # the products from the device's own dgu, the weights dense again
    dense = so.bf16_to_f64(so.unpack_2to4(sl.bf16_to_host(vals_t), meta_t.cpu().numpy())).T
    check_product(sl.bf16_to_host(dx), f64(dgu) @ dense, "dX")
    xr = inputs.f32_to_bf16_bits(oo.restored(codes_of(xq), xs.cpu().numpy()).astype(np.float32))
    check_product(sl.bf16_to_host(dw), so.wgrad_masked(sl.bf16_to_host(dgu), xr, p.meta.cpu().numpy()), "dW")


def test_captured_and_replayed_with_new_inputs_between_eager_calls():
    """Two graphs of the whole step on one set of buffers each, replayed in turn with eager work between."""
    b, d_ff, d_in, r = 70, 264, 512, 32
    runs = []
    for seed in (1, 2):
        p = Layer(b, d_ff, d_in, r, seed=seed)
        ws = torch.empty(max(256, sl.slope_workspace_bytes(sl.SLOPE_CALL_GATED_FWD, b, d_in, d_ff, r)), dtype=torch.uint8, device="cuda")
        dh = sl.bf16_to_device(inputs.gaussian_bf16((b, d_ff), 1e-3, seed, 3))

        def step(p=p, ws=ws, dh=dh):
            h, _, q, s = sl.slope_gated_fwd(p.x, p.vals, p.meta, L=p.l, R=p.r, want_q8=True, workspace=ws)
            xq, xs = sl.slope_checkpoint_q8(p.x)
            dgu, again = sl.slope_gated_bwd(dh, q8=q, scale=s)
            return h, dgu, again, sl.slope_wgrad_masked_q8(dgu, xq, xs, p.meta), sl.slope_restore_q8(xq, xs)

        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = step()
        runs.append((graph, held, p, step))
    for turn in range(4):
        for graph, held, p, step in runs:
            p.x.copy_(torch.randn(p.x.shape, generator=torch.Generator().manual_seed(turn)).to(sl.BF16))
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in held]
            for a, e in zip(got, step()):
                assert torch.equal(a, e)


# ------------------------------------------------------------------------------------------------- offsets that pass 32 bits
def far_rows(b):
    """Rows at both ends and on both sides of the middle ones."""
    return torch.cat([torch.arange(0, 40), torch.arange(b // 2 - 20, b // 2 + 20), torch.arange(b - 40, b)]).cuda()


def test_checkpoints_and_gradient_of_more_than_two_to_the_32_elements():
    say("more than 2^32 elements")
    rows, d = 560_008, 8200                                                 # 4.6e9
    x = torch.randn(4099, d, device="cuda").to(sl.BF16).repeat(rows // 4099 + 1, 1)[:rows].contiguous()
    q, scale = sl.slope_checkpoint_q8(x)
    back = sl.slope_restore_q8(q, scale)
    at = far_rows(rows)
    q1, s1 = sl.slope_checkpoint_q8(x[at].contiguous())
    assert torch.equal(codes(q)[at], codes(q1)) and torch.equal(scale[at], s1) and torch.equal(back[at], sl.slope_restore_q8(q1, s1))
    del back
    b, d_ff = rows // 2, d                                                  # the rows as a gate and an up projection each
    dh = torch.randn(4099, d_ff, device="cuda").to(sl.BF16).repeat(b // 4099 + 1, 1)[:b].contiguous()
    at = far_rows(b)
    pairs = lambda t: t.view(b, -1)[at].contiguous()                        # noqa: E731
    dgu, h = sl.slope_gated_bwd(dh, gu=x.view(b, 2 * d_ff))
    dgu1, h1 = sl.slope_gated_bwd(dh[at].contiguous(), gu=pairs(x))
    assert torch.equal(dgu[at], dgu1) and torch.equal(h[at], h1)
    del dgu, h
    dgu, h = sl.slope_gated_bwd(dh, q8=q.view(b, 2 * d_ff), scale=scale.view(b, 2, -1))
    dgu1, h1 = sl.slope_gated_bwd(dh[at].contiguous(), q8=codes(q).view(b, -1)[at].contiguous().view(q.dtype).view(len(at), 2 * d_ff),
                                  scale=pairs(scale).view(len(at), 2, -1))
    assert torch.equal(dgu[at], dgu1) and torch.equal(h[at], h1)


def codes(q):
    return q.view(torch.uint8)


@pytest.mark.parametrize("b,d_out,d_in", [(1_060_001, 64, 4160), (1_060_001, 72, 4104), (40, 64, (1 << 24) + 64)])
def test_weight_gradient_of_long_batches_and_wide_layers(b, d_out, d_in):
    """More than 2^32 codes, restored on the way by wavefronts that load, and a layer wider than the tiles take: as from X restored first."""
    say(f"wgrad_masked_q8 b={b} d_out={d_out} d_in={d_in}")
    gen = torch.Generator(device="cuda").manual_seed(1)
    part = min(b, 4099)
    x = torch.randn(part, d_in, generator=gen, device="cuda").to(sl.BF16)
    q, scale = (t.repeat(b // part + 1, 1)[:b].contiguous() for t in map(codes, sl.slope_checkpoint_q8(x)))
    dy = torch.randn(b, d_out, generator=gen, device="cuda").mul_(1e-3).to(sl.BF16)
    _, meta, _ = sl.slope_prune_rows(torch.randn(d_out, d_in, generator=gen, device="cuda").to(sl.BF16))
    got = sl.slope_wgrad_masked_q8(dy, q.view(torch.float8_e4m3fn), scale, meta)
    want = sl.slope_wgrad_masked(dy, sl.slope_restore_q8(q.view(torch.float8_e4m3fn), scale), meta)
    if d_in > 1 << 20:                                                      # (then the same kernel)
        assert torch.equal(got, want)
    else:
        check_product(sl.bf16_to_host(got), f64(want), "dW")


def test_forward_of_more_than_two_to_the_32_elements():
    say("gated_fwd of long batches")
    b, d_ff, d_in = 1_060_001, 2048, 128                                    # kept projections: 4.3e9
    p = Layer(3, d_ff, d_in, 0, seed=5)
    p.x = torch.randn(b, d_in, device="cuda").to(sl.BF16)
    h, gu, q, scale = sl.slope_gated_fwd(p.x, p.vals, p.meta, want_gu=True, want_q8=True)
    at = far_rows(b)
    x, w = double(p.x[at]), dense_of(p.vals, p.meta).t().contiguous()
    want, off = x @ w, (d_in / 2 + 8) * 2.0 ** -24 * (x.abs() @ w.abs())
    check_h(h[at], want, off, "silu", "h")
    check_kept(gu[at], want, off, "gu")
    check_blocks(codes(q)[at].view(-1, d_ff), scale[at].view(2 * len(at), -1), want.view(-1, d_ff), off.view(-1, d_ff), "codes")


def test_on_another_stream():
    p = Layer(150, 264, 640, 0, seed=4)
    want = sl.slope_gated_fwd(p.x, p.vals, p.meta)[0]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = sl.slope_gated_fwd(p.x, p.vals, p.meta)[0]
    side.synchronize()
    assert torch.equal(got, want)


def test_two_graphs_share_a_workspace():
    """Calls of two layers, each captured, with one workspace: its contents are a call's own."""
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    runs = []
    for b, d_ff, d_in, r, seed in ((128, 200, 4096, 32, 1), (1000, 520, 1000, 0, 2), (4053, 1504, 392, 0, 3)):
        p = Layer(b, d_ff, d_in, r, seed=seed)
        dgu = sl.bf16_to_device(inputs.gaussian_bf16((b, 2 * d_ff), 1e-3, seed, 3))
        xq, xs = sl.slope_checkpoint_q8(p.x)

        def step(p=p, dgu=dgu, xq=xq, xs=xs):
            h, _, q, s = sl.slope_gated_fwd(p.x, p.vals, p.meta, L=p.l, R=p.r, want_q8=True, workspace=ws)
            return h, codes(q), s, sl.slope_wgrad_masked_q8(dgu, xq, xs, p.meta, workspace=ws)

        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = step()
        runs.append((graph, held, want, step))                              # (step holds the operands, which the graph reads)
    for turn in range(3):
        for graph, held, want, _ in runs:
            ws.fill_(255)                                                   # NaN, were it read
            graph.replay()
            for a, e in zip(held, want):
                assert torch.equal(a, e)


def test_two_streams_at_once():
    p = Layer(515, 1000, 256, 96, seed=6)
    want = sl.slope_gated_fwd(p.x, p.vals, p.meta, L=p.l, R=p.r, want_gu=True)[:2]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for turn in range(8):
        with torch.cuda.stream(streams[turn % 2]):
            got.append(sl.slope_gated_fwd(p.x, p.vals, p.meta, L=p.l, R=p.r, want_gu=True)[:2])
    torch.cuda.synchronize()
    for h, gu in got:
        assert torch.equal(h, want[0]) and torch.equal(gu, want[1])


def test_the_binding_refuses_wrong_types_shapes_and_strides():
    b, d_ff, d_in = 8, 64, 128
    p = Layer(b, d_ff, d_in, 32, seed=7)
    h, gu, q, s = sl.slope_gated_fwd(p.x, p.vals, p.meta, L=p.l, R=p.r, want_gu=True, want_q8=True)
    xq, xs = sl.slope_checkpoint_q8(p.x)
    small = torch.empty(16, dtype=torch.uint8, device="cuda")
    wide = torch.zeros(b, 2 * d_in, dtype=sl.BF16, device="cuda")
    bad = [lambda: sl.slope_gated_fwd(wide[:, :d_in], p.vals, p.meta), lambda: sl.slope_gated_fwd(p.x.float(), p.vals, p.meta),
           lambda: sl.slope_gated_fwd(p.x, p.vals, p.meta[:-1]), lambda: sl.slope_gated_fwd(p.x, p.vals[:-1], p.meta[:-1]),
           lambda: sl.slope_gated_fwd(p.x, p.vals, p.meta, L=p.l), lambda: sl.slope_gated_fwd(p.x, p.vals, p.meta, L=p.l, R=p.r[:, :d_ff]),
           lambda: sl.slope_gated_fwd(p.x, p.vals, p.meta, L=p.l, R=p.r, workspace=small), lambda: sl.slope_gated_fwd(p.x, p.vals, p.meta, out=(gu, None, None, None)),
           lambda: sl.slope_gated_fwd(p.x, p.vals, p.meta, out=(h, h, None, None)), lambda: sl.slope_gated_fwd(p.x, p.vals, p.meta, out=(h, None, q, s[:, :1])),
           lambda: sl.slope_gated_bwd(h, gu=gu, q8=q, scale=s), lambda: sl.slope_gated_bwd(h, gu=h), lambda: sl.slope_gated_bwd(h, q8=q), lambda: sl.slope_gated_bwd(h, q8=gu, scale=s),
           lambda: sl.slope_checkpoint_q8(p.x.t()), lambda: sl.slope_restore_q8(xq, xs[:, :1]), lambda: sl.slope_restore_q8(codes(xq), xs),
           lambda: sl.slope_wgrad_masked_q8(gu, xq, xs[:-1], p.meta), lambda: sl.slope_wgrad_masked_q8(gu[:-1], xq, xs, p.meta),
           lambda: sl.slope_wgrad_masked_q8(gu, p.x, xs, p.meta), lambda: sl.slope_wgrad_masked_q8(gu, xq, xs, p.meta[:, :-1])]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: sl.slope_gated_fwd(p.x, p.vals, p.meta, act=3), lambda: sl.slope_gated_bwd(h, act=-1, gu=gu),
                 lambda: sl.slope_gated_fwd(p.x, p.vals, p.meta, L=p.l, R=p.r, workspace=None), lambda: sl.slope_gated_fwd(p.x, p.vals, p.meta, out=(h, None, q, None))):
        with pytest.raises(sl.SlopeError):
            call()
