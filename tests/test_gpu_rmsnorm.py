"""RMS norm with residual and 8-bit output, and its gradient: HIP path vs the fp64 oracle.

Bounds.  bf16 has 8 significant bits: rounding to it is off by at most 2^-8 of the value.  The sum over a row is a sum of at most 2^8 fp32
roundings in sequence per lane, then a tree: its relative error stays below 2^-16 for all positive terms, that of its root below
2^-17; products add a few 2^-24.  e4m3: neighbours are 1/8 of a value or 2^-9 apart, so codes are off by 2^-4 of the value or
2^-10 at most, plus the scale's error.
"""
import numpy as np
import pytest
import torch

from oracle import slope_oracle as so
from oracle import surroundings_oracle as oo
from paper_2405_16325_amd import binding as sl
from paper_2405_16325_amd import inputs

pytestmark = pytest.mark.gpu

EPS = 1e-5
# every way rows are shared out: 8, 16, 32 lanes a row, one wavefront with one or more pieces a lane, several wavefronts, rows
# that stay in memory (past 24576 elements for the gradient, past 32768 forward); rows that do not fill the last workgroup
SHAPES = [(1, 8), (33, 64), (5, 72), (70, 128), (9, 136), (9, 256), (1, 264), (6, 512), (17, 520), (1, 768), (1000, 1000), (2, 2048),
          (3, 2056), (2100, 2056), (2049, 768), (2, 4104), (5, 9216), (2050, 9216), (3, 20480), (2048, 5120), (2, 36864), (1, 65536),
          (2, 65544), (3, 131080)]


def say(msg):
    print(msg, flush=True)


def bf16(shape, std, seed, stream):
    bits = inputs.gaussian_bf16(shape, std, seed, stream)
    return bits, sl.bf16_to_device(bits)


def host(t):
    return so.bf16_to_f64(sl.bf16_to_host(t))


def weights(d, seed):
    bits = inputs.f32_to_bf16_bits((1 + 0.1 * np.random.default_rng(seed).standard_normal(d)).astype(np.float32))
    return bits, sl.bf16_to_device(bits)


def norm_case(b, d, residual, scale=1.0):
    x, dx = bf16((b, d), scale, b * 7 + d, 1)
    r, dr = bf16((b, d), 2.0 * scale, b * 7 + d, 2) if residual else (None, None)
    w, dw = weights(d, d)
    h = x if r is None else inputs.f32_to_bf16_bits(inputs.bf16_bits_to_f32(x) + inputs.bf16_bits_to_f32(r))
    return dx, dr, dw, h, so.bf16_to_f64(h), so.bf16_to_f64(w)


def check_outputs(h, w, y, rstd, q, scale):
    want, r = oo.rmsnorm(h, w, EPS)
    if y is not None:
        assert (np.abs(host(y) - want) <= (2.0 ** -8 + 2.0 ** -16) * np.abs(want) + 1e-38).all()
    if rstd is not None:
        assert (np.abs(rstd.cpu().numpy() - r) <= 2.0 ** -16 * r).all()
    if q is not None:
        s = np.abs(want).max(1) / 448
        got_s = scale.cpu().numpy().astype(np.float64)
        assert (np.abs(got_s - s) <= 2.0 ** -15 * s).all()
        codes = q.view(torch.uint8).cpu().numpy()
        off = np.abs(oo.e4m3_value(codes) * got_s[:, None] - want)
        assert (off <= (2.0 ** -4 * np.abs(want) + 2.0 ** -10 * got_s[:, None]) * (1 + 2.0 ** -12) + 2.0 ** -14 * np.abs(want)).all()


@pytest.mark.parametrize("b,d", SHAPES)
@pytest.mark.parametrize("residual", [False, True])
def test_forward(b, d, residual):
    say(f"rmsnorm_fwd b={b} d={d} residual={residual}")
    x, res, w, h_bits, h, wv = norm_case(b, d, residual)
    y, H, rstd, q, scale = sl.slope_rmsnorm_fwd(x, w, EPS, residual=res, want_rstd=True, want_q8=True)
    torch.cuda.synchronize()
    assert (H is None) == (not residual)
    if residual:
        assert (sl.bf16_to_host(H) == h_bits).all()
    check_outputs(h, wv, y, rstd, q, scale)


@pytest.mark.parametrize("b,d", [(3, 768), (40, 64), (2, 65544)])
def test_outputs_alone_equal_outputs_together(b, d):
    say(f"rmsnorm_fwd outputs apart b={b} d={d}")
    x, res, w, _, _, _ = norm_case(b, d, True)
    y, H, rstd, q, scale = sl.slope_rmsnorm_fwd(x, w, EPS, residual=res, want_rstd=True, want_q8=True)
    y2 = sl.slope_rmsnorm_fwd(x, w, EPS, residual=res)[0]
    _, H2, _, q2, scale2 = sl.slope_rmsnorm_fwd(x, w, EPS, residual=res, want_y=False, want_q8=True)
    assert torch.equal(y, y2) and torch.equal(H, H2) and torch.equal(scale, scale2)
    assert torch.equal(q.view(torch.uint8), q2.view(torch.uint8))


@pytest.mark.parametrize("b,d", [(5, 72), (3, 5120), (2, 65544)])
@pytest.mark.parametrize("into", ["x", "residual"])
def test_the_stream_in_place(b, d, into):
    say(f"rmsnorm_fwd in place b={b} d={d} into={into}")
    x, res, w, h_bits, h, wv = norm_case(b, d, True)
    y, q, scale = torch.empty_like(x), torch.empty((b, d), dtype=sl.E4M3, device="cuda"), torch.empty(b, device="cuda")
    H = x if into == "x" else res
    sl.slope_rmsnorm_fwd(x, w, EPS, residual=res, out=(y, H, None, q, scale))
    torch.cuda.synchronize()
    assert (sl.bf16_to_host(H) == h_bits).all()
    check_outputs(h, wv, y, None, q, scale)


@pytest.mark.parametrize("d", [64, 768, 9216, 65544])
def test_rows_of_zeros_infinities_and_nan_stay_by_themselves(d):
    say(f"rmsnorm_fwd special rows d={d}")
    x, _, w, _, h, wv = norm_case(6, d, False)
    x[1] = 0.0
    x[3, 5] = float("inf")
    x[4, d - 1] = float("nan")
    y, _, rstd, q, scale = sl.slope_rmsnorm_fwd(x, w, EPS, want_rstd=True, want_q8=True)
    torch.cuda.synchronize()
    keep = [0, 2, 5]
    check_outputs(h[keep], wv, y[keep], rstd[keep], q.view(torch.uint8)[keep].view(sl.E4M3), scale[keep])
    assert (host(y)[1] == 0).all() and scale[1] == 0 and (q.view(torch.uint8)[1] & 0x7F == 0).all()
    assert abs(float(rstd[1]) - EPS ** -0.5) < 1e-3
    assert torch.isnan(y[4]).all() and not torch.isfinite(scale[4]) and not torch.isfinite(scale[3])


def test_magnitudes_far_from_one():
    for scale in (1e-15, 1e15):
        x, res, w, h_bits, h, wv = norm_case(4, 776, True, scale)
        y, H, rstd, q, s = sl.slope_rmsnorm_fwd(x, w, EPS, residual=res, want_rstd=True, want_q8=True)
        assert (sl.bf16_to_host(H) == h_bits).all()
        check_outputs(h, wv, y, rstd, q, s)


def test_nothing_outside_the_outputs_is_written_and_another_stream():
    b, d = 5, 776
    x, res, w, h_bits, h, wv = norm_case(b, d, True)
    big = [torch.full((b * d + 4096,), 7.0, dtype=sl.BF16, device="cuda") for _ in range(2)]
    qb = torch.full((b * d + 4096,), 0x55, dtype=torch.uint8, device="cuda")
    sb = torch.full((b + 1024,), 7.0, device="cuda")
    y, H = (t[2048:2048 + b * d].view(b, d) for t in big)
    q, s = qb[2048:2048 + b * d].view(sl.E4M3).view(b, d), sb[512:512 + b]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        sl.slope_rmsnorm_fwd(x, w, EPS, residual=res, out=(y, H, None, q, s))
    stream.synchronize()
    check_outputs(h, wv, y, None, q, s)
    for t in big:
        assert (t[:2048] == 7).all() and (t[2048 + b * d:] == 7).all()
    assert (qb[:2048] == 0x55).all() and (qb[2048 + b * d:] == 0x55).all() and (sb[:512] == 7).all() and (sb[512 + b:] == 7).all()


def grad_case(b, d, residual):
    hb, h = bf16((b, d), 2.0, b + d, 3)
    yb, dy = bf16((b, d), 1e-3, b + d, 4)
    eb, dh = bf16((b, d), 1e-3, b + d, 5) if residual else (None, None)
    wb, w = weights(d, d + 1)
    hv = so.bf16_to_f64(hb)
    r = (1 / np.sqrt((hv * hv).mean(1) + EPS)).astype(np.float32)
    values = [so.bf16_to_f64(t) if t is not None else None for t in (yb, hb, wb, eb)]
    return dy, h, w, torch.from_numpy(r).cuda(), dh, values, r.astype(np.float64)


def check_grads(dx, dw, values, r):
    """bf16 rounding, plus fp32 sums: 2^-16 of the magnitudes that are added (dx: three terms; dw: the tokens')."""
    dyv, hv, wv, ev = values
    want_dx, want_dw = oo.rmsnorm_grad(dyv, hv, wv, r, ev)
    xh = np.abs(hv) * r[:, None]
    g = np.abs(dyv * wv)
    terms = r[:, None] * (g + xh * (g * xh).mean(1, keepdims=True)) + (0 if ev is None else np.abs(ev))
    assert (np.abs(host(dx) - want_dx) <= (2.0 ** -8 + 2.0 ** -16) * np.abs(want_dx) + 2.0 ** -16 * terms).all()
    assert (np.abs(host(dw) - want_dw) <= (2.0 ** -8 + 2.0 ** -16) * np.abs(want_dw) + 2.0 ** -16 * (np.abs(dyv) * xh).sum(0)).all()


@pytest.mark.parametrize("b,d", SHAPES)
@pytest.mark.parametrize("residual", [False, True])
def test_gradient(b, d, residual):
    say(f"rmsnorm_bwd b={b} d={d} residual={residual}")
    dy, h, w, rstd, dh, values, r = grad_case(b, d, residual)
    dx, dw = sl.slope_rmsnorm_bwd(dy, h, w, rstd, dh=dh)
    again = sl.slope_rmsnorm_bwd(dy, h, w, rstd, dh=dh)
    torch.cuda.synchronize()
    check_grads(dx, dw, values, r)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])


@pytest.mark.parametrize("b,d", [(70, 128), (3, 5120), (3, 36864)])
@pytest.mark.parametrize("into", ["dy", "dh"])
def test_gradient_in_place(b, d, into):
    say(f"rmsnorm_bwd in place b={b} d={d} into={into}")
    dy, h, w, rstd, dh, values, r = grad_case(b, d, True)
    dx, dw = sl.slope_rmsnorm_bwd(dy, h, w, rstd, dh=dh, out=(dy if into == "dy" else dh, torch.empty_like(w)))
    torch.cuda.synchronize()
    check_grads(dx, dw, values, r)


# both gradients in one launch and, written over dY or of more rows or elements, in two: every number of lanes or wavefronts a row
@pytest.mark.parametrize("b,d", [(1, 8), (1024, 8), (1025, 8), (1023, 64), (1100, 72), (1024, 136), (1500, 256), (700, 264), (1024, 1032),
                                 (1030, 768), (100, 1544), (300, 2056), (65, 2568), (600, 3080), (9, 8192), (640, 8192), (641, 8192), (1, 8200), (5, 9216), (569, 9216), (570, 9216),
                                 (3, 12296), (320, 16384), (2, 16392)])
@pytest.mark.parametrize("over_dy", [False, True])
def test_gradient_in_one_launch_and_in_two(b, d, over_dy):
    say(f"rmsnorm_bwd launches b={b} d={d} over_dy={over_dy}")
    dy, h, w, rstd, dh, values, r = grad_case(b, d, b % 2 == 0)
    dx, dw = sl.slope_rmsnorm_bwd(dy, h, w, rstd, dh=dh, out=(dy if over_dy else torch.empty_like(dy), torch.empty_like(w)))
    torch.cuda.synchronize()
    check_grads(dx, dw, values, r)


def test_gradient_against_differences_of_the_forward():
    """The forward's own fp32 row statistics and 8 significant bits of y bound a difference: steps of a quarter of the values'
    size, so that the second-order term, not the rounding, is what the fp64 function's own difference also has."""
    b, d = 4, 64
    dy, h, w, rstd, _, (dyv, hv, wv, _), r = grad_case(b, d, False)
    dx, _ = sl.slope_rmsnorm_bwd(dy, h, w, rstd)
    step = 1e-4
    for i, j in ((0, 0), (1, 17), (3, 63)):
        e = np.zeros_like(hv)
        e[i, j] = step
        diff = ((oo.rmsnorm(hv + e, wv, EPS)[0] - oo.rmsnorm(hv - e, wv, EPS)[0]) * dyv).sum() / (2 * step)
        scale = float(np.abs(dyv[i] * wv).max() * r[i])
        assert abs(float(dx[i, j]) - diff) <= 2.0 ** -8 * abs(diff) + 1e-4 * scale


def test_graph_replays_equal_eager_calls():
    b, d = 40, 776
    x, res, w, _, _, _ = norm_case(b, d, True)
    dy, h, w2, rstd, dh, _, _ = grad_case(b, d, True)
    ws = torch.empty(sl.slope_workspace_bytes(sl.SLOPE_CALL_RMSNORM_BWD, b, d, 0), dtype=torch.uint8, device="cuda")
    fwd = (torch.empty_like(x), torch.empty_like(x), None, torch.empty((b, d), dtype=sl.E4M3, device="cuda"), torch.empty(b, device="cuda"))
    bwd = (torch.empty_like(dy), torch.empty_like(w2))

    def call():
        sl.slope_rmsnorm_fwd(x, w, EPS, residual=res, out=fwd)
        sl.slope_rmsnorm_bwd(dy, h, w2, rstd, dh=dh, out=bwd, workspace=ws)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for turn in range(4):
        x.copy_(torch.randn(b, d, device="cuda") * (turn + 1))
        dy.copy_(torch.randn(b, d, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (fwd[0], fwd[1], fwd[3].view(torch.uint8), fwd[4], *bwd)]
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (fwd[0], fwd[1], fwd[3].view(torch.uint8), fwd[4], *bwd)))


# calls that move more than the last-level cache holds go past it: every number of pieces a lane, the last workgroup's rows and the last
# pieces of a row incomplete among them.  Compared on the device, in fp64, within the bounds of the small shapes.
@pytest.mark.parametrize("b,d", [(4200, 8184), (4100, 9216), (2201, 16376), (1701, 20488), (1100, 32768)])
@pytest.mark.parametrize("residual", [False, True])
def test_forward_past_the_last_level_cache(b, d, residual):
    if not residual:
        b = (256 << 20) // (5 * d) + 1
    assert b * d * (9 if residual else 5) > 256 << 20
    say(f"rmsnorm_fwd past the caches b={b} d={d} residual={residual}")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(b + d)
    x = torch.randn(b, d, generator=gen, device="cuda").to(sl.BF16)
    res = (2 * torch.randn(b, d, generator=gen, device="cuda")).to(sl.BF16) if residual else None
    w = (1 + 0.1 * torch.randn(d, generator=gen, device="cuda")).to(sl.BF16)
    y, H, rstd, q, scale = sl.slope_rmsnorm_fwd(x, w, EPS, residual=res, want_rstd=True, want_q8=True)
    h = x if res is None else (x.float() + res.float()).to(sl.BF16)
    assert H is None if res is None else torch.equal(H, h)
    for at in range(0, b, 1000):
        rows = slice(at, at + 1000)
        want = h[rows].double()
        r = (want.square().mean(1) + EPS).rsqrt()
        want = want * r[:, None] * w.double()
        assert bool(((y[rows].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -16) * want.abs() + 1e-38).all())
        assert bool(((rstd[rows].double() - r).abs() <= 2.0 ** -16 * r).all())
        s, got = want.abs().amax(1) / 448, scale[rows].double()
        assert bool(((got - s).abs() <= 2.0 ** -15 * s).all())
        off = (q[rows].double() * got[:, None] - want).abs()
        assert bool((off <= (2.0 ** -4 * want.abs() + 2.0 ** -10 * got[:, None]) * (1 + 2.0 ** -12) + 2.0 ** -14 * want.abs()).all())


@pytest.mark.parametrize("b,d", [(4200, 8184), (4100, 9216), (2201, 16376), (1701, 20488), (1401, 24576)])
@pytest.mark.parametrize("residual", [False, True])
def test_gradient_past_the_last_level_cache(b, d, residual):
    if not residual:
        b = (256 << 20) // (6 * d) + 1
    assert b * d * (8 if residual else 6) > 256 << 20
    say(f"rmsnorm_bwd past the caches b={b} d={d} residual={residual}")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(b + d + 1)
    h = (2 * torch.randn(b, d, generator=gen, device="cuda")).to(sl.BF16)
    dy = (1e-3 * torch.randn(b, d, generator=gen, device="cuda")).to(sl.BF16)
    dh = (1e-3 * torch.randn(b, d, generator=gen, device="cuda")).to(sl.BF16) if residual else None
    w = (1 + 0.1 * torch.randn(d, generator=gen, device="cuda")).to(sl.BF16)
    rstd = (h.float().square().mean(1) + EPS).rsqrt()
    dx, dw = sl.slope_rmsnorm_bwd(dy, h, w, rstd, dh=dh)
    want_dw, terms_dw = torch.zeros(d, dtype=torch.float64, device="cuda"), torch.zeros(d, dtype=torch.float64, device="cuda")
    for at in range(0, b, 1000):
        rows = slice(at, at + 1000)
        r = rstd[rows].double()[:, None]
        dyv, xh = dy[rows].double(), h[rows].double() * r
        g = dyv * w.double()
        want = r * (g - xh * (g * xh).mean(1, keepdim=True))
        terms = r * (g.abs() + xh.abs() * (g * xh).abs().mean(1, keepdim=True))
        if residual:
            want, terms = want + dh[rows].double(), terms + dh[rows].double().abs()
        assert bool(((dx[rows].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -16) * want.abs() + 2.0 ** -16 * terms).all())
        want_dw += (dyv * xh).sum(0)
        terms_dw += (dyv * xh).abs().sum(0)
    assert bool(((dw.double() - want_dw).abs() <= (2.0 ** -8 + 2.0 ** -16) * want_dw.abs() + 2.0 ** -16 * terms_dw).all())
    dw2 = torch.empty_like(dw)
    sl.slope_rmsnorm_bwd(dy, h, w, rstd, dh=dh, out=(dy, dw2))
    torch.cuda.synchronize()
    assert torch.equal(dy, dx) and torch.equal(dw, dw2)
