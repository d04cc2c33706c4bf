"""The oracle of the norm, the 8-bit format, the 8-bit product and the optimizer, pinned on its own (no GPU)."""
import numpy as np
import pytest

from oracle import surroundings_oracle as oo

F32 = np.float32


def rng(seed):
    return np.random.default_rng(seed)


def test_e4m3_values_by_hand():
    known = {0x00: 0.0, 0x01: 2.0 ** -9, 0x07: 7 * 2.0 ** -9, 0x08: 2.0 ** -6, 0x38: 1.0, 0x39: 1.125, 0x3F: 1.875, 0x40: 2.0,
             0x7E: 448.0, 0xB8: -1.0, 0xFE: -448.0}
    for code, value in known.items():
        assert oo.e4m3_value([code])[0] == value
    assert np.isnan(oo.e4m3_value([0x7F, 0xFF])).all()


def test_nearest_code_round_trip_ties_and_brute_force():
    codes = np.array([c for c in range(256) if c & 0x7F != 0x7F], np.uint8)
    assert (oo.e4m3_nearest(oo.e4m3_value(codes)) == codes).all()
    # halfway between neighbours: the even code
    mags = oo.e4m3_value(np.arange(0x7F))
    half = (mags[:-1] + mags[1:]) / 2
    got = oo.e4m3_nearest(half)
    assert (got % 2 == 0).all() and (np.abs(got.astype(int) - np.arange(0x7E) - 0.5) == 0.5).all()
    x = rng(1).normal(size=2000) * 10.0 ** rng(2).uniform(-4, 2, 2000)
    best = np.abs(np.minimum(np.abs(x), 448)[:, None] - mags[None]).min(1)
    assert np.allclose(np.abs(oo.e4m3_value(oo.e4m3_nearest(x)) - np.clip(x, -448, 448)), best, rtol=0, atol=0)


def test_norm_by_hand_and_scale_invariance():
    y, r = oo.rmsnorm([[3.0, 4.0]], [1.0, 2.0], 0.0)
    assert np.allclose(r, 1 / np.sqrt(12.5)) and np.allclose(y, [[3 / np.sqrt(12.5), 8 / np.sqrt(12.5)]])
    h, w = rng(3).normal(size=(4, 24)), rng(4).normal(size=24)
    assert np.allclose(oo.rmsnorm(7 * h, w, 0.0)[0], oo.rmsnorm(h, w, 0.0)[0])
    assert np.allclose(oo.rmsnorm(np.zeros((1, 8)), np.ones(8), 1e-5)[0], 0.0)


def test_norm_gradient_against_differences():
    h, w, dy, dh = rng(5).normal(size=(3, 16)), rng(6).normal(size=16), rng(7).normal(size=(3, 16)), rng(8).normal(size=(3, 16))
    eps, step = 1e-3, 1e-6
    loss = lambda a, b: float((oo.rmsnorm(a, b, eps)[0] * dy).sum() + (a * dh).sum())        # noqa: E731
    dx, dw = oo.rmsnorm_grad(dy, h, w, oo.rmsnorm(h, w, eps)[1], dh)
    for i in np.ndindex(h.shape):
        e = np.zeros_like(h)
        e[i] = step
        assert abs((loss(h + e, w) - loss(h - e, w)) / (2 * step) - dx[i]) < 1e-7
    for j in range(16):
        e = np.zeros_like(w)
        e[j] = step
        assert abs((loss(h, w + e) - loss(h, w - e)) / (2 * step) - dw[j]) < 1e-7


def test_product_against_triple_loop():
    b, d_out, d_in = 3, 8, 16
    g = rng(9)
    q, wq = g.integers(0, 0x7F, (b, d_in)).astype(np.uint8), g.integers(0, 0x7F, (d_out, d_in // 2)).astype(np.uint8)
    pairs = np.array([4, 8, 9, 12, 13, 14])
    nib = pairs[g.integers(0, 6, (d_out, d_in // 4))]
    meta = (nib[:, ::2] | nib[:, 1::2] << 4).astype(np.uint8)
    xs, ws = g.uniform(0.5, 2, b), g.uniform(0.5, 2, d_out)
    y, _ = oo.product_q8(q, xs, wq, meta, ws)
    for i in range(b):
        for j in range(d_out):
            want = 0.0
            for group in range(d_in // 4):
                for k in range(2):
                    col = 4 * group + (nib[j, group] >> (2 * k) & 3)
                    want += oo.e4m3_value([q[i, col]])[0] * oo.e4m3_value([wq[j, 2 * group + k]])[0]
            assert np.isclose(y[i, j], want * xs[i] * ws[j])


def test_dithered_rounding_brackets_the_value_and_is_unbiased():
    a = (rng(10).uniform(0, 448, 512) * 10.0 ** -rng(11).uniform(0, 5, 512)).astype(F32)
    steps = 500
    got = np.stack([oo.dithered(a, oo.threshold(a.size, t, False)) for t in range(1, steps + 1)])
    i = np.searchsorted(oo._VALUES, a.astype(np.float64), side="right") - 1
    low, high = oo._VALUES[i], oo._VALUES[np.minimum(i + 1, 0x7E)]
    assert ((got == low) | (got == high)).all()
    # evenly spread thresholds: the share of steps that round up is off by at most a few steps, not their square root
    off = np.abs(got.mean(0) - a) / np.maximum(high - low, 1e-9)
    assert off[a < 448].max() <= 4 / steps


def test_states_round_trip_within_a_code_and_a_root_never_vanishes():
    x = (rng(12).normal(size=1000) * 1e-4).astype(F32)
    codes, scales = oo.store_states(x, 17, False)
    back = oo.load_states(codes, scales)
    s = np.repeat(scales, oo.BLOCK)[:1000]
    assert (np.abs(back - x) <= np.maximum(0.125 * np.abs(x), 2.0 ** -9 * s) * (1 + 1e-6)).all()
    tiny = np.array([1.0] + [1e-12] * 50 + [0.0] * 20, F32)
    codes, scales = oo.store_states(tiny, 3, True)
    assert (codes[1:51] > 0).all() and (codes[51:] == 0).all()
    codes, scales = oo.store_states(np.zeros(130, F32), 3, True)
    assert (codes == 0).all() and (scales == 0).all()


def adamw_64(p, gs, lr, b1, b2, eps, wd):
    m = v = 0.0
    for t, g in enumerate(gs, 1):
        m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
        p = p - lr * wd * p - lr * (m / (1 - b1 ** t)) / (np.sqrt(v / (1 - b2 ** t)) + eps)
    return p


def test_adamw_against_the_definition_step_by_step():
    gs = rng(13).normal(size=(20, 64)).astype(F32)
    p0 = rng(14).normal(size=64)
    p, m, v = p0, np.zeros(64, F32), np.zeros(64, F32)
    for t, g in enumerate(gs, 1):
        p, m, v = oo.adamw(p, g, m, v, 1.0, 1e-2, 0.9, 0.99, 1e-8, 0.1, t)
    assert np.allclose(p, adamw_64(p0, gs.astype(np.float64), 1e-2, 0.9, 0.99, 1e-8, 0.1), rtol=1e-6, atol=1e-6)


def nearest_states(x, step, root):
    a = np.abs(x).reshape(-1, oo.BLOCK)
    scale, inv = oo.q8_scale(a.max(1))
    return oo.e4m3_nearest(np.minimum(a * inv[:, None], 448)).reshape(-1), scale


def follow(store, beta2, n=256, steps=3000):
    """Median of the stored root over the true one, for elements whose gradients become ten times smaller halfway and for
    their neighbours, whose do not."""
    level = 10.0 ** rng(15).uniform(-2, 0, n)
    v, codes, scales = np.zeros(n), np.zeros(n, np.uint8), np.zeros(n // oo.BLOCK, F32)
    for t in range(1, steps + 1):
        small = (np.arange(n) % 2 == 0) & (t >= steps // 2)
        g = (rng(1000 + t).normal(size=n) * level * np.where(small, 0.1, 1.0)).astype(F32)
        v = beta2 * v + (1 - beta2) * g.astype(np.float64) ** 2
        root = oo.load_states(codes, scales)
        codes, scales = store(np.sqrt((root * root) * F32(beta2) + (g * g) * F32(1 - beta2)).astype(F32), t, True)
    ratio = oo.load_states(codes, scales) / np.sqrt(v)
    return [float(np.median(ratio[i::2])) for i in (0, 1)]


@pytest.mark.parametrize("beta2", [0.95, 0.999])
def test_eight_bit_second_moment_follows_its_average(beta2):
    """A stored root is off by a code or two (each an eighth to a sixteenth), unbiased: the median of 128 of them is within
    four of its standard errors, 4 x 1.25 x 0.17 / sqrt(128) = 0.075, and the bias that the square adds, below 0.05."""
    assert all(abs(mid - 1) < 0.125 for mid in follow(oo.store_states, beta2))


def test_rounding_to_the_nearest_code_would_not_follow():
    """A step of a slow average is smaller than half a code, so elements keep their place relative to their block's largest."""
    shrunk, kept = follow(nearest_states, 0.999)
    assert shrunk > 1.25 and kept < 0.8
