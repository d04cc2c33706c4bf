"""The oracle of the gated layer and of activations kept in 8 bits, pinned on its own (no GPU)."""
import numpy as np
import pytest

from oracle import surroundings_oracle as oo

ACTS = ("silu", "gelu", "relu")


def rng(seed):
    return np.random.default_rng(seed)


def test_activations_by_hand():
    assert np.allclose(oo.activation([0.0, 1.0, -1.0], "silu")[0], [0.0, 0.7310585786300049, -0.2689414213699951])
    assert np.allclose(oo.activation([0.0, 1.0, -1.0, 30.0], "gelu")[0], [0.0, 0.8411919906082768, -0.15880800939172324, 30.0])
    a, d = oo.activation([-2.0, 0.0, 3.0], "relu")
    assert a.tolist() == [0.0, 0.0, 3.0] and d.tolist() == [0.0, 0.0, 1.0]


@pytest.mark.parametrize("act", ACTS)
def test_gradient_against_differences(act):
    gu, dh = rng(1).normal(size=(5, 16)) * 2, rng(2).normal(size=(5, 8))
    gu[np.abs(gu) < 1e-3] = 1.0                                             # away from relu's corner
    dgu, h = oo.gated_grad(dh, gu, act)
    assert np.allclose(h, oo.gated(gu, act), rtol=1e-14, atol=0)
    step = 1e-5
    for j in range(16):
        up, down = gu.copy(), gu.copy()
        up[:, j] += step
        down[:, j] -= step
        slope = ((oo.gated(up, act) - oo.gated(down, act)) * dh).sum(1) / (2 * step)
        assert np.allclose(dgu[:, j], slope, rtol=1e-7, atol=1e-8)


def test_blocks_by_hand():
    x = np.zeros((1, 72))
    x[0, 0], x[0, 1], x[0, 31] = 448.0, -1.0, 2.0 ** -9                      # scale 1
    x[0, 32] = 449.0                                                        # scale 2
    x[0, 64], x[0, 71] = 1.75, 0.25                                         # a short block: 1.75 = 448 2^-8
    codes, bytes_ = oo.checkpoint(x)
    assert bytes_.tolist() == [[127, 128, 119]]
    assert codes[0, 0] == 0x7E and codes[0, 1] == 0xB8 and codes[0, 31] == 1 and codes[0, 64] == 0x7E
    back = oo.restored(codes, bytes_)
    assert back[0, 0] == 448 and back[0, 32] == 448 and back[0, 71] == 0.25 and back.shape == x.shape


def test_blocks_at_the_ends_of_the_range():
    x = np.zeros((4, 32))
    x[1, 3] = 2.0 ** -133                                                   # bf16's smallest
    x[2, 0] = 3.3895313892515355e38                                         # bf16's largest, 255 2^120
    x[3, 5] = np.inf
    codes, bytes_ = oo.checkpoint(x)
    assert bytes_[:, 0].tolist() == [1, 1, 247, 255]
    back = oo.restored(codes, bytes_)
    assert (back[0] == 0).all() and back[1, 3] == 2.0 ** -133 and np.isnan(back[3]).all() and abs(back[2, 0] / x[2, 0] - 1) <= 2.0 ** -4


def test_blocks_round_to_half_a_step_and_keep_what_they_hold():
    x = rng(3).normal(size=(40, 200)) * np.exp(3 * rng(4).normal(size=(40, 200)))
    codes, bytes_ = oo.checkpoint(x)
    back, scale = oo.restored(codes, bytes_), np.repeat(2.0 ** (bytes_ - 127.0), 32, axis=1)[:, :200]
    assert (np.abs(back - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * scale)).all()
    again = oo.checkpoint(back)
    assert (oo.restored(*again) == back).all()
    # a power of two changes nothing but the bytes
    assert (oo.checkpoint(x * 64)[0] == codes).all() and (oo.checkpoint(x * 64)[1] == bytes_ + 6).all()
