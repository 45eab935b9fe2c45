"""The plain definitions of the 4-bit format and of AdamW against hand-worked numbers and properties (no GPU)."""
import numpy as np
import pytest

from oracle import mx_oracle as mx


def test_nearest_codes_of_every_tie_and_neighbour():
    # a block whose largest is 6 has scale 1: ties between neighbours go to the even code
    ties = [(0.25, 0), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6)]
    for t, code in ties:
        below, above = np.nextafter(np.float32(t), np.float32(0)), np.nextafter(np.float32(t), np.float32(9))
        x = np.zeros((1, 32), np.float32)
        x[0, :5] = [6.0, t, -t, below, above]
        codes, e = mx.quantize(x)
        lo = int(np.searchsorted(mx.E2M1, t)) - 1
        assert e[0, 0] == 127 and list(codes[0, :5]) == [7, code, code + 8, lo, lo + 1], t


def test_scale_is_the_smallest_that_cuts_nothing_off():
    for top, e in ((6.0, 127), (np.nextafter(np.float32(6), np.float32(9)), 128), (3.0, 126), (3.0000002, 127), (4.0, 127), (0.0, 0),
                   (2.0 ** -149, 0), (6 * 2.0 ** -127, 0), (6.1 * 2.0 ** -127, 1), (3.4028234e38, 253)):
        x = np.zeros((1, 32), np.float32)
        x[0, 7] = -top
        assert mx.quantize(x)[1][0, 0] == e, top


def test_layout():
    x = np.arange(2 * 130, dtype=np.float32).reshape(2, 130)
    buf = mx.quantized(x)
    assert buf.size == 2 * 2 * 64 + 2 * 2 * 4   # two rows of two chunks, and their scale words
    v = mx.unpack(buf, 2, 130)
    assert v.shape == (2, 130) and np.abs(v - x).max() <= x.max() / 6
    assert v[0, 128] == 128 and v[1, 2] == 128 and (buf[256:] != 0).sum() == 2 * 5   # blocks 0 to 4 of each row


def test_values_survive_a_second_rounding():
    x = np.random.default_rng(0).standard_normal((5, 200)).astype(np.float32)
    v = mx.unpack(mx.quantized(x), 5, 200)
    again = mx.unpack(mx.quantized(v.astype(np.float32)), 5, 200)
    assert np.array_equal(v, again)


def test_stochastic_rounding_is_right_in_the_mean():
    rng = np.random.default_rng(1)
    x = np.tile(rng.uniform(-6, 6, (1, 32)).astype(np.float32), (4096, 1))
    x[:, 0] = 6.0
    for columns in (False, True):
        X = np.ascontiguousarray(x.T) if columns else x
        v = mx.unpack(mx.quantized(X, mx.STOCHASTIC, 12345, columns), 4096, 32)
        # the mean of 4096 draws, each within the gap of 2 at most: 5 standard deviations of at most 1 / sqrt(4096)
        assert np.abs(v.mean(0) - x[0]).max() <= 5 / 64


def test_bits_of_neighbouring_elements_and_seeds_are_unrelated():
    a, b = mx.draws(64, 512, 7), mx.draws(64, 512, 8)
    for d in (a ^ b, a[:, 1:] ^ a[:, :-1], a[1:] ^ a[:-1], (a >> 16) ^ (a & 0xFFFF)):
        bits = np.unpackbits(d.astype(np.uint32).view(np.uint8)).mean() * (2 if d.max() < 65536 else 1)
        assert abs(bits - 0.5) < 5 * 0.5 / np.sqrt(d.size * (16 if d.max() < 65536 else 32))


def test_adamw_first_step_moves_by_the_learning_rate():
    # from zero states the first step is lr * sign(g) (eps aside) and the decay
    g = np.array([1e-3, -2.0, 5e-6, 0.0], np.float32)
    w = np.array([0.5, -0.5, 1.0, 0.25], np.float32)
    new, m, v, r = mx.adamw(w, g, np.zeros(4, np.float32), np.zeros(4, np.float32), 1, lr=0.01, weight_decay=0.1)
    want = w.astype(np.float64) * (1 - 0.001) - 0.01 * np.sign(g) * np.abs(g) / (np.abs(g) + 1e-8)
    assert np.abs(new - want).max() < 3e-7
    clipped = mx.adamw(np.array([1.0], np.float32), np.array([-1.0], np.float32), np.zeros(1, np.float32), np.zeros(1, np.float32), 1, clip=True)[0]
    assert clipped[0] == 1.0


@pytest.mark.parametrize("t", [1, 2, 3, 1000, 123456])
def test_power(t):
    assert abs(mx.power(0.999, t) / 0.999 ** t - 1) < 1e-10


def test_8_bit_states_follow_a_decaying_gradient():
    """beta2 = 0.999 moves v by less than a code a step; with the random bits it decays as it should, and stays bounded where
    the gradient is steady."""
    rng = np.random.default_rng(2)
    n = 256
    w = np.zeros(n, np.float32)
    m, ms, v, vs = np.zeros(n, np.int8), np.zeros(n // 32, np.uint8), np.zeros(n, np.uint8), np.zeros(n // 32, np.uint8)
    exact = np.zeros(n)
    for step in range(1, 3001):
        g = (rng.standard_normal(n) * (1.0 if step < 1500 else 0.1)).astype(np.float32)
        w, m, ms, v, vs = mx.adamw8(w, g, m, ms, v, vs, step, step * 977, 0)
        exact = 0.999 * exact + 0.001 * g.astype(np.float64) ** 2
    root = mx.adamw_decode(v, vs).astype(np.float64)
    ratio = root / np.sqrt(exact)
    assert 0.9 < np.median(ratio) < 1.1 and ratio.min() > 0.7 and ratio.max() < 1.4
