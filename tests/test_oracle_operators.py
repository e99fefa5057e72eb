"""Pins of the oracle of the 4-bit microscaled format and of AdamW (no GPU)."""
import numpy as np
import pytest

from oracle import adamw, mx4, ref


def test_random_blocks_are_the_librarys_generator():
    seed, epoch, purpose = 0x123456789ABCDEF0, 77, 6
    blocks = np.array([0, 1, 5, 2 ** 32 - 1, 2 ** 32, 2 ** 40 + 3], np.uint64)
    got = mx4.philox_blocks(blocks, epoch, purpose, seed)
    for b, w in zip(blocks, got):
        want = ref.philox4x32_10([int(b) & 0xFFFFFFFF, int(b) >> 32, epoch, purpose], [seed & 0xFFFFFFFF, seed >> 32])
        assert [int(x) for x in want] == [int(x) for x in w]


def test_numbers_of_the_grid_stay_and_ties_go_to_the_even_code():
    x = np.zeros((1, 32))
    x[0, :8] = mx4.GRID
    x[0, 8:15] = (mx4.GRID[1:] + mx4.GRID[:-1]) / 2
    x[0, 15:22] = -x[0, 8:15]
    codes, scales = mx4.quantize(x)
    assert scales[0, 0] == 127
    assert list(codes[0, :8]) == list(range(8))
    assert list(codes[0, 8:15]) == [0, 2, 2, 4, 4, 6, 6]
    assert list(codes[0, 15:22]) == [8, 10, 10, 12, 12, 14, 14]
    assert np.array_equal(mx4.values(codes, scales)[0, :8], mx4.GRID)


@pytest.mark.parametrize("most,s", [(6.0, 127), (np.nextafter(6.0, 7), 128), (3.0, 126), (3.1, 127), (2.0 ** -140, 0),
                                    (float(np.finfo(np.float32).max), 253), (np.inf, 255), (np.nan, 255), (0.0, 0)])
def test_the_scale_is_the_smallest_that_clamps_nothing(most, s):
    x = np.zeros((1, 32))
    x[0, 3] = most
    codes, scales = mx4.quantize(x)
    assert scales[0, 0] == s
    if s < 255:
        assert abs(mx4.values(codes, scales)[0, 3] - most) <= 2.0 ** (s - 127)


def test_packing_is_undone():
    c = np.random.default_rng(0).integers(0, 16, (3, 128)).astype(np.uint8)
    assert np.array_equal(mx4.unpack(mx4.pack(c)), c)
    assert mx4.pack(c)[1, 5] == c[1, 10] + 16 * c[1, 11]


def test_stochastic_rounding_is_unbiased():
    """The mean over n draws of a value between two numbers a step apart has a standard deviation of at most
    step / (2 sqrt n), and the rule is unbiased to 1 / 512 of the step: six deviations and that."""
    x = np.full((1, 32), 6.0)
    x[0, 1:8] = [0.1, 0.6, 1.3, 1.9, 2.2, 3.7, 5.0]
    n = 2000
    mean = sum(mx4.values(*mx4.quantize(x, True, epoch=e, seed=9))[0] for e in range(n)) / n
    step = np.array([0.5, 0.5, 0.5, 0.5, 1, 1, 2])
    assert np.all(np.abs(mean[1:8] - x[0, 1:8]) <= step * (6 * 0.5 / np.sqrt(n) + 1 / 512))
    assert mean[0] == 6.0 and np.all(mean[8:32] == 6.0)


def test_state_formats_hold_their_numbers_whatever_the_draw():
    for kind, codes in (("m", np.arange(0, 127)), ("v", np.arange(0, 248))):
        n = adamw.numbers(kind)[codes]
        for c0 in range(0, len(codes), 31):
            x = np.zeros(32, np.float32)
            x[0] = adamw.FORMATS[kind][1]  # keeps the scale at one
            part = codes[c0:c0 + 31]
            x[1:1 + len(part)] = n[c0:c0 + 31]
            for u in (0, 65535):
                got, s = adamw.write(x, np.full(32, u), kind)
                assert s[0] == 127 and list(got[1:1 + len(part)]) == list(part)


@pytest.mark.parametrize("kind", ["m", "v"])
def test_state_rounding_is_unbiased(kind):
    rng = np.random.default_rng(3)
    x = np.exp(rng.uniform(-14, 0, 32)).astype(np.float32)
    n = 4000
    got = np.zeros((n, 32))
    for k in range(n):
        got[k] = adamw.read(*adamw.write(x, rng.integers(0, 65536, 32), kind), kind)
    step = np.maximum(x / 8, x.max() * 2.0 ** -15 if kind == "m" else 0)  # a step is at most x / 8, or the least one
    assert np.all(np.abs(got.mean(0) - x) <= step * (6 * 0.5 / np.sqrt(n) + 2.0 ** -16))


def test_a_first_step_moves_by_the_learning_rate():
    """m / sqrt(v) after the first step is the sign of the gradient, whatever its size."""
    g = np.array([1e-3, -5.0, 2e4])
    p, m, v = adamw.step(np.zeros(3), g, np.zeros(3), np.zeros(3), 1, 1e-2, 0.9, 0.999, 1e-12, 0.0)
    assert np.allclose(p, -1e-2 * np.sign(g), rtol=1e-8)
