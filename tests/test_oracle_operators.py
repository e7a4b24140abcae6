"""The plain forms of the norm, the expert sorting and AdamW: gradients against differences, properties that the
formulas promise."""
import numpy as np
import pytest

from oracle import operators as oo


def test_norm_gradient_is_the_derivative():
    rng = np.random.default_rng(1)
    b = [2, 0, 3]
    x, res = rng.standard_normal((5, 7)), rng.standard_normal((5, 7))
    gain, c, d = rng.standard_normal(7), rng.standard_normal((5, 7)), rng.standard_normal((5, 7))

    def loss(x, gain_of_row):
        s = x + res
        rstd = 1 / np.sqrt((s * s).mean(1) + 1e-5)
        return (c * s * rstd[:, None] * gain_of_row).sum() + (d * s).sum()

    s, rstd, _ = oo.rms_norm(x, res, gain, 1e-5)
    dx, dgain = oo.rms_norm_grad(s, rstd, gain, c, d, b)
    h = 1e-6
    for r in range(5):
        for j in range(7):
            e = np.zeros((5, 7))
            e[r, j] = h
            assert abs((loss(x + e, gain) - loss(x - e, gain)) / (2 * h) - dx[r, j]) < 1e-7
    worker = np.repeat([0, 1, 2], b)
    for k in range(3):
        for j in range(7):
            e = np.zeros((5, 7))
            e[worker == k, j] = h
            assert abs((loss(x, gain + e) - loss(x, gain - e)) / (2 * h) - dgain[k, j]) < 1e-7


def test_route_gradient_is_the_derivative():
    rng = np.random.default_rng(2)
    ids = np.array([[0, 2], [2, -1], [-1, -1], [1, 0]])
    offsets, slot, source = oo.route_plan(ids, 3)
    assert offsets.tolist() == [0, 2, 3, 5] and source.tolist() == [0, 7, 6, 1, 2, -1, -1, -1]
    assert slot.tolist() == [[0, 3], [4, -1], [-1, -1], [2, 1]]
    assert oo.route_segments(offsets, source, [1, 3], 2).tolist() == [[0, 1, 2], [2, 2, 3], [3, 4, 5]]
    y, w, c = rng.standard_normal((8, 5)), rng.standard_normal((4, 2)), rng.standard_normal((4, 5))
    loss = lambda y, w: (c * oo.route_combine(y, slot, w, None)).sum()  # noqa: E731
    dy, dw = oo.route_combine_grad(c, y, slot, w)
    h = 1e-6
    for r in range(8):
        for j in range(5):
            e = np.zeros((8, 5))
            e[r, j] = h
            assert abs((loss(y + e, w) - loss(y - e, w)) / (2 * h) - dy[r, j]) < 1e-7
    for t in range(4):
        for j in range(2):
            e = np.zeros((4, 2))
            e[t, j] = h
            assert abs((loss(y, w + e) - loss(y, w - e)) / (2 * h) - dw[t, j]) < 1e-7
    # the way there: <gather(x), z> = <x, combine(z)> with weights of one
    x, z = rng.standard_normal((4, 5)), rng.standard_normal((8, 5))
    assert abs((oo.route_gather(x, slot) * z).sum() - (x * oo.route_combine(z, slot, None, None)).sum()) < 1e-12


@pytest.mark.parametrize("bits", [7, 8])
def test_state_codes_are_monotone_exact_at_zero_and_reach_the_largest(bits):
    table = oo.code_values(bits)
    assert table[0] == 0 and (np.diff(table) > 0).all()
    assert abs(table[-1] - oo.TOPS[bits]) < 2.0 ** -14
    x = table * 3.7
    codes, scales = oo.encode(x, bits, np.full(len(x), 0.5))
    assert np.array_equal(codes & ((1 << bits) - 1), np.arange(len(x)))
    assert np.allclose(oo.decode(codes, scales, bits), x, rtol=1e-3, atol=1e-6)


@pytest.mark.parametrize("bits", [7, 8])
def test_state_rounding_is_unbiased_and_within_a_step(bits):
    rng = np.random.default_rng(3)
    x = np.abs(rng.standard_normal(BLOCKED := 256)) * 10.0 ** rng.uniform(-4, 0, BLOCKED)
    total, n = np.zeros(256), 400
    steps = np.diff(oo.code_values(bits))
    for seed in range(n):
        r = oo.random_bits(256, 5, seed)
        codes, scales = oo.encode(x, bits, (r >> 16 if bits == 7 else r & 65535) / 65536)
        v = oo.decode(codes, scales, bits)
        low = np.clip(np.searchsorted(oo.code_values(bits), x / scales[0], side="right") - 1, 0, len(steps) - 1)
        assert (np.abs(v - x) <= steps[low] * scales[0] * (1 + 1e-9)).all()
        total += v
    # the mean of n roundings is within 5 standard deviations (at most half a step each)
    assert (np.abs(total / n - x) <= 5 * 0.5 / np.sqrt(n) * steps[low] * scales[0]).all()


def test_second_moment_falls_with_unbiased_rounding_and_stays_with_nearest():
    """Why the states are not rounded to nearest: without gradients v has to fall by 1 - beta2 a step."""
    n, steps, beta2 = 256, 300, 0.999
    u = np.random.default_rng(4)
    start = u.uniform(0.5, 1.0, n)
    for unbiased in (True, False):
        codes, scales = oo.encode(np.sqrt(start), 8, np.full(n, 0.5))
        first = (oo.decode(codes, scales, 8) ** 2).mean()
        for _ in range(steps):
            v = beta2 * oo.decode(codes, scales, 8) ** 2
            v[0] = start[0]                      # (one element keeps the block's scale)
            codes, scales = oo.encode(np.sqrt(v), 8, u.random(n) if unbiased else np.full(n, 0.5))
        last = (oo.decode(codes, scales, 8) ** 2).mean()
        if unbiased:
            assert abs(last / first - beta2 ** steps) < 0.05
        else:
            assert last / first > 0.95


def test_random_bits_are_spread():
    r = oo.random_bits(4096, 3, 12345)
    for part in (r >> 16, r & 65535):
        u = part / 65536
        assert abs(u.mean() - 0.5) < 5 * np.sqrt(1 / 12 / 4096)
        assert np.abs(np.histogram(u, 16, (0, 1))[0] - 256).max() < 5 * np.sqrt(256)
    assert abs(np.corrcoef(r >> 16, r & 65535)[0, 1]) < 5 / 64


def test_adamw_is_decoupled_decay_and_adam():
    p, m, v = np.array([1.0, -2.0]), np.zeros(2), np.zeros(2)
    g = np.array([[0.5, 0.0], [9.0, 9.0], [-0.5, 4.0]])
    q, m, v = oo.adamw(p, m, v, g, [3, 0, 1], 0.1, 0.01, 0.9, 0.99, 0.0, 1)
    mean = np.array([0.25, 1.0])
    assert np.allclose(m, 0.1 * mean) and np.allclose(v, 0.01 * mean ** 2)
    assert np.allclose(q, p * (1 - 0.001) - 0.01)      # first step: sign of the gradient
