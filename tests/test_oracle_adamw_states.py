"""Many steps with 8-bit states beside the same steps with states that are not rounded, in 64 bits: where the values of a
block differ by many octaves, no step may grow beyond what the learning rate allows."""
import numpy as np
import pytest

from oracle import operators as oo

STEPS, N, EPS = 400, 256, 1e-8


def largest_steps(sizes, beta2, spike=None, encode_root=oo.encode_root):
    """Largest |step| / lr of every element over the run: 8-bit states, states as they are."""
    rng = np.random.default_rng(5)
    eight, plain = [np.zeros(N)] * 2, [np.zeros(N)] * 2
    worst = np.zeros((2, N))
    for t in range(1, STEPS + 1):
        g = rng.standard_normal(N) * sizes
        if t == spike:
            g[0] *= 1e7
        for i, state in enumerate((eight, plain)):
            p, m, v = oo.adamw(np.zeros(N), *state, g[None], [1], 0.0, 1.0, 0.9, beta2, EPS, t)
            worst[i] = np.maximum(worst[i], np.abs(p))
            if i == 0:
                r = oo.random_bits(N, 0, t)
                m = oo.decode(*oo.encode(m, 7, (r >> 16) / 65536), 7)
                v = oo.decode(*encode_root(np.sqrt(v), (r & 65535) / 65536), 8) ** 2
            state[:] = [m, v]
    return worst


CASES = [("one element larger", r, b) for r in (1e3, 1e6, 1e7, 1e9) for b in (0.95, 0.999)]
CASES += [("spread", s, b) for s in (1.0, 3.0, 5.0) for b in (0.95, 0.999)] + [("spike", 20, 0.95), ("spike", 20, 0.999)]


def sizes_of(kind, x):
    sizes = np.ones(N)
    if kind == "spread":
        sizes = np.exp(x * np.random.default_rng(6).standard_normal(N))
    elif kind == "one element larger":
        sizes[0] = x
    return sizes


@pytest.mark.parametrize("kind,x,beta2", CASES)
def test_no_step_without_bound(kind, x, beta2):
    """The smallest m that is kept is 2^-18 / 1.875 of the block's largest, the smallest root 2^-19 / 1.9375 of its: of an
    element that keeps both, m / sqrt(v) is up to 2.07 times that of the two largest values.  These are (1 - beta1) /
    sqrt(1 - beta2) = 3.2 at most for one gradient of its own size, and the corrections of the first steps divide m by 1 -
    beta1 at least; 2.07 * 3.2 = 6.6, and codes above the lowest are off by two steps at most: 10 in all."""
    eight, plain = largest_steps(sizes_of(kind, x), beta2, x if kind == "spike" else None)
    assert plain.max() <= 4 and eight.max() <= 10


def test_a_positive_root_has_a_code_and_zero_has_none():
    root = np.zeros(600)
    root[:256:3] = 10.0 ** np.linspace(-30, 0, 86)
    root[300:] = 1e-20
    for u in (0.0, 0.5, 65535 / 65536):
        codes, scales = oo.encode_root(root, np.full(600, u))
        assert np.array_equal(codes > 0, root > 0)
        free, same = oo.encode(root, 8, np.full(600, u))
        assert np.array_equal(scales, same) and np.array_equal(np.maximum(free, root > 0), codes)
    assert not oo.encode_root(np.full(256, 1e-31), np.zeros(256))[0].any()       # (a block that counts as zeros)


def test_without_the_lowest_code_steps_have_no_bound():
    """What the rule is for."""
    eight, _ = largest_steps(sizes_of("one element larger", 1e7), 0.999, encode_root=lambda r, u: oo.encode(r, 8, u))
    assert eight.max() > 1000
