"""How far the hierarchical attention's operands may be off, as lynx.h states it: the
kernel's roundings to fp16 one by one in numpy, over every code, alpha up to 1e30,
channels of very different sizes and maps whose offset is 0 or cancels."""
import numpy as np
import pytest

from tests.hier_ref import BIASED, CENTRED, INT4, level_table

FORMS = [(BIASED, False), (BIASED, True), (CENTRED, False), (CENTRED, True), (INT4, False)]
ALPHAS = [1e-3, 1.0, 255.0, 1e3, 1e4, 1e6, 1e12, 1e30]


def bound(level, b, m, top):
    """lynx.h's for x = level b + m where the context's largest |b| + |m| is `top`; 1.05
    for products of roundings and fp32."""
    x = level * b + m
    return 1.05 * 2.0 ** -11 * (2 * abs(level * b) + abs(m) + abs(x)) + 2.0 ** -25 * abs(b) + 2.0 ** -36 * top


def f16(x):
    return np.asarray(x, np.float64).astype(np.float16).astype(np.float64)


def rounded(level, b, m, top):
    """x as the kernel makes it: level, b and m rounded, one multiply-add; b and m scaled
    so that the largest |b| + |m| is just below 2^14."""
    s = 2.0 ** (14 - (np.floor(np.log2(top)) + 1))
    return f16(f16(level) * f16(b * s) + f16(m * s)) / s


def maps(kind, g):
    """b and m of 128 channels."""
    b = g.uniform(0.1, 2.0, 128) * np.where(g.random(128) < 0.5, 1, -1)
    if kind == "no offset":
        return b, np.zeros(128)
    if kind == "cancels":
        return b, -b * g.uniform(0, 1, 128)
    b *= 2.0 ** -g.uniform(0, 42, 128)
    return b, g.uniform(-1, 1, 128) * 2.0 ** -g.uniform(0, 42, 128)


@pytest.mark.parametrize("variant,full", FORMS)
@pytest.mark.parametrize("kind", ["no offset", "cancels", "of all sizes"])
@pytest.mark.parametrize("alpha", ALPHAS)
def test_operands_are_inside_the_bound(alpha, kind, variant, full):
    g = np.random.default_rng(5)
    level = level_table(alpha, variant, full).numpy()[:, None]
    for _ in range(20):
        b, m = maps(kind, g)
        top = (abs(b) + abs(m)).max()
        off = abs(rounded(level, b, m, top) - (level * b + m))
        assert (off <= bound(level, b, m, top)).all(), f"{(off / bound(level, b, m, top)).max():.2f} of the bound"


def test_what_the_terms_are_for():
    """Without the level's own term, codes of a large alpha are outside (49 times at 1e6);
    without that of the largest, small channels are."""
    level = level_table(1e6, CENTRED, True).numpy()[:, None]
    b, m = np.array([1.0]), np.array([0.0])
    off = abs(rounded(level, b, m, 1.0) - level * b)
    assert (off > 2.0 ** -11 * 3 * abs(level * b) + 2.0 ** -37).any()
    g = np.random.default_rng(6)
    b, m = maps("of all sizes", g)
    level = level_table(255.0, INT4, False).numpy()[:, None]
    top = (abs(b) + abs(m)).max()
    off = abs(rounded(level, b, m, top) - (level * b + m))
    assert (off > bound(level, b, m, 0.0)).any()
