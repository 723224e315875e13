"""Frequencies of scaled rotary positions, with the defaults that each kind was
published with, against the definitions pair by pair (no GPU)."""
import math

import pytest


@pytest.fixture(scope="module")
def tree():
    from paper_2504_18583_gb300 import _build
    _build.build()
    from paper_2504_18583_gb300 import tree
    return tree


def definition(kind, rot, theta, factor, first, low, high):
    out = []
    for i in range(rot // 2):
        f = theta ** (-2 * i / rot)
        if kind == "parts":
            share = (first * f / (2 * math.pi) - low) / (high - low)
        else:  # the ramp runs over the pair's index, between whole ones
            at = lambda turns: rot * math.log(first / (turns * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
            a, b = max(math.floor(at(high)), 0), min(math.ceil(at(low)), rot - 1)
            share = 1 - (i - a) / max(b - a, 0.001)
        share = min(1.0, max(0.0, share))
        out.append(f * share + f / factor * (1 - share))
    return out


@pytest.mark.parametrize("rot,theta,factor,first", [(128, 500000.0, 8.0, 8192), (64, 10000.0, 4.0, 2048), (32, 1e6, 40.0, 4096)])
@pytest.mark.parametrize("kind,high", [("parts", 4.0), ("yarn", 32.0)])
def test_defaults_are_the_published_ones(tree, kind, high, rot, theta, factor, first):
    got, _ = tree.rope_frequencies(rot, theta, kind, factor, first, device="cpu")
    want = definition(kind, rot, theta, factor, first, 1.0, high)
    assert all(math.isclose(float(x), y, rel_tol=2.0 ** -23) for x, y in zip(got, want))  # rounded once to 32 bits
    given, _ = tree.rope_frequencies(rot, theta, kind, factor, first, 1.5, 20.0, device="cpu")
    want = definition(kind, rot, theta, factor, first, 1.5, 20.0)
    assert all(math.isclose(float(x), y, rel_tol=2.0 ** -23) for x, y in zip(given, want))
