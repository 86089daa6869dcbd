"""What the references of layer_ref.py rest on, on a CPU: the generator's published values, the shares that a dropout keeps, slopes against
differences, a gradient of log probabilities and entropy against differences."""
import os

import numpy as np
import pytest

from tests import layer_ref as ref


def test_philox_is_the_published_one():
    path = os.path.join(os.path.dirname(__file__), "golden", "philox4x32_10_kat.txt")
    lines = [line.split() for line in open(path) if line.strip() and not line.startswith("#")]
    assert lines
    for line in lines:
        v = [int(q, 16) for q in line if all(c in "0123456789abcdefABCDEFxX" for c in q)]
        assert [int(w) for w in ref.philox(v[:4], v[4:6])] == v[6:10]


@pytest.mark.parametrize("p", [0.0, 2.0 ** -17, 0.1, 0.5, 0.9, 1 - 2.0 ** -20])
def test_a_share_of_one_minus_p_stays(p):
    stay, scale = ref.kept(3, 100, 1003, p, 0x123456789abcdef, 5 << 40)
    share = 1 - ref.limit(p) / 65536
    assert abs(stay.mean() - share) <= 5 * np.sqrt(share * (1 - share) / stay.size) and abs(scale * share - 1) < 1e-12
    # neighbours, rows and replicas drawn apart
    a = stay - share
    for q, r in ((a[:, :, 1:], a[:, :, :-1]), (a[:, 1:], a[:, :-1]), (a[1:], a[:-1])):
        assert abs((q * r).mean()) <= 6 * max(share * (1 - share), 1e-9) / np.sqrt(q.size) + 1e-12


@pytest.mark.parametrize("kind", ["none", "gelu", "silu"])
def test_slopes_against_differences(kind):
    z, h = np.linspace(-9, 9, 1001), 1e-5
    assert np.abs((ref.activate(z + h, kind) - ref.activate(z - h, kind)) / (2 * h) - ref.slope(z, kind)).max() < 1e-8


def test_gradient_of_the_scores_against_differences():
    rng = np.random.default_rng(0)
    z, tokens = rng.normal(size=(4, 30)) * 2, rng.integers(-1, 31, size=(4, 3))
    tokens[1, 2] = tokens[1, 0]
    dlogp, dh = rng.normal(size=(4, 3)), rng.normal(size=4)
    value = lambda a: (lambda r: (dlogp * r["logp"]).sum() + (dh * r["entropy"]).sum())(ref.scores(a, tokens, 0))  # noqa: E731
    got = ref.scores_grad(ref.scores(z, tokens, 0), dlogp, dh)
    for at in ((0, 0), (1, 7), (2, 29), (3, 4), (1, int(tokens[1, 0]) % 30)):
        up, down = z.copy(), z.copy()
        up[at] += 1e-5
        down[at] -= 1e-5
        assert abs((value(up) - value(down)) / 2e-5 - got[at]) < 1e-8
