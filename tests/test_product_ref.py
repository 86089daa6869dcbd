"""The bound that the GPU's 32-bit products are held to rejects products of fewer parts, at every contraction that the GPU tests have."""
import numpy as np
import pytest

from tests import product_ref as ref
from tests.test_gpu_layers import LAYER, LARGE, ROUTES

LENGTHS = sorted({k for q in LAYER + [q[:4] for q in ROUTES + LARGE if not q[4]] for k in q[1:]})


@pytest.mark.parametrize("k", LENGTHS)
def test_the_bound_sees_every_product_that_is_left_out(k):
    rng = np.random.default_rng(k)
    x, w = rng.normal(size=(48, k)).astype(np.float32), rng.normal(size=(k, 48)).astype(np.float32)
    want = x.astype(np.float64) @ w.astype(np.float64)
    assert ref.off(ref.product(x, w), want) < 2.0 ** -25      # six products lose nothing that 32 bits hold
    three = [p for p in ref.PAIRS if sum(p) < 2]
    for pairs in (three, three[:1]):
        assert ref.off(ref.product(x, w, pairs), want) > 1.2 * ref.norm_bound(k), (k, pairs)
    if k <= 5000:                                             # one of the small products is 2.5e-6 of the norm, the bound 2.34e-6 at 5000
        for gone in ref.PAIRS[3:]:
            assert ref.off(ref.product(x, w, [p for p in ref.PAIRS if p != gone]), want) > ref.norm_bound(k), (k, gone)


def test_a_sum_in_32_bits_stays_within_it():
    # six products of sixteen terms each added to one 32-bit sum, as the kernels do
    rng = np.random.default_rng(0)
    for k in (64, 512, 4096):
        x, w = rng.normal(size=(24, k)).astype(np.float32), rng.normal(size=(k, 24)).astype(np.float32)
        a, b = ref.parts(x), ref.parts(w)
        acc = np.zeros((24, 24), np.float32)
        for s in range(0, k, 16):
            for i, j in reversed(ref.PAIRS):
                acc += (a[i][:, s:s + 16] @ b[j][s:s + 16]).astype(np.float32)
        assert ref.off(acc.astype(np.float64), x.astype(np.float64) @ w.astype(np.float64)) <= ref.norm_bound(k), k
