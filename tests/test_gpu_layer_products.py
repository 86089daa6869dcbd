"""The 32-bit products of a layer and its gradient against 64 bits in the norm, where a small product that is left out shows (product_ref.py), on every
route that the layers' tests have."""
import pytest

from paper_2111_08274_amd import hadfl
from tests import layer_ref
from tests import product_ref as ref
from tests.test_gpu_head import _torch
from tests.test_gpu_layers import LAYER, LARGE, ROUTES

pytestmark = pytest.mark.gpu


def _t(a):
    return a.transpose(-1, -2).contiguous()


@pytest.mark.parametrize("n,rows,i,o", LAYER + [q[:4] for q in ROUTES + LARGE if not q[4]])
def test_32_bit_products_lose_what_32_bit_sums_lose(n, rows, i, o):
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(rows + o)
    x, w, dy = (torch.randn(s, device="cuda", generator=g) for s in ((n, rows, i), (n, i, o), (n, rows, o)))
    stay, scale = layer_ref.kept(n, rows, o, 0.5, 1, 2)       # the scale is two: a dropout loses nothing, but dz is formed
    assert scale == 2.0
    half = hadfl.DenseLayer(n, rows, i, o, drop=0.5)
    pairs = [("y", hadfl.DenseLayer(n, rows, i, o, grad=False).forward(x, w), x, w)]
    dz = torch.where(torch.as_tensor(stay).cuda(), 2 * dy, torch.zeros_like(dy))
    for name, z, grads in (("dy as it lies", dy, hadfl.DenseLayer(n, rows, i, o).backward(dy, x, w)), ("dz", dz, half.backward(dy, x, w, seed=1, call=2))):
        pairs += [("dx of " + name, grads[0], z, _t(w)), ("dw of " + name, grads[1], _t(x), z)]
    for name, got, a, b in pairs:
        if got.numel() < 64:
            continue
        off = norm = 0.0
        for k in range(n):
            want = a[k].double() @ b[k].double()
            off, norm = off + float((got[k].double() - want).square().sum()), norm + float(want.square().sum())
        assert off ** 0.5 <= ref.norm_bound(a.shape[2]) * norm ** 0.5, "%s: %.3g of the norm where %.3g is allowed" % (name, (off / norm) ** 0.5, ref.norm_bound(a.shape[2]))
