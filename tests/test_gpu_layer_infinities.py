"""A unit that ReLU has switched off passes nothing on, whatever its gradient holds: max(z, 0) does not depend on z there."""
import numpy as np
import pytest

from paper_2111_08274_amd import hadfl
from tests import layer_ref as ref
from tests.test_gpu_head import _dtype, _torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("drop", [0.0, 0.3])
@pytest.mark.parametrize("rows", [20, 300])
@pytest.mark.parametrize("bf16", [0, 1])
def test_a_unit_that_is_off_has_no_gradient_whatever_dy_holds(bf16, rows, drop):
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(rows)
    n, i, o = 2, 64, 96
    x, w, dy, pre = (torch.randn(s, device="cuda", generator=g).to(_dtype(bf16)) for s in ((n, rows, i), (n, i, o), (n, rows, o), (n, rows, o)))
    pre[:, 1, :8] = 0.0                                       # at zero a unit is off
    plan, kw = hadfl.DenseLayer(n, rows, i, o, bf16=bf16, activation="relu", drop=drop), dict(seed=3, call=4)
    want = plan.backward(dy, x, w, pre=pre, **kw)
    off = pre <= 0
    for bad in (float("inf"), float("-inf"), float("nan")):
        got = plan.backward(torch.where(off, torch.full_like(dy, bad), dy), x, w, pre=pre, **kw)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    # where it is on, an infinity stays one, and a NaN before the activation stays a NaN
    stay = torch.as_tensor(ref.kept(n, rows, o, drop, 3, 4)[0] if drop else np.ones((n, rows, o), bool)).cuda()
    t, j = [int(q) for q in (~off & stay)[1].nonzero()[5]]
    dy[1, t, j] = float("inf")
    assert plan.backward(dy, x, w, pre=pre, want=("db",), **kw)[2][1, j] == float("inf")
    pre[1, t, j] = float("nan")
    db = plan.backward(dy, x, w, pre=pre, want=("db",), **kw)[2]
    assert torch.isnan(db[1, j]) and int(torch.isnan(db).sum()) == 1
