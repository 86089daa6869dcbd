"""What a bf16 layer's gradient loses: its outputs' rounding and what a 32-bit sum loses, also where dz is no bf16 value (a curved activation, a
dropout's scale).  dz enters the products in two parts, the first cut off after eight significant bits, the second rounded to eight: off by
2^-7 2^-8 = 2^-15 of a value at most."""
import numpy as np
import pytest

from paper_2111_08274_amd import hadfl
from tests import layer_ref as ref
from tests.test_gpu_head import _check, _out, _torch, _values
from tests.test_gpu_layers import CALL, LAYER, LAYOUTS, LARGE, ROUTES, SEED, _layer_case

pytestmark = pytest.mark.gpu
TWO_PARTS = 2.0 ** -15


def _grad(dy, pre, x, w, kind, p, seed, call):
    """-> dx, dw and bounds: those of a 32-bit gradient, two parts' loss, an output's rounding"""
    want, bound = ref.layer_grad(dy, pre, x, w, kind, p, seed, call, 0)
    dz = np.abs((ref.dropped(dy, p, seed, call) if p else dy) * (ref.slope(pre, kind) if kind != "none" else 1.0))
    t = lambda a: np.swapaxes(a, -1, -2)  # noqa: E731
    for name, terms in (("dx", np.matmul(dz, np.abs(t(w)))), ("dw", np.matmul(np.abs(t(x)), dz))):
        bound[name] = bound[name] + TWO_PARTS * terms
        bound[name] = bound[name] + ref.HALF_BF16 * (np.abs(want[name]) + bound[name])
    return want, bound


def _check_grad(n, rows, i, o, layout, kind, p, seed):
    c = _layer_case(n, rows, i, o, 1, layout, seed)
    plan = hadfl.DenseLayer(n, rows, i, o, bf16=1, activation=kind, drop=p)
    dx, dw, db = _out((n, rows, i), 1, layout), _out((n, i, o), 1, layout), _out((n, o), 0, layout)
    plan.backward(c["dy"], c["x"], c["w"], pre=c["pre"], dx=dx.t, dw=dw.t, db=db.t, seed=SEED, call=CALL)
    h = {k: _values(v) for k, v in c.items()}
    want, bound = _grad(h["dy"], h["pre"], h["x"], h["w"], kind, p, SEED, CALL)
    for name, got in (("db", db), ("dx", dx), ("dw", dw)):
        _check(got.get(), want[name], bound[name], name)
        assert got.untouched(), name


@pytest.mark.parametrize("n,rows,i,o", LAYER)
def test_a_bf16_gradient_is_as_exact_as_its_outputs(n, rows, i, o):
    at = LAYER.index((n, rows, i, o))
    for kind, p in (("gelu", 0.2), ("silu", 0.0), ("none", 0.1)):
        _check_grad(n, rows, i, o, LAYOUTS[at % 3], kind, p, at)


@pytest.mark.parametrize("n,rows,i,o", [q[:4] for q in ROUTES if q[4]])
def test_a_bf16_gradient_is_as_exact_on_every_route(n, rows, i, o):
    at = [q[:4] for q in ROUTES].index((n, rows, i, o))
    _check_grad(n, rows, i, o, LAYOUTS[at % 2 * 2], *(("gelu", 0.0), ("silu", 0.1))[at % 2], seed=at)


@pytest.mark.parametrize("n,rows,i,o", [q[:4] for q in LARGE if q[4]])
def test_a_large_bf16_gradient_is_as_exact(n, rows, i, o):
    # 64 rows of dx and dw against 64 bits on the device: values, slopes and kept ones as the kernel is given them
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(o)
    x, w, dy, pre = (torch.randn(s, device="cuda", generator=g).bfloat16() for s in ((n, rows, i), (n, i, o), (n, rows, o), (n, rows, o)))
    dx, dw, _ = hadfl.DenseLayer(n, rows, i, o, bf16=1, activation="silu").backward(dy, x, w, pre=pre)

    def check(got, a, b, name):
        want, terms = a @ b.contiguous(), a.abs() @ b.abs().contiguous()
        # 32 roundings of a slope, a sum's, two parts
        err = (32 + a.shape[1] + 16) * ref.EPS32 * terms + TWO_PARTS * terms
        assert bool(((got.double() - want).abs() <= err + ref.HALF_BF16 * (want.abs() + err)).all()), name

    for k in (0, n - 1):
        z = pre[k].double()
        s = torch.sigmoid(z)
        dz = dy[k].double() * (s + z * s * torch.sigmoid(-z))
        some = torch.randint(0, rows, (64,), device="cuda", generator=g)
        some[0], some[1] = 0, rows - 1
        check(dx[k, some], dz[some], w[k].double().t(), "dx")
        some = torch.randint(0, i, (64,), device="cuda", generator=g)
        some[0], some[1] = 0, i - 1
        check(dw[k, some], x[k][:, some].double().t(), dz, "dw")


@pytest.mark.parametrize("rows", [20, 300])
def test_infinite_operands_of_a_bf16_gradient(rows):
    # an infinity times a value that is not zero is an infinity, in the parts' products too; also of a dz that is a bf16 value (the slope is one), that is
    # infinite itself, or larger than bf16's largest finite value
    torch = _torch()
    n, i, o = 1, 40, 72
    dy = torch.full((n, rows, o), 0.375, device="cuda").bfloat16()
    pre = torch.full((n, rows, o), 20.0, device="cuda").bfloat16()
    pre[:, :, ::3] = 0.7
    x, w = torch.ones((n, rows, i), device="cuda").bfloat16(), torch.ones((n, i, o), device="cuda").bfloat16()
    x[0, rows // 2, 5] = float("inf")
    x[0, rows // 2, 6] = float("-inf")
    w[0, 7, o // 2] = float("-inf")
    w[0, 8, 0] = float("inf")
    plan = hadfl.DenseLayer(n, rows, i, o, bf16=1, activation="gelu")
    dx, dw, _ = plan.backward(dy, x, w, pre=pre)
    for got, at, sign in ((dw[0], 5, 1), (dw[0], 6, -1), (dx[0].t(), 7, -1), (dx[0].t(), 8, 1)):
        assert bool((got[at] == sign * float("inf")).all())
    assert bool(torch.isfinite(dw[0, [j for j in range(i) if j not in (5, 6)]]).all())
    assert bool(torch.isfinite(dx[0][:, [j for j in range(i) if j not in (7, 8)]]).all())
    for value in (float("inf"), 3.3e38):                       # 3.3e38 times 65536 / (65536 - t) is beyond every finite value
        dy = torch.ones((n, rows, o), device="cuda").bfloat16()
        dy[0, 3, 4] = value
        plan = hadfl.DenseLayer(n, rows, i, o, bf16=1, activation="silu", drop=0.2)
        call = next(c for c in range(50) if ref.kept(n, rows, o, 0.2, 0, c)[0][0, 3, 4])
        dx, dw, db = plan.backward(dy, x.clamp(-1, 1), w.clamp(-1, 1).abs(), pre=pre, call=call)
        assert bool((dx[0, 3] == float("inf")).all()) and bool((dw[0, :5, 4] == float("inf")).all()) and db[0, 4] == float("inf")
        assert bool(torch.isfinite(dx[0, :3]).all()) and bool(torch.isfinite(dw[0, :, 5:]).all())


@pytest.mark.parametrize("rows", [20, 300])
def test_small_and_large_magnitudes_of_a_bf16_gradient(rows):
    # the second part is no smaller than a normal number, the first no larger than the largest: bounds as everywhere
    n, i, o = 2, 96, 136
    for e, f in ((-100, 80), (90, -70)):
        c = _layer_case(n, rows, i, o, 1, "whole", seed=7)
        dy, x, w = c["dy"] * 2.0 ** e, c["x"] * 2.0 ** f, c["w"] * 2.0 ** f
        dx, dw, db = hadfl.DenseLayer(n, rows, i, o, bf16=1, activation="silu", drop=0.1).backward(dy, x, w, pre=c["pre"], seed=SEED, call=CALL)
        want, bound = _grad(_values(dy), _values(c["pre"]), _values(x), _values(w), "silu", 0.1, SEED, CALL)
        for name, got in (("db", db), ("dx", dx), ("dw", dw)):
            _check(_values(got), want[name], bound[name], name)


def test_a_bf16_gradient_of_no_rows_repeats_and_of_each_alone():
    torch = _torch()
    for i, o in ((96, 136), (3, 136), (96, 5), (512, 2048)):
        plan = hadfl.DenseLayer(2, 0, i, o, bf16=1, activation="gelu", drop=0.2)
        t = lambda *s: torch.randn(s, device="cuda").bfloat16()  # noqa: E731
        dx, dw, db = plan.backward(t(2, 0, o), t(2, 0, i), t(2, i, o), pre=t(2, 0, o))
        assert dx.shape == (2, 0, i) and not dw.any() and not db.any()
        for rows in (1, 40, 300):
            c = _layer_case(2, rows, i, o, 1, "odd", seed=3)
            plan = hadfl.DenseLayer(2, rows, i, o, bf16=1, activation="gelu", drop=0.2)
            whole = plan.backward(c["dy"], c["x"], c["w"], pre=c["pre"], seed=1)
            for k, name in enumerate(("dx", "dw", "db")):
                got = plan.backward(c["dy"], c["x"] if name == "dw" else None, c["w"] if name == "dx" else None, pre=c["pre"], want=(name,), seed=1)
                assert torch.equal(got[k], whole[k])
