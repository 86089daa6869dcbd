"""A dense layer with its epilogue, dropout and the scores of tokens on the GPU against the same in 64 bits (layer_ref.py).  Tensors lie inside
larger buffers as in test_gpu_head.py: inputs between NaNs, outputs between marks that must survive."""
import numpy as np
import pytest

from paper_2111_08274_amd import hadfl
from tests import layer_ref as ref
from tests.test_gpu_head import _check, _dtype, _in, _out, _torch, _values

pytestmark = pytest.mark.gpu
SEED, CALL = 0xfedcba9876543210, (3 << 32) + 5
LAYOUTS = ["whole", "padded", "odd"]


def _counter(value):
    return _torch().tensor([value], dtype=_torch().int64, device="cuda")


# ---- dropout ---------------------------------------------------------------------------------------------------------
DROP = [(1, 1, 1), (1, 1, 512), (2, 3, 7), (3, 17, 33), (2, 40, 128), (2, 5, 1111), (1, 70, 2056), (5, 300, 64), (1030 // 2, 3, 24)]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("bf16", [0, 1])
@pytest.mark.parametrize("n,rows,cols", DROP)
def test_dropout_and_its_gradient(n, rows, cols, bf16, layout):
    # kept values times the scale: one rounding, one more for the residual, and the output's; dropped ones are zero exactly
    rng = np.random.default_rng(n + cols)
    x, r = _in(rng.normal(size=(n, rows, cols)), bf16, layout), _in(rng.normal(size=(n, rows, cols)), bf16, layout)
    half = ref.HALF_BF16 if bf16 else ref.EPS32
    for p in (0.0, 0.1, 0.9):
        plan = hadfl.Dropout(n, rows, cols, p, bf16=bf16)
        want = ref.dropped(_values(x), p, SEED, CALL + 2) if p else _values(x)
        y = _out((n, rows, cols), bf16, layout)
        plan.forward(x, y=y.t, seed=SEED, call=CALL, counter=_counter(2))
        _check(y.get(), want, (half + ref.EPS32) * np.abs(want), "y")
        assert y.untouched() and bool((y.t[_torch().as_tensor(want == 0).cuda()] == 0).all())
        dx = _out((n, rows, cols), bf16, layout)
        plan.backward(x, dx=dx.t, seed=SEED, call=CALL + 2)
        assert _torch().equal(dx.t, y.t) and dx.untouched()
        plan.forward(x, residual=r, y=y.t, seed=SEED, call=CALL + 1, counter=_counter(1))
        want = want + _values(r)
        _check(y.get(), want, half * np.abs(want) + 4 * ref.EPS32 * (np.abs(want) + 2 * np.abs(_values(r))), "y with a residual")
        assert y.untouched()


def test_dropout_in_place_without_rows_and_of_masked_values():
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(0)
    for bf16 in (0, 1):
        x, r = (torch.randn((2, 30, 41), device="cuda", generator=g).to(_dtype(bf16)) for _ in range(2))
        plan = hadfl.Dropout(2, 30, 41, 0.3, bf16=bf16)
        want = plan.forward(x, residual=r, seed=1, call=2)
        for mine in (0, 1):
            a, b = x.clone(), r.clone()
            assert torch.equal(plan.forward(a, residual=b, y=(a, b)[mine], seed=1, call=2), want)
        stay = torch.as_tensor(ref.kept(2, 30, 41, 0.3, 1, 2)[0]).cuda()
        bad = torch.where(stay, x, torch.full_like(x, float("nan")))       # a dropped value is zero whatever it holds
        assert torch.equal(plan.forward(bad, residual=r, seed=1, call=2), want)
        bad = torch.where(stay, torch.full_like(x, float("inf")), torch.full_like(x, float("-inf")))
        assert torch.equal(torch.isinf(plan.forward(bad, seed=1, call=2)), stay)
        assert hadfl.Dropout(2, 0, 41, 0.3, bf16=bf16).forward(x[:, :0]).shape == (2, 0, 41)
        one = x[:1, :1].expand(2, 30, 41)                                  # one row for all
        assert torch.equal(plan.forward(one, seed=1, call=2), plan.forward(one.contiguous(), seed=1, call=2))
        # other seeds, calls and replicas drop others
        same = [plan.forward(torch.ones_like(x), seed=s, call=c) for s, c in ((1, 2), (1, 3), (2, 2), (1, 2 + (1 << 32)), (1 + (1 << 32), 2))]
        assert all(not torch.equal(same[0], q) for q in same[1:]) and not torch.equal(same[0][0], same[0][1])


@pytest.mark.parametrize("p,limit", [(2.0 ** -18, 0), (2.0 ** -16, 1), (1 - 2.0 ** -16, 65535), (1 - 2.0 ** -24, 65535)])
def test_probabilities_at_the_ends_of_their_range(p, limit):
    torch = _torch()
    assert ref.limit(p) == limit
    x = torch.ones((1, 512, 2048), device="cuda")
    got = hadfl.Dropout(1, 512, 2048, p).forward(x, seed=4, call=9).cpu().numpy()
    stay, scale = ref.kept(1, 512, 2048, p, 4, 9)
    assert np.array_equal(got, np.where(stay, np.float32(scale), np.float32(0)))


# ---- dense layer -----------------------------------------------------------------------------------------------------
LAYER = [(1, 1, 1, 1), (1, 1, 512, 2048), (2, 3, 5, 40), (3, 33, 40, 9), (2, 17, 9, 130), (2, 64, 130, 257), (4, 32, 784, 128), (1, 5, 2048, 72), (1, 40, 2056, 130),
         (1, 65, 64, 96), (2, 200, 333, 519), (2, 300, 40, 7), (1, 700, 520, 264), (1, 300, 2048, 130), (16, 1024, 72, 768), (2, 520, 1096, 9)]
# sizes, with the type, that between them take every tile, through registers and in planes, in one share and in several
ROUTES = [(4, 4624, 8, 10, 1), (8, 71, 5672, 9, 1), (3, 8, 1919, 1049, 1), (16, 39, 9, 3984, 0), (32, 149, 8, 1712, 1), (1, 4120, 3131, 8, 1), (32, 33, 3701, 72, 0),
          (8, 3648, 129, 67, 0), (4, 96, 1117, 800, 0), (3, 8, 4456, 917, 1), (4, 8056, 66, 72, 0), (4, 168, 6064, 176, 1), (2, 928, 78, 2128, 0), (3, 2096, 1992, 72, 1),
          (8, 86, 280, 5048, 1), (1, 2890, 3030, 142, 1), (3, 1830, 71, 2097, 1), (4, 2392, 207, 1349, 0), (1, 135, 5672, 4296, 1), (2, 4288, 2744, 175, 1),
          (8, 8, 212, 3288, 1), (8, 8, 3288, 212, 1), (32, 23, 265, 288, 0), (4, 61, 300, 600, 1), (2, 50, 1000, 90, 0)]
# and the largest tiles in several shares, some rows of whose results are looked at
LARGE = [(1, 4096, 512, 4096, 0), (1, 2048, 16384, 1000, 1), (1, 2048, 1000, 16384, 1), (2, 16384, 1000, 1000, 1), (4, 16384, 1000, 1000, 1), (1, 4096, 1000, 16384, 1),
         (1, 4096, 16384, 1000, 1), (1, 6000, 4096, 3000, 0)]
OPTIONS = [("none", 0.0, False, False), ("relu", 0.0, True, False), ("gelu", 0.2, True, True), ("silu", 0.1, False, True), ("none", 0.1, True, True)]


def _layer_case(n, rows, i, o, bf16, layout, seed=0):
    rng = np.random.default_rng(seed)
    return dict(x=_in(rng.normal(size=(n, rows, i)), bf16, layout), w=_in(rng.normal(size=(n, i, o)) / np.sqrt(i), bf16, layout),
                bias=_in(rng.normal(size=(n, o)), 0, layout), residual=_in(rng.normal(size=(n, rows, o)), bf16, layout),
                dy=_in(rng.normal(size=(n, rows, o)), bf16, layout), pre=_in(rng.normal(size=(n, rows, o)) * 2, bf16, layout))


def _check_layer(n, rows, i, o, bf16, layout, options, seed=0):
    kind, p, bias, residual = options
    c = _layer_case(n, rows, i, o, bf16, layout, seed)
    plan = hadfl.DenseLayer(n, rows, i, o, bf16=bf16, activation=kind, drop=p)
    y, pre = _out((n, rows, o), bf16, layout), _out((n, rows, o), bf16, layout)
    b, r = c["bias"] if bias else None, c["residual"] if residual else None
    plan.forward(c["x"], c["w"], b, residual=r, pre=pre.t, y=y.t, seed=SEED, call=CALL, counter=_counter(-3))
    h = {k: _values(v) for k, v in c.items()}
    want, bound = ref.layer(h["x"], h["w"], h["bias"] if bias else None, h["residual"] if residual else None, kind, p, SEED, CALL - 3, bf16)
    _check(pre.get(), want["pre"], bound["pre"], "pre")
    _check(y.get(), want["y"], bound["y"], "y")
    assert y.untouched() and pre.untouched()
    # without room for a gradient, without pre: the same y
    alone = hadfl.DenseLayer(n, rows, i, o, bf16=bf16, activation=kind, drop=p, grad=False)
    assert _torch().equal(alone.forward(c["x"], c["w"], b, residual=r, seed=SEED, call=CALL - 3), y.t)
    dx, dw, db = _out((n, rows, i), bf16, layout), _out((n, i, o), bf16, layout), _out((n, o), 0, layout)
    plan.backward(c["dy"], c["x"], c["w"], pre=c["pre"], dx=dx.t, dw=dw.t, db=db.t, seed=SEED, call=CALL, counter=_counter(-3))
    want, bound = ref.layer_grad(h["dy"], h["pre"], h["x"], h["w"], kind, p, SEED, CALL - 3, bf16)
    for name, got in (("db", db), ("dx", dx), ("dw", dw)):
        _check(got.get(), want[name], bound[name], name)
        assert got.untouched(), name


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("bf16", [0, 1])
@pytest.mark.parametrize("n,rows,i,o", LAYER)
def test_dense_layer_and_its_gradient(n, rows, i, o, bf16, layout):
    at = LAYER.index((n, rows, i, o)) + LAYOUTS.index(layout)
    _check_layer(n, rows, i, o, bf16, layout, OPTIONS[at % len(OPTIONS)])


@pytest.mark.parametrize("n,rows,i,o,bf16", ROUTES)
def test_dense_layer_on_every_route(n, rows, i, o, bf16):
    at = ROUTES.index((n, rows, i, o, bf16))
    _check_layer(n, rows, i, o, bf16, LAYOUTS[at % 2 * 2], OPTIONS[at % len(OPTIONS)], seed=at)


@pytest.mark.parametrize("n,rows,i,o,bf16", LARGE)
def test_large_layers(n, rows, i, o, bf16):
    # 64 rows of y, dx and dw, the first and last among them, against 64 bits on the device; bounds as everywhere
    torch = _torch()
    t = _dtype(bf16)
    g = torch.Generator(device="cuda").manual_seed(i)
    x, w, dy, pre = (torch.randn(s, device="cuda", generator=g).to(t) for s in ((n, rows, i), (n, i, o), (n, rows, o), (n, rows, o)))
    plan = hadfl.DenseLayer(n, rows, i, o, bf16=bf16, activation="relu")
    y = plan.forward(x, w)
    dx, dw, db = plan.backward(dy, x, w, pre=pre)
    half = ref.HALF_BF16 if bf16 else ref.EPS32

    def check(got, a, b, name, relu=False):
        want, terms = a.double() @ b.double().contiguous(), a.double().abs() @ b.double().abs().contiguous()
        err = (a.shape[1] + 16) * ref.EPS32 * terms
        want = want.clamp(min=0) if relu else want
        assert bool(((got.double() - want).abs() <= err + half * (want.abs() + err)).all()), name

    for k in (0, n - 1):
        some = torch.randint(0, rows, (64,), device="cuda", generator=g)
        some[0], some[1] = 0, rows - 1
        z = torch.where(pre[k] > 0, dy[k], torch.zeros_like(dy[k]))
        check(y[k, some], x[k, some], w[k], "y", relu=True)
        check(dx[k, some], z[some], w[k].t(), "dx")
        some = torch.randint(0, i, (64,), device="cuda", generator=g)
        some[0], some[1] = 0, i - 1
        check(dw[k, some], x[k][:, some].t(), z, "dw")
        want, terms = z.double().sum(0), z.double().abs().sum(0)
        assert bool(((db[k].double() - want).abs() <= (rows + 16) * ref.EPS32 * terms).all())


@pytest.mark.parametrize("options", OPTIONS)
@pytest.mark.parametrize("n,rows,i,o,bf16", [(2, 20, 72, 136, 0), (2, 20, 72, 136, 1), (2, 100, 72, 136, 0), (2, 100, 72, 136, 1)])
def test_what_follows_the_product(n, rows, i, o, bf16, options):
    _check_layer(n, rows, i, o, bf16, "whole", options, seed=1)


@pytest.mark.parametrize("n,rows,i,o", [(2, 5, 40, 72), (2, 100, 130, 72), (1, 600, 96, 1030), (1, 3, 1, 3)])
@pytest.mark.parametrize("bf16", [0, 1])
def test_gradient_from_a_checkpoint(n, rows, i, o, bf16):
    from tests import head_ref
    c = _layer_case(n, rows, i, o, bf16, "odd", seed=2)
    plan, kept = hadfl.DenseLayer(n, rows, i, o, bf16=bf16, activation="relu"), hadfl.PackedRows(n, rows, i, bf16=bf16).pack(c["x"])
    dx, dw, db = plan.backward(c["dy"], kept, c["w"], pre=c["pre"])
    h = {k: _values(v) for k, v in c.items()}
    x = head_ref.checkpoint(c["x"].float().cpu().numpy())[0]
    want, bound = ref.layer_grad(h["dy"], h["pre"], x, h["w"], "relu", 0.0, 0, 0, bf16)
    for name, got in (("db", db), ("dx", dx), ("dw", dw)):
        _check(_values(got), want[name], bound[name], name)


def test_each_gradient_of_a_layer_alone_is_the_same_and_repeats_bit_for_bit():
    torch = _torch()
    for bf16, rows in ((0, 20), (1, 20), (0, 300), (1, 300)):
        for kind, p in (("none", 0.0), ("gelu", 0.2)):
            c = _layer_case(2, rows, 96, 520, bf16, "whole", seed=3)
            plan = hadfl.DenseLayer(2, rows, 96, 520, bf16=bf16, activation=kind, drop=p)
            whole = plan.backward(c["dy"], c["x"], c["w"], pre=c["pre"], seed=1)
            for _ in range(2):
                assert all(torch.equal(a, b) for a, b in zip(whole, plan.backward(c["dy"], c["x"], c["w"], pre=c["pre"], seed=1)))
            for k, name in enumerate(("dx", "dw", "db")):
                got = plan.backward(c["dy"], c["x"] if name == "dw" else None, c["w"] if name == "dx" else None, pre=c["pre"], want=(name,), seed=1)
                assert [q is None for q in got] == [name != q for q in ("dx", "dw", "db")] and torch.equal(got[k], whole[k])


def test_a_layer_onto_its_residual_and_without_rows():
    torch = _torch()
    for bf16 in (0, 1):
        for rows in (20, 300):
            c = _layer_case(2, rows, 96, 136, bf16, "whole", seed=4)
            plan = hadfl.DenseLayer(2, rows, 96, 136, bf16=bf16, activation="silu", drop=0.2)
            want = plan.forward(c["x"], c["w"], residual=c["residual"], seed=2)
            r = c["residual"].clone()
            assert torch.equal(plan.forward(c["x"], c["w"], residual=r, y=r, seed=2), want)
        for i, o in ((96, 136), (3, 136)):
            plan = hadfl.DenseLayer(2, 0, i, o, bf16=bf16, activation="relu")
            t = lambda *s: torch.randn(s, device="cuda").to(_dtype(bf16))  # noqa: E731
            assert plan.forward(t(2, 0, i), t(2, i, o)).shape == (2, 0, o)
            dx, dw, db = plan.backward(t(2, 0, o), t(2, 0, i), t(2, i, o), pre=t(2, 0, o))
            assert dx.shape == (2, 0, i) and not dw.any() and not db.any()


def test_one_x_or_one_w_for_all_replicas_of_a_layer():
    torch = _torch()
    for bf16 in (0, 1):
        for rows in (20, 300):
            c = _layer_case(3, rows, 64, 128, bf16, "whole", seed=5)
            plan = hadfl.DenseLayer(3, rows, 64, 128, bf16=bf16, activation="gelu")
            x, w, dy = c["x"][:1, :1].expand(3, rows, 64), c["w"][:1].expand(3, 64, 128), c["dy"][:, :1].expand(3, rows, 128)
            assert torch.equal(plan.forward(x, w), plan.forward(x.contiguous(), w.contiguous()))
            a, b = plan.backward(dy, x, w, pre=c["pre"]), plan.backward(dy.contiguous(), x.contiguous(), w.contiguous(), pre=c["pre"])
            assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("rows", [20, 300])
@pytest.mark.parametrize("bf16", [0, 1])
def test_activations_and_slopes_far_out(rows, bf16):
    # x w = x: what the activation makes of the largest magnitudes, of zero and of NaN
    torch = _torch()
    far = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 5.0, -5.0, 9.9, -9.9, 11.0, -11.0, 79.0, -79.0, 1e4, -1e4, 1e30, -1e30], device="cuda").to(_dtype(bf16))
    x = far.expand(1, rows, 16)
    eye = torch.eye(16, device="cuda").to(_dtype(bf16))[None]
    z = _values(x)
    half = ref.HALF_BF16 if bf16 else 8 * ref.EPS32
    for kind in ("relu", "gelu", "silu"):
        plan = hadfl.DenseLayer(1, rows, 16, 16, bf16=bf16, activation=kind)
        with np.errstate(over="ignore", invalid="ignore"):
            want = np.where(np.abs(z) > 50, np.maximum(z, 0), ref.activate(np.clip(z, -50, 50), kind))
            steep = np.where(np.abs(z) > 100, (z > 0) * 1.0, ref.slope(np.clip(z, -100, 100), kind))
        _check(_values(plan.forward(x, eye)), want, half * np.abs(want) + 8 * ref.EPS32 * np.minimum(np.abs(z), 100), kind)
        one = torch.ones((1, rows, 16), device="cuda").to(_dtype(bf16))
        db = plan.backward(one, None, None, pre=x, want=("db",))[2]
        _check(_values(db)[0], rows * steep[0, 0], rows * 64 * ref.EPS32, kind)
        pre = x.clone()
        pre[0, rows // 2, 3] = float("nan")
        db = plan.backward(one, None, None, pre=pre, want=("db",))[2]
        assert torch.isnan(db[0]).tolist() == [j == 3 for j in range(16)]
        bad = torch.zeros((1, rows, 16), device="cuda").to(_dtype(bf16))
        bad[0, rows // 2, 2] = float("nan")
        y = plan.forward(bad, eye)
        assert bool(torch.isnan(y[0, rows // 2]).all()) and not y[0, :rows // 2].any() and not y[0, rows // 2 + 1:].any()


def test_a_dropped_value_has_no_gradient_whatever_it_holds():
    torch = _torch()
    for bf16 in (0, 1):
        for rows in (20, 300):
            c = _layer_case(2, rows, 64, 96, bf16, "whole", seed=6)
            plan = hadfl.DenseLayer(2, rows, 64, 96, bf16=bf16, activation="gelu", drop=0.5)
            stay = torch.as_tensor(ref.kept(2, rows, 96, 0.5, 7, 8)[0]).cuda()
            want = plan.backward(c["dy"], c["x"], c["w"], pre=c["pre"], seed=7, call=8)
            nan = torch.full_like(c["dy"], float("nan"))
            got = plan.backward(torch.where(stay, c["dy"], nan), c["x"], c["w"], pre=torch.where(stay, c["pre"], nan), seed=7, call=8)
            assert all(torch.equal(p, q) for p, q in zip(want, got))


@pytest.mark.parametrize("rows", [20, 300])
@pytest.mark.parametrize("kind", ["columns", "far apart", "outlier"])
def test_32_bit_layers_of_uneven_magnitude(rows, kind):
    # what enters the products in parts of 16 bits; the bounds are those of 32-bit sums
    rng = np.random.default_rng(12)
    n, i, o = 2, 96, 200
    x, w, dy = rng.normal(size=(n, rows, i)), rng.normal(size=(n, i, o)), rng.normal(size=(n, rows, o))
    if kind == "columns":
        e, f = 2.0 ** rng.integers(-30, 31, size=i), 2.0 ** rng.integers(-30, 31, size=o)
        x, w, dy = x * e, w / e[:, None] * f, dy / f
    elif kind == "far apart":
        x, w = x * 2.0 ** 90, w * 2.0 ** -90
    else:
        x[0, 3, 5] = 2.0 ** 40
        w[:, 5] = 0
    t = [_in(v, 0, "whole") for v in (x, w, dy)]
    plan = hadfl.DenseLayer(n, rows, i, o)
    y = plan.forward(t[0], t[1])
    dx, dw, db = plan.backward(t[2], t[0], t[1])
    x, w, dy = (_values(v) for v in t)
    want, bound = ref.layer(x, w, None, None, "none", 0.0, 0, 0, 0)
    _check(_values(y), want["y"], bound["y"], "y")
    want, bound = ref.layer_grad(dy, dy, x, w, "none", 0.0, 0, 0, 0)
    for name, got in (("dx", dx), ("dw", dw), ("db", db)):
        _check(_values(got), want[name], bound[name], name)


def test_layer_gradient_against_differences():
    # central differences of sum(y * v) along a direction, 32-bit passes: |h| = 2^-7 leaves a third derivative's h^2 and rounding of 2^-24 / h
    torch = _torch()
    for kind in ("gelu", "silu"):
        c = _layer_case(2, 24, 48, 80, 0, "whole", seed=9)
        plan = hadfl.DenseLayer(2, 24, 48, 80, activation=kind, drop=0.3)
        kw = dict(seed=5, call=6)
        pre = torch.empty_like(c["pre"])
        plan.forward(c["x"], c["w"], c["bias"], residual=c["residual"], pre=pre, **kw)
        grads = dict(zip(("x", "w", "bias"), plan.backward(c["dy"], c["x"], c["w"], pre=pre, **kw)))
        value = lambda a: float((plan.forward(a["x"], a["w"], a["bias"], residual=a["residual"], **kw).double() * c["dy"].double()).sum())  # noqa: E731
        for name in ("x", "w", "bias"):
            v = torch.sign(grads[name]) / grads[name].numel() ** 0.5
            a, b = dict(c), dict(c)
            a[name], b[name] = c[name] + 2.0 ** -7 * v, c[name] - 2.0 ** -7 * v
            want = float((grads[name].double() * v.double()).sum())
            assert abs((value(a) - value(b)) * 2.0 ** 6 - want) <= 1e-2 * abs(want), (kind, name)


# ---- scores ----------------------------------------------------------------------------------------------------------
SCORES = [(1, 1, 1), (2, 3, 7), (1, 2, 40), (2, 5, 300), (1, 3, 1000), (2, 3, 2050), (1, 3, 4104), (1, 2, 8193), (1, 3, 16390), (2, 1, 32001), (1, 2, 40001), (1, 2, 65536), (1, 2, 65537),
          (1, 1, 131073), (1, 2, 300000), (1, 1, 530001), (1, 1, 1 << 20), (40, 9, 130)]


def _scores_case(n, rows, v, bf16, layout, tokens=3, seed=0):
    rng = np.random.default_rng(seed)
    z = rng.normal(size=(n, rows, v)) * 3 + rng.normal(size=(n, rows, 1)) * 5
    z[rng.random(z.shape) < 0.1] = -np.inf
    z[..., v // 2] = 1.0
    y = rng.integers(0, v, size=(n, rows, tokens)).astype(np.int32)
    y[rng.random(y.shape) < 0.1] = -1
    if tokens > 2:
        y[..., 2] = np.where(rng.random((n, rows)) < 0.5, y[..., 0], v + 5)             # given twice, or none
    return _in(z, bf16, layout), _torch().as_tensor(y).cuda(), y


def _check_scores(z, y, yh, n_top, bf16, plan=None, in_place=False):
    torch = _torch()
    n, rows, v = z.shape
    plan = plan or hadfl.TokenScores(n, rows, v, n_tokens=yh.shape[2], n_top=n_top, bf16=bf16)
    logp, entropy, top, top_logp = plan.forward(z, y)
    rng = np.random.default_rng(1)
    g, dh = (torch.as_tensor(rng.normal(size=s)).float().cuda() for s in (yh.shape, (n, rows)))
    whole = _out((n, rows, v), bf16, "odd")
    out = z if in_place else whole.t
    zh = _values(z)
    plan.backward(z, y, g, dh, dlogits=out)
    assert in_place or whole.untouched()
    for k in range(n):
        r = ref.scores(zh[k], yh[k].astype(np.int64), n_top)
        b = ref.scores_bounds(r, _values(g[k]), _values(dh[k]), bf16)
        of = np.take_along_axis(b["lp"], r["at"], 1)
        fin = np.isfinite(r["logp"])
        got = _values(logp[k])
        assert np.array_equal(got[~fin], r["logp"][~fin])
        _check(got[fin], r["logp"][fin], of[fin], "logp")
        _check(_values(entropy[k]), r["entropy"], b["entropy"], "entropy")
        if n_top:
            assert np.array_equal(top[k].cpu().numpy(), r["top"])
            fin = np.isfinite(r["top_logp"])
            got = _values(top_logp[k])
            assert np.array_equal(got[~fin], r["top_logp"][~fin])
            _check(got[fin], r["top_logp"][fin], np.take_along_axis(b["lp"], r["top"], 1)[fin], "top_logp")
        _check(_values(out[k]), ref.scores_grad(r, _values(g[k]), _values(dh[k])), b["dz"], "dlogits")


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("bf16", [0, 1])
@pytest.mark.parametrize("n,rows,v", SCORES)
def test_scores_and_their_gradient(n, rows, v, bf16, layout):
    z, y, yh = _scores_case(n, rows, v, bf16, layout)
    for n_top in sorted({0, min(v, 5), min(v, 32)}):
        _check_scores(z, y, yh, n_top, bf16)
    _check_scores(z, y, yh, 0, bf16, in_place=True)


@pytest.mark.parametrize("v", [20011, 33001, 60000])
@pytest.mark.parametrize("bf16", [0, 1])
def test_scores_of_many_rows(v, bf16):
    # more logits than one launch takes whole rows of: two rows over and over, the first and the last of each against 64 bits
    torch = _torch()
    n, rows = 2, 1100
    z, y, yh = _scores_case(n, 1, v, bf16, "odd")
    plan = hadfl.TokenScores(n, rows, v, n_tokens=3, n_top=5, bf16=bf16)
    y, yh = y.repeat(1, rows, 1), yh.repeat(rows, 1)
    out = plan.forward(z.expand(n, rows, v), y)
    _check_scores(z.expand(n, 2, v), y[:, :2].contiguous(), yh[:, :2], 5, bf16)
    g, dh = torch.randn((n, 1, 3), device="cuda"), torch.randn((n, 1), device="cuda")
    dz = plan.backward(z.expand(n, rows, v), y, g.repeat(1, rows, 1), dh.repeat(1, rows))
    for t in out + (dz,):
        assert bool((t == t[:, :1]).all())
    r = [ref.scores(_values(z[k]), yh[k, :1].astype(np.int64), 5) for k in range(n)]
    for k in range(n):
        b = ref.scores_bounds(r[k], _values(g[k]), _values(dh[k]), bf16)
        assert np.array_equal(out[2][k, 0].cpu().numpy(), r[k]["top"][0])
        _check(_values(out[1][k, -1:]), r[k]["entropy"], b["entropy"], "entropy")
        _check(_values(dz[k, -1:]), ref.scores_grad(r[k], _values(g[k]), _values(dh[k])), b["dz"], "dlogits")


@pytest.mark.parametrize("v", [5, 32, 200, 3000, 20000, 70001, 140001])
@pytest.mark.parametrize("bf16", [0, 1])
def test_ties_masks_and_rows_of_nothing(v, bf16):
    # rows whose logits all tie, at zeros of both signs, at the type's lowest value, at -inf; one finite logit; two values alone; ascending and
    # descending rows, whose largest lie side by side
    torch = _torch()
    rng = np.random.default_rng(3)
    low = float(torch.finfo(_dtype(bf16)).min)
    z = np.zeros((1, 9, v))
    z[0, 0] = 2.5
    z[0, 1] = np.where(rng.random(v) < 0.5, 0.0, -0.0)
    z[0, 2] = low
    z[0, 3] = -np.inf
    z[0, 4] = -np.inf
    z[0, 4, v // 2] = -7.0
    z[0, 5] = rng.integers(0, 2, size=v)
    z[0, 6], z[0, 7] = np.arange(v), -np.arange(v)
    z[0, 8] = low
    z[0, 8, v // 3] = 0.0
    z = _in(z, bf16, "odd")
    yh = np.stack([rng.integers(0, v, size=(1, 9)), np.full((1, 9), v // 2), np.full((1, 9), -1)], -1).astype(np.int32)
    for n_top in (1, 5, min(v, 32)):
        _check_scores(z, torch.as_tensor(yh).cuda(), yh, n_top, bf16)


@pytest.mark.parametrize("v", [40, 5000, 70001, 140001])
@pytest.mark.parametrize("bf16", [0, 1])
def test_rows_with_a_nan_or_an_infinity(v, bf16):
    torch = _torch()
    z = torch.randn((1, 6, v), device="cuda", generator=torch.Generator(device="cuda").manual_seed(0)).to(_dtype(bf16))
    clean = z.clone()
    z[0, 1, v // 3] = float("nan")
    z[0, 2, v - 1] = float("inf")
    z[0, 3] = float("nan")
    z[0, 4] = float("-inf")
    z[0, 4, 0] = float("nan")
    y = torch.full((1, 6, 2), 3, dtype=torch.int32, device="cuda")
    y[..., 1] = -1
    plan = hadfl.TokenScores(1, 6, v, n_tokens=2, n_top=3, bf16=bf16)
    logp, entropy, top, top_logp = plan.forward(z, y)
    g, dh = torch.randn((1, 6, 2), device="cuda"), torch.randn((1, 6), device="cuda")
    dz = plan.backward(z, y, g, dh)
    for t in (1, 2, 3, 4):
        assert torch.isnan(logp[0, t, 0]) and logp[0, t, 1] == 0 and torch.isnan(entropy[0, t]) and bool(torch.isnan(top_logp[0, t]).all())
        assert bool(torch.isnan(dz[0, t]).any())
    assert top[0, 1, 0] == v // 3 and top[0, 2, 0] == v - 1 and top[0, 3].tolist() == [0, 1, 2] and top[0, 4].tolist() == [0, 1, 2]
    want = plan.forward(clean, y)
    for a, b in zip((logp, entropy, top, top_logp), want):
        assert torch.equal(a[0, 0], b[0, 0]) and torch.equal(a[0, 5], b[0, 5])
    same = plan.backward(clean, y, g, dh)
    assert torch.equal(dz[0, 0], same[0, 0]) and torch.equal(dz[0, 5], same[0, 5]) and bool(torch.isfinite(same).all())


def test_scores_without_tokens_rows_or_entropy():
    torch = _torch()
    for bf16 in (0, 1):
        for v in (600, 70000):
            z, y, yh = _scores_case(2, 5, v, bf16, "whole")
            logp, entropy, top, top_logp = hadfl.TokenScores(2, 5, v, n_tokens=3, n_top=4, bf16=bf16).forward(z, y)
            plan = hadfl.TokenScores(2, 5, v, n_tokens=0, n_top=4, bf16=bf16)
            got = plan.forward(z)
            assert got[0] is None and torch.equal(got[1], entropy) and torch.equal(got[2], top) and torch.equal(got[3], top_logp)
            dh = torch.randn((2, 5), device="cuda")
            full = hadfl.TokenScores(2, 5, v, n_tokens=3, n_top=0, bf16=bf16)
            assert torch.equal(full.forward(z, y)[0], logp)
            assert torch.equal(full.backward(z, y, torch.zeros((2, 5, 3), device="cuda"), dh), plan.backward(z, None, None, dh))
            g = torch.randn((2, 5, 3), device="cuda")
            assert torch.equal(full.backward(z, y, g), full.backward(z, y, g, torch.zeros_like(dh)))
            empty = hadfl.TokenScores(2, 0, v, n_tokens=3, n_top=4, bf16=bf16)
            assert [tuple(t.shape) for t in empty.forward(z[:, :0], y[:, :0].contiguous())] == [(2, 0, 3), (2, 0), (2, 0, 4), (2, 0, 4)]
            one = z[:1, :1].expand(2, 5, v)
            assert all(torch.equal(a, b) for a, b in zip(plan.forward(one)[1:], plan.forward(one.contiguous())[1:]))


def test_the_most_tokens_and_statistics_of_the_caller():
    torch = _torch()
    rng = np.random.default_rng(5)
    z, _, _ = _scores_case(2, 4, 9001, 0, "padded")
    yh = rng.integers(0, 40, size=(2, 4, 64)).astype(np.int32)                       # many of them twice
    y = torch.as_tensor(yh).cuda()
    _check_scores(z, y, yh, 32, 0)
    plan = hadfl.TokenScores(2, 4, 9001, n_tokens=64)
    mine = torch.empty((2, 4, 3), device="cuda")
    g = torch.randn((2, 4, 64), device="cuda")
    plan.forward(z, y)
    want = plan.backward(z, y, g)
    plan.forward(z, y, stats=mine)
    plan.forward(z * 0, y, stats=False)
    assert torch.equal(plan.backward(z, y, g, stats=mine), want) and torch.equal(plan.backward(z, y, g), want)


def test_scores_gradient_against_differences():
    torch = _torch()
    gen = torch.Generator(device="cuda").manual_seed(1)
    z = torch.randn((2, 6, 500), device="cuda", generator=gen)
    y = torch.randint(0, 500, (2, 6, 3), device="cuda", generator=gen, dtype=torch.int32)
    g, dh = torch.randn((2, 6, 3), device="cuda", generator=gen), torch.randn((2, 6), device="cuda", generator=gen)
    plan = hadfl.TokenScores(2, 6, 500, n_tokens=3)
    value = lambda a: (lambda o: float((o[0].double() * g).sum() + (o[1].double() * dh).sum()))(plan.forward(a, y))  # noqa: E731
    value(z)
    grad = plan.backward(z, y, g, dh)
    v = torch.sign(grad) / grad.numel() ** 0.5
    want = float((grad.double() * v).sum())
    h = 2.0 ** -5                                             # rounding: some 36 values of 2^-22 over 2h; curvature: h^2 of the step's own size
    assert abs((value(z + h * v) - value(z - h * v)) / (2 * h) - want) <= 1e-2 * abs(want)


# ---- together ----------------------------------------------------------------------------------------------------------
def _step(n, rows, d, hidden, v, bf16):
    """A block with its residual, logits and their scores, and back: what a program keeps and one pass"""
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(2)
    t = lambda *s, std=1.0: (torch.randn(s, device="cuda", generator=g) * std).to(_dtype(bf16))  # noqa: E731
    s = dict(x=t(n, rows, d), w1=t(n, d, hidden, std=d ** -0.5), w2=t(n, hidden, d, std=hidden ** -0.5), w3=t(n, d, v, std=d ** -0.5),
             b1=torch.randn((n, hidden), device="cuda", generator=g), y=torch.randint(0, v, (n, rows, 2), device="cuda", generator=g, dtype=torch.int32),
             g=torch.randn((n, rows, 2), device="cuda", generator=g), dh=torch.randn((n, rows), device="cuda", generator=g),
             counter=torch.tensor([11], dtype=torch.int64, device="cuda"))
    up, down = hadfl.DenseLayer(n, rows, d, hidden, bf16=bf16, activation="gelu"), hadfl.DenseLayer(n, rows, hidden, d, bf16=bf16, drop=0.1)
    last, drop = hadfl.DenseLayer(n, rows, d, v, bf16=bf16), hadfl.Dropout(n, rows, d, 0.2, bf16=bf16)
    scores = hadfl.TokenScores(n, rows, v, n_tokens=2, n_top=3, bf16=bf16)
    pre = torch.empty((n, rows, hidden), dtype=_dtype(bf16), device="cuda")

    def step():
        k = dict(seed=3, counter=s["counter"])
        x = drop.forward(s["x"], call=0, **k)
        a = up.forward(x, s["w1"], s["b1"], pre=pre)
        h = down.forward(a, s["w2"], residual=x, call=1 << 32, **k)
        z = last.forward(h, s["w3"])
        out = scores.forward(z, s["y"])
        dz = scores.backward(z, s["y"], s["g"], s["dh"])
        dh, dw3, _ = last.backward(dz, h, s["w3"], want=("dx", "dw"))
        da, dw2, _ = down.backward(dh, a, s["w2"], want=("dx", "dw"), call=1 << 32, **k)
        dx, dw1, db1 = up.backward(da, x, s["w1"], pre=pre)
        return out + (drop.backward(dx + dh, call=0, **k), dw1, db1, dw2, dw3)
    return s, step


@pytest.mark.parametrize("rows", [40, 200])
def test_a_block_and_its_answers_against_64_bits(rows):
    # autograd's gradients of the formulas in 64 bits; 32-bit passes are off by some hundred roundings of a tensor's largest value at these sizes: 1e-4
    # of it is far above that and far below what a wrong operand or another mask would show
    torch = _torch()
    n, d, hidden, v = 2, 64, 96, 300
    s, step = _step(n, rows, d, hidden, v, 0)
    got = step()
    p = {k: s[k].double().requires_grad_() for k in ("x", "w1", "b1", "w2", "w3")}
    keep = lambda q, c: torch.as_tensor(ref.kept(n, rows, d, q, 3, c + 11)[0] / (1 - ref.limit(q) / 65536)).cuda()  # noqa: E731
    x = p["x"] * keep(0.2, 0)
    z = x @ p["w1"] + p["b1"][:, None]
    a = 0.5 * z * (1 + torch.tanh(ref.GELU[0] * (z + ref.GELU[1] * z ** 3)))
    h = x + a @ p["w2"] * keep(0.1, 1 << 32)
    lp = torch.log_softmax(h @ p["w3"], -1)
    logp, entropy = lp.gather(2, s["y"].long()), -(lp.exp() * lp).sum(-1)
    ((logp * s["g"]).sum() + (entropy * s["dh"]).sum()).backward()
    want = (logp, entropy, None, lp.topk(3, -1).values, p["x"].grad, p["w1"].grad, p["b1"].grad, p["w2"].grad, p["w3"].grad)
    for i, (q, w) in enumerate(zip(got, want)):
        if w is not None:
            assert float((q.double() - w.detach()).abs().max()) <= 1e-4 * float(w.abs().max()), i
    assert torch.equal(got[2].long(), lp.topk(3, -1).indices)


@pytest.mark.parametrize("bf16,rows,v", [(0, 20, 300), (1, 20, 300), (1, 200, 70000), (0, 200, 40000)])
def test_a_block_replayed_from_a_graph_and_on_a_stream_of_its_own(bf16, rows, v):
    torch = _torch()
    s, step = _step(2, rows, 64, 96, v, bf16)
    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    seen = []
    for i in range(4):
        s["x"].copy_(torch.randn(s["x"].shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(i // 2)))
        s["counter"].fill_(i)                                 # the step's number: other values are dropped
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in out]
        assert all(torch.equal(a, b) for a, b in zip(got, step()))
        seen.append(got[4])
    assert not torch.equal(seen[0], seen[1])
