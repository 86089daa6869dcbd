"""The operators of a language model's head on the GPU where their routes, strides and values end: each kernel that a plan can choose, inputs
whose rows overlap, tensors whose offsets pass 32 bits, logits near the largest float.  References and bounds as in test_gpu_head.py."""
import numpy as np
import pytest

from paper_2111_08274_amd import hadfl
from tests import head_ref as ref
from tests import test_gpu_head as base

pytestmark = pytest.mark.gpu


def _dense(n, rows, i, o, bf16, x, dy, layout="whole"):
    """Checks dw and db for the tensors x, dy"""
    plan, packed = hadfl.DenseGrad(n, rows, i, o, bf16=bf16), hadfl.PackedRows(n, rows, i, bf16=bf16).pack(x)
    dw, db = base._out((n, i, o), 0, layout), base._out((n, o), 0, layout)
    plan.backward(packed, dy, dw=dw.t, db=db.t)
    v, d = ref.checkpoint(x.float().cpu().numpy())[0], base._values(dy)
    base._check(db.get(), d.sum(1), (rows + 16) * ref.EPS32 * np.abs(d).sum(1), "db")
    base._check(dw.get(), np.matmul(v.transpose(0, 2, 1), d), (rows + 16) * ref.EPS32 * np.matmul(np.abs(v).transpose(0, 2, 1), np.abs(d)), "dw")
    assert dw.untouched() and db.untouched()


# rows that do not fill the last 64, in the sizes' different kernels
@pytest.mark.parametrize("n,rows,i,o,bf16", [(1, 1000, 2048, 2048, 1), (4, 1000, 2048, 2048, 1), (1, 8200, 896, 896, 1), (2, 70, 64, 128, 1), (1, 1100, 4104, 3592, 0)])
@pytest.mark.parametrize("stride", [0, 16])
def test_dense_gradient_of_rows_that_overlap(n, rows, i, o, bf16, stride):
    # one row for all rows (the gradient behind a mean over tokens), and rows that begin 16 values after another
    torch = base._torch()
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((n, rows, i), device="cuda", generator=g).to(base._dtype(bf16))
    line = torch.randn(rows * stride + n * o + 64, device="cuda", generator=g).to(base._dtype(bf16))
    _dense(n, rows, i, o, bf16, x, line.as_strided((n, rows, o), (o if n > 1 else 0, stride, 1)))


def _loss(c, k, out, bf16, names=("row_loss", "loss", "dx", "dw", "db")):
    """Checks replica k of what ClassLoss.grad returned against 64 bits"""
    r, b = base._loss_reference(c, k, bf16)
    for name, got in zip(("loss", "row_loss", "dx", "dw", "db"), out):
        if got is not None and name in names:
            base._check(base._values(got[k]), r[name], b[name], name)


@pytest.mark.parametrize("rows,d,v,bf16", [(400, 200, 2056, 1), (20, 200, 2056, 1), (400, 200, 2056, 0), (20, 200, 2056, 0)])
@pytest.mark.parametrize("stride", [0, 8])
def test_loss_with_rows_of_w_that_overlap(rows, d, v, bf16, stride):
    # 200 features do not fill the last 64: what lies beyond W's last row must not be taken for one.  A class whose weights are -inf
    # is out where x is positive; its dx is 0 * inf and not looked at
    torch = base._torch()
    rng = np.random.default_rng(2)
    x = base._in(rng.uniform(0.1, 1, size=(1, rows, d)), bf16, "whole")
    line = torch.as_tensor(rng.normal(size=d * stride + v) / d).cuda().to(base._dtype(bf16))
    y = rng.integers(0, v, size=(1, rows)).astype(np.int32)
    for out in (False, True)[:1 + bf16]:                      # (parts of a 32-bit infinity are NaNs)
        w = line.as_strided((1, d, v), (0, stride, 1))
        if out:
            line[v // 2] = float("-inf")                      # a weight of one class, or of one class a row
        dead = torch.isinf(w[0]).any(0).cpu().numpy()
        y[0][dead[y[0]]] = v - 1
        c = dict(x=x, w=w, bias=None, y=torch.as_tensor(y).cuda(), yh=y)
        got = hadfl.ClassLoss(1, rows, d, v, bf16=bf16).grad(c["x"], c["w"], c["y"])
        if not out:
            _loss(c, 0, got, bf16)
        else:
            # W with the dead classes' weights at a value that leaves exp nothing either
            finite = dict(c, w=torch.where(torch.as_tensor(dead).cuda(), torch.full_like(w, -1e4), w))
            _loss(finite, 0, got, bf16, ("row_loss", "loss", "dw"))


@pytest.mark.parametrize("rows,v", [(5, 300), (100, 300), (600, 1000)])
@pytest.mark.parametrize("bf16", [0, 1])
def test_logits_near_the_largest_float(rows, v, bf16):
    # 2.95e38 = 0.87 of the largest float: its product with log2(e) is none.  Where z lies so far apart the softmax is one class, or
    # an even share of those that tie
    torch = base._torch()
    x, w = torch.zeros((1, rows, 16), device="cuda"), torch.zeros((1, 16, v), device="cuda")
    x[:, :, 0] = 2.0 ** 63
    w[:, 0, 7] = w[:, 0, 9] = 2.0 ** 64 * 1.734375
    w[:, 0, 11] = -2.0 ** 64 * 1.734375
    low = torch.zeros_like(w)
    low[:, 0] = -2.0 ** 64 * 1.734375                         # the same logit, far below zero, for every class
    y = torch.full((1, rows), 7, dtype=torch.int32, device="cuda")
    plan = hadfl.ClassLoss(1, rows, 16, v, bf16=bf16)
    t = base._dtype(bf16)
    loss, row, dx, dw, _ = plan.grad(x.to(t), w.to(t), y)
    assert (row - float(np.log(2))).abs().max() < 1e-6 and (loss - float(np.log(2))).abs() < 1e-6
    share = torch.zeros(v, device="cuda")
    share[7], share[9] = -0.5, 0.5
    assert torch.equal(dw[0, 0].float() / 2.0 ** 63, share) and not dw[0, 1:].any()
    assert not dx.any()                                       # (p_7 - 1 + p_9) times the weight that 7 and 9 share
    loss, row, dx, dw, _ = plan.grad(x.to(t), low.to(t), y)
    assert (row - float(np.log(v))).abs().max() < 1e-5
    even = torch.full((v,), 1.0 / v, device="cuda", dtype=torch.float64)
    even[7] -= 1
    assert ((dw[0, 0].double() / 2.0 ** 63 - even).abs() <= 2.0 ** -7 * even.abs()).all()


@pytest.mark.parametrize("shared", [False, True])
def test_a_vocabulary_whose_last_piece_would_hold_three_classes(shared):
    # 1024 replicas of 130 rows: pieces of 1024 classes would leave three for the eighth; W a full tensor, and one line for all features
    # that ends with its last class
    torch = base._torch()
    n, rows, d, v = 1024, 130, 16, 7171
    c = base._loss_case(1, rows, d, v, 0, "whole", True, seed=6)
    c["x"].nan_to_num_(nan=0.5, posinf=0.5)
    if shared:
        line = torch.full((v + 8,), float("nan"), device="cuda")
        line[:v] = c["w"][0, 0] / 4
        c["w"] = line[:v].expand(1, d, v)
    args = c["x"].expand(n, rows, d), c["w"].expand(n, d, v), c["y"].repeat(n, 1), c["bias"].expand(n, v)
    out = hadfl.ClassLoss(n, rows, d, v).grad(*args)
    one = dict(x=c["x"], w=c["w"], bias=c["bias"], yh=c["yh"])
    _loss(one, 0, [o[:1] for o in out], 0)
    assert all(torch.equal(o[0], o[k]) for o in out for k in (1, n - 1))


def test_more_rows_than_one_launch_has_threads_for():
    # 2^24 rows of 4128 values, all the same one in memory: 2^32 threads and 2^27 more; the checkpoint's first lines and its last
    torch = base._torch()
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("needs 72 GB of device memory")
    n, rows, cols = 16, 1 << 20, 4128
    x = torch.randn((1, 1, cols), device="cuda", generator=torch.Generator(device="cuda").manual_seed(0)).bfloat16()
    one = hadfl.PackedRows(1, 1, cols, bf16=1).pack(x)
    many = hadfl.PackedRows(n, rows, cols, bf16=1).pack(x.expand(n, rows, cols))
    q, e = one.data[:cols], one.data[cols // 256 * 256 + 256:][:cols // 32]
    got_q = many.data[:n * rows * cols].view(n * rows, cols)
    got_e = many.data[n * rows * cols:][:n * rows * (cols // 32)].view(n * rows, cols // 32)
    for t in (0, 1, 1 << 20, (1 << 23) + 5, n * rows - 1):
        assert torch.equal(got_q[t], q) and torch.equal(got_e[t], e), t
    assert bool((got_e == e).all())
    del many, got_q, got_e
    torch.cuda.empty_cache()


def test_more_tiles_than_one_launch_has_threads_for():
    # 2^22 rows and 2^17 classes are 2^23 tiles of 512 threads
    torch = base._torch()
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 18 GB of device memory")
    n, rows, d, v = 1024, 4096, 8, 131072
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w = torch.randn((1, rows, d), device="cuda", generator=g).bfloat16(), torch.randn((1, d, v), device="cuda", generator=g).bfloat16()
    y = torch.randint(0, v, (1, rows), device="cuda", generator=g, dtype=torch.int32)
    loss, row = hadfl.ClassLoss(n, rows, d, v, bf16=1, grad=False).loss(x.expand(n, rows, d), w.expand(n, d, v), y.repeat(n, 1))
    assert bool((row == row[:1]).all()) and bool((loss == loss[0]).all())
    some = slice(0, 64)
    r = ref.class_loss(base._values(x[0, some]), base._values(w[0]), None, y[0, some].cpu().numpy().astype(np.int64))
    b = ref.class_loss_bounds(r, base._values(w[0]), None, 1)
    base._check(base._values(row[0, some]), r["row_loss"], b["row_loss"], "row_loss")
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n,rows,d,v,bf16", [(2, 5, 40, 300, 0), (2, 100, 40, 300, 1), (2, 500, 40, 1000, 0), (1, 500, 800, 2056, 1)])
def test_db_without_a_bias(n, rows, d, v, bf16):
    c = base._loss_case(n, rows, d, v, bf16, "whole", False)
    db = base._out((n, v), 0, "odd")
    out = hadfl.ClassLoss(n, rows, d, v, bf16=bf16).grad(c["x"], c["w"], c["y"], db=db.t)
    assert out[4] is db.t and db.untouched()
    for k in range(n):
        _loss(c, k, out, bf16)


def test_an_evaluation_between_a_forward_pass_and_its_gradient():
    torch = base._torch()
    c, other = base._norm_case(2, 9, 200, 0, "whole"), base._norm_case(2, 9, 200, 0, "whole", seed=1)
    plan = hadfl.LayerNorm(2, 9, 200)
    y = plan.forward(c["x"], c["gamma"], c["beta"])
    want = plan.backward(c["dy"], c["x"], c["gamma"])
    mine = torch.empty((2, 9), device="cuda"), torch.empty((2, 9), device="cuda")
    seen = plan.forward(other["x"], other["gamma"], other["beta"], stats=False)
    assert torch.equal(seen, plan.forward(other["x"], other["gamma"], other["beta"], stats=mine))
    assert all(torch.equal(p, q) for p, q in zip(want, plan.backward(c["dy"], c["x"], c["gamma"])))
    fresh = hadfl.LayerNorm(2, 9, 200)
    assert torch.equal(fresh.forward(other["x"], other["gamma"], other["beta"]), seen)
    assert all(torch.equal(p, q) for p, q in zip(fresh.backward(other["dy"], other["x"], other["gamma"]),
                                                 plan.backward(other["dy"], other["x"], other["gamma"], stats=mine)))
    assert torch.equal(plan.forward(c["x"], c["gamma"], c["beta"]), y)


# with the sizes of test_gpu_head.py these reach every kernel (test_head_launches.py)
DENSE = [(1, 1000, 2048, 2048, 1), (6, 1001, 1288, 1544, 1), (6, 1001, 1287, 1543, 1), (1, 8200, 896, 896, 1), (1, 8199, 895, 900, 1), (1, 1101, 4104, 3592, 0),
         (1, 1101, 4101, 3595, 0), (1, 4501, 4104, 4090, 0),
         (31, 3588, 101, 2078, 1), (15, 631, 10, 1537, 1), (1, 9000, 40, 5, 0), (1, 9000, 40, 5, 1)]


@pytest.mark.parametrize("layout", ["whole", "padded", "odd"])
@pytest.mark.parametrize("n,rows,i,o,bf16", DENSE)
def test_dense_gradient_with_operands_from_memory(n, rows, i, o, bf16, layout):
    rng = np.random.default_rng(13)
    x, dy = rng.normal(size=(n, rows, i)).clip(0), rng.normal(size=(n, rows, o)) * 2.0 ** rng.integers(-8, 8, size=(n, rows, 1))
    _dense(n, rows, i, o, bf16, base._in(x, bf16, layout), base._in(dy, bf16, layout), layout)


LOSS = [(1, 450, 776, 2500, 1), (2, 430, 1030, 2312, 1), (2, 1000, 776, 4200, 1), (2, 1000, 100, 8400, 1), (2, 1000, 500, 4203, 1), (2, 1000, 100, 8400, 0), (2, 1001, 300, 8403, 0),
        (2, 1000, 500, 4203, 0), (2, 380, 64, 9001, 1), (2, 380, 64, 9001, 0), (1, 3000, 72, 520, 1), (1, 3000, 72, 520, 0), (1, 1175, 152, 78, 0),
        (2, 84, 505, 124, 1), (1, 97, 325, 68, 0), (3, 39, 391, 71, 1)]
PIECES = [(64, 500, 64, 8400, 0), (64, 500, 300, 8403, 0), (64, 500, 64, 16500, 1), (64, 500, 300, 16501, 1), (64, 180, 10, 8001, 1), (64, 32, 16, 66001, 0),
          (8, 260, 16400, 1030, 0)]


@pytest.mark.parametrize("layout", ["whole", "padded", "odd"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("n,rows,d,v,bf16", LOSS)
def test_loss_with_operands_from_memory(n, rows, d, v, bf16, bias, layout):
    torch = base._torch()
    c = base._loss_case(n, rows, d, v, bf16, layout, bias)
    plan = hadfl.ClassLoss(n, rows, d, v, bf16=bf16)
    dx, dw, db = base._out((n, rows, d), bf16, layout), base._out((n, d, v), bf16, layout), base._out((n, v), 0, layout)
    out = plan.grad(c["x"], c["w"], c["y"], c["bias"], dx=dx.t, dw=dw.t, db=db.t if bias else None)
    for k in range(n):
        _loss(c, k, out, bf16)
        dead = torch.as_tensor((c["yh"][k] < 0) | (c["yh"][k] >= v)).cuda()
        assert not out[1][k][dead].any() and not dx.t[k][dead].any()
    assert dx.untouched() and dw.untouched() and (not bias or db.untouched())
    alone = plan.loss(c["x"], c["w"], c["y"], c["bias"])
    assert torch.equal(alone[0], out[0]) and torch.equal(alone[1], out[1])


@pytest.mark.parametrize("n,rows,d,v,bf16", PIECES)
def test_a_vocabulary_in_pieces_of_every_kind(n, rows, d, v, bf16):
    # replicas with one x and one W whose logits, or W's copies, pass what one piece holds
    torch = base._torch()
    c = base._loss_case(1, rows, d, v, bf16, "whole", True)
    c["x"].nan_to_num_(nan=0.5, posinf=0.5)
    y = c["y"].repeat(n, 1)
    y[-1] = torch.flip(y[-1], dims=[0])
    out = hadfl.ClassLoss(n, rows, d, v, bf16=bf16).grad(c["x"].expand(n, rows, d), c["w"].expand(n, d, v), y, c["bias"].expand(n, v))
    for k in (0, n - 1):
        _loss(dict(x=c["x"], w=c["w"], bias=c["bias"], yh=y[k:k + 1].cpu().numpy()), 0, [o[k:k + 1] for o in out], bf16)
    assert all(torch.equal(o[0], o[n - 2]) for o in out)


def _far(values, bf16, pitch):
    """[1][rows][cols] as a view whose rows are `pitch` elements apart, in memory that holds zeros"""
    torch = base._torch()
    rows, cols = values.shape
    t = torch.zeros(((rows - 1) * pitch + cols,), dtype=base._dtype(bf16), device="cuda").as_strided((1, rows, cols), (0, pitch, 1))
    return t.copy_(torch.as_tensor(values)[None].to(t.dtype))


@pytest.mark.parametrize("bf16", [0, 1])
def test_offsets_that_pass_32_bits_in_norm_checkpoint_and_dense_gradient(bf16):
    torch = base._torch()
    torch.cuda.empty_cache()
    rng = np.random.default_rng(21)
    rows, cols, pitch = 300, 264, (1 << 24) + 8               # the last rows lie beyond 2^32 elements
    x, dy = _far(rng.normal(size=(rows, cols)), bf16, pitch), torch.as_tensor(rng.normal(size=(1, rows, cols))).cuda().to(base._dtype(bf16))
    gamma, near = torch.rand((1, cols), device="cuda"), x.contiguous()
    plan = hadfl.LayerNorm(1, rows, cols, bf16=bf16)
    y = plan.forward(near, gamma, gamma)
    want = plan.backward(dy, near, gamma)
    out = _far(np.zeros((rows, cols)), bf16, pitch)
    assert torch.equal(plan.forward(x, gamma, gamma, y=out), y)
    got = plan.backward(dy, x, gamma, dx=out)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    packed, same = hadfl.PackedRows(1, rows, cols, bf16=bf16).pack(x), hadfl.PackedRows(1, rows, cols, bf16=bf16).pack(near)
    assert torch.equal(packed.unpack(out), same.unpack())
    out.copy_(dy)
    dense = hadfl.DenseGrad(1, rows, cols, cols, bf16=bf16)
    assert all(torch.equal(p, q) for p, q in zip(dense.backward(packed, out), dense.backward(packed, dy)))
    del x, out, got
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows,bf16", [(8, 0), (40, 0), (600, 0), (8, 1), (40, 1), (600, 1)])
def test_offsets_that_pass_32_bits_in_the_loss(rows, bf16):
    # W's rows as far apart as a product reads them from where they lie, and a little farther
    torch = base._torch()
    torch.cuda.empty_cache()
    rng = np.random.default_rng(22)
    d, v = 1100, 1000
    for pitch in (1 << 22, (1 << 22) + 8):
        w = _far(rng.normal(size=(d, v)) / 33, bf16, pitch)
        x = torch.as_tensor(rng.normal(size=(1, rows, d))).cuda().to(w.dtype)
        y = torch.as_tensor(rng.integers(0, v, size=(1, rows)).astype(np.int32)).cuda()
        plan = hadfl.ClassLoss(1, rows, d, v, bf16=bf16)
        want = plan.grad(x, w.contiguous(), y)
        dw = _far(np.zeros((d, v)), bf16, pitch)
        got = plan.grad(x, w, y, dw=dw)
        assert all(torch.equal(p, q) for p, q in zip(got, want) if p is not None)
        del w, dw, got
        torch.cuda.empty_cache()
