"""The operators of a language model's head refuse what they cannot do before they touch the device: status and text."""
import ctypes

import numpy as np
import pytest

from paper_2111_08274_amd import hadfl
from tests import head_ref as ref

R = hadfl.HadflRows
GOOD = 1 << 20                                    # an address that is aligned to anything; never read here


def _refused(call, text):
    assert call() == hadfl.EINVAL
    assert text in hadfl.lib().hadfl_last_error(None).decode(), hadfl.lib().hadfl_last_error(None)


def _size(query, desc, *more):
    n = ctypes.c_size_t()
    assert query(ctypes.byref(desc), *more, ctypes.byref(n)) == hadfl.OK
    return n.value


def test_sizes_out_of_range_are_refused():
    L, n = hadfl.lib(), ctypes.c_size_t(7)
    out = ctypes.byref(n)
    for desc, query, more in ((hadfl.HadflNorm(2, 3, 4, 0, 1e-5), L.hadfl_norm_workspace, ()), (hadfl.HadflPack(2, 3, 4, 0), L.hadfl_packed_bytes, ()),
                              (hadfl.HadflDense(2, 3, 4, 5, 0), L.hadfl_dense_workspace, ()), (hadfl.HadflLoss(2, 3, 4, 5, 0), L.hadfl_loss_workspace, (1,))):
        kind = type(desc)
        values = [getattr(desc, f[0]) for f in kind._fields_]
        assert _size(query, desc, *more) > 0
        _refused(lambda: query(None, *more, out), "is null")
        _refused(lambda: query(ctypes.byref(desc), *more, None), "bytes is null")
        for field, value in [("n_replicas", 0), ("n_replicas", 1025), ("n_rows", -1), ("n_rows", (1 << 20) + 1), ("bf16", 2), ("bf16", -1), ("eps", -1.0),
                             ("eps", float("nan")), ("eps", float("inf")), ("n_features", 0), ("n_features", (1 << 17) + 1), ("n_in", 0),
                             ("n_out", -5), ("n_classes", 0), ("n_classes", (1 << 20) + 1)]:
            if field not in [f[0] for f in kind._fields_]:
                continue
            bad = kind(*values)
            setattr(bad, field, value)
            _refused(lambda: query(ctypes.byref(bad), *more, out), field)
        big = kind(*values)
        big.n_replicas, big.n_rows = 1024, 1 << 15
        _refused(lambda: query(ctypes.byref(big), *more, out), "2^24")
    assert n.value == 7                            # nothing is written on an error


def test_tensors_that_do_not_fit_are_refused():
    L = hadfl.lib()
    d = hadfl.HadflNorm(2, 3, 8, 1, 1e-5)
    ok, vec = R(GOOD, 24, 8), R(GOOD, 8, 0)

    def norm(x=ok, gamma=vec, beta=vec, y=ok, mean=GOOD, rstd=GOOD):
        return L.hadfl_norm_forward(ctypes.byref(d), *(None if r is None else ctypes.byref(r) for r in (x, gamma, beta, y)), mean, rstd, None)

    for kw, text in ((dict(x=None), "x is null"), (dict(x=R(None, 24, 8)), "x has no data"), (dict(x=R(GOOD + 1, 24, 8)), "x is not aligned"),
                     (dict(x=R(GOOD, -1, 8)), "x: strides"), (dict(x=R(GOOD, 24, 1 << 41)), "x: strides"), (dict(y=R(GOOD, 24, 7)), "y: row_stride"),
                     (dict(y=R(GOOD, 23, 8)), "y: the replicas"), (dict(y=R(GOOD, 0, 8)), "y: the replicas"), (dict(gamma=R(GOOD + 2, 8, 0)), "gamma is not"),
                     (dict(beta=None), "beta is null"), (dict(mean=None), "mean and rstd"), (dict(rstd=GOOD + 1), "rstd must be")):
        _refused(lambda: norm(**kw), text)

    def norm_back(dy=ok, x=ok, packed=None, dx=ok, dgamma=vec, work=GOOD, mean=GOOD):
        refs = lambda r: None if r is None else ctypes.byref(r)  # noqa: E731
        return L.hadfl_norm_backward(ctypes.byref(d), refs(dy), refs(x), packed, refs(vec), mean, GOOD, refs(dx), refs(dgamma), refs(vec), work, None)

    for kw, text in ((dict(dy=None), "dy is null"), (dict(x=None), "x is null"), (dict(packed=GOOD + 64), "packed must be 256"), (dict(mean=None), "mean is null"),
                     (dict(dgamma=R(GOOD, 7, 0)), "dgamma: the replicas"), (dict(work=None), "work is null"), (dict(work=GOOD + 128), "work must be 256"),
                     (dict(dx=R(GOOD, 24, 4)), "dx: row_stride")):
        _refused(lambda: norm_back(**kw), text)

    p = hadfl.HadflPack(2, 3, 8, 0)
    _refused(lambda: L.hadfl_pack_rows(ctypes.byref(p), ctypes.byref(ok), None, None), "packed is null")
    _refused(lambda: L.hadfl_pack_rows(ctypes.byref(p), ctypes.byref(R(GOOD + 2, 24, 8)), GOOD, None), "x is not aligned")
    _refused(lambda: L.hadfl_unpack_rows(ctypes.byref(p), GOOD, ctypes.byref(R(GOOD, 8, 8)), None), "out: the replicas")

    g = hadfl.HadflDense(2, 3, 8, 8, 0)
    dw = R(GOOD, 64, 8)
    _refused(lambda: L.hadfl_dense_grad_packed(ctypes.byref(g), GOOD + 1, ctypes.byref(ok), ctypes.byref(dw), None, GOOD, None), "packed must be")
    _refused(lambda: L.hadfl_dense_grad_packed(ctypes.byref(g), GOOD, ctypes.byref(ok), ctypes.byref(R(GOOD, 60, 8)), None, GOOD, None), "dw: the replicas")
    _refused(lambda: L.hadfl_dense_grad_packed(ctypes.byref(g), GOOD, None, ctypes.byref(dw), None, GOOD, None), "dy is null")
    _refused(lambda: L.hadfl_dense_grad_packed(ctypes.byref(g), GOOD, ctypes.byref(ok), ctypes.byref(dw), None, None, None), "work is null")

    s = hadfl.HadflLoss(2, 3, 8, 10, 0)
    w = R(GOOD, 80, 10)

    def loss(x=ok, w=w, bias=None, labels=GOOD, out=GOOD, row=None, dx=None, dw=None, db=None, work=GOOD):
        refs = lambda r: None if r is None else ctypes.byref(r)  # noqa: E731
        return L.hadfl_loss_grad(ctypes.byref(s), refs(x), refs(w), refs(bias), labels, out, row, refs(dx), refs(dw), refs(db), work, None)

    for kw, text in ((dict(x=None), "x is null"), (dict(w=None), "w is null"), (dict(labels=None), "labels is null"), (dict(out=None), "loss is null"),
                     (dict(labels=GOOD + 2), "labels must be 4"), (dict(row=GOOD + 1), "row_loss must be"), (dict(bias=R(GOOD, -4, 0)), "bias: strides"),
                     (dict(dx=R(GOOD, 16, 8)), "dx: the replicas"), (dict(dw=R(GOOD, 80, 9)), "dw: row_stride"), (dict(db=R(GOOD, 9, 0)), "db: the replicas"),
                     (dict(work=None), "work is null"), (dict(work=GOOD + 4), "work must be 256")):
        _refused(lambda: loss(**kw), text)
    assert L.hadfl_loss_forward(ctypes.byref(s), None, None, None, None, None, None, None, None) == hadfl.EINVAL


def test_the_loss_keeps_pieces_of_the_logits_only():
    # 2^21 rows x classes x 64 would be 8 GiB of 32-bit logits; the working memory is bounded by the piece and the parts
    d = hadfl.HadflLoss(8, 4096, 512, 65536, 0)
    assert _size(hadfl.lib().hadfl_loss_workspace, d, 1) < 8 * 4096 * 65536 * 4 / 4


def test_reference_gradients_against_differences():
    rng = np.random.default_rng(0)
    x, g, b, dy = rng.normal(size=(3, 10)), rng.normal(size=10), rng.normal(size=10), rng.normal(size=(3, 10))
    f = lambda x, g, b: (ref.layer_norm(x, g, b, 1e-5)[0] * dy).sum()  # noqa: E731
    _, mean, rstd = ref.layer_norm(x, g, b, 1e-5)
    for k, grad in enumerate(ref.layer_norm_grad(dy, x, g, mean, rstd)):
        args = [x, g, b]
        v = rng.normal(size=args[k].shape)
        up, down = list(args), list(args)
        up[k], down[k] = args[k] + 1e-5 * v, args[k] - 1e-5 * v
        assert abs((f(*up) - f(*down)) / 2e-5 - (grad * v).sum()) < 1e-7
    x, w, bias, y = rng.normal(size=(4, 5)), rng.normal(size=(5, 7)), rng.normal(size=7), np.array([1, -1, 6, 7])
    r = ref.class_loss(x, w, bias, y)
    assert r["n"] == 2 and r["row_loss"][1] == 0 and r["row_loss"][3] == 0 and not r["dx"][[1, 3]].any()
    for k, name in enumerate(("dx", "dw", "db")):
        args = [x, w, bias]
        v = rng.normal(size=args[k].shape)
        up, down = list(args), list(args)
        up[k], down[k] = args[k] + 1e-5 * v, args[k] - 1e-5 * v
        diff = (ref.class_loss(*up, y)["loss"] - ref.class_loss(*down, y)["loss"]) / 2e-5
        assert abs(diff - (r[name] * v).sum()) < 1e-7


@pytest.mark.parametrize("x,q,e", [([127.0, -1.0], [127, -1], 0), ([127.5, 1.0], [64, 0], 1), ([0.0, 0.0], [0, 0], -126), ([1.0, 0.5], [64, 32], -6),
                                   ([254.0, 3.0], [127, 2], 1), ([254.0, 1.0], [127, 0], 1)])
def test_reference_checkpoint_by_hand(x, q, e):
    # 127.5 exceeds 127 * 2^0, so the step is 2: 63.75 -> 64, 0.5 -> 0 (ties to even); 3 / 2 = 1.5 -> 2
    v, gq, ge = ref.checkpoint(np.array(x))
    assert gq[:2].tolist() == q and int(ge[0]) - 127 == e and v.tolist() == [i * 2.0 ** e for i in q]
