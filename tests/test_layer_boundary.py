"""The operators of a next-word model's layers and answers refuse what they cannot do before they touch the device: status and text."""
import ctypes

import pytest

from paper_2111_08274_amd import hadfl
from tests.test_head_boundary import GOOD, R, _refused, _size
from tests.test_head_binding import Device, Machine, Stream, Tensor

DRAW = hadfl.HadflDraw(1, 2, None)


def _p(v):
    return None if v is None else ctypes.byref(v) if isinstance(v, ctypes.Structure) else v


def test_sizes_out_of_range_are_refused():
    L, n = hadfl.lib(), ctypes.c_size_t(7)
    out = ctypes.byref(n)
    ok = R(GOOD, 1 << 20, 1 << 10)
    descs = ((hadfl.HadflLayer(2, 3, 4, 5, 0, 0, 0.5), lambda d: L.hadfl_layer_workspace(d, 1, out)),
             (hadfl.HadflScores(2, 3, 40, 1, 2, 0), lambda d: L.hadfl_scores_workspace(d, out)),
             (hadfl.HadflDropout(2, 3, 4, 0, 0.5), lambda d: L.hadfl_dropout_rows(d, _p(ok), None, _p(DRAW), None, None)))
    for desc, query in descs:
        kind = type(desc)
        values = [getattr(desc, f[0]) for f in kind._fields_]
        _refused(lambda: query(None), "is null")
        for field, value, text in [("n_replicas", 0, ""), ("n_replicas", 1025, ""), ("n_rows", -1, ""), ("n_rows", (1 << 20) + 1, ""), ("bf16", 2, ""), ("n_features", 0, ""),
                                   ("n_features", (1 << 17) + 1, ""), ("n_in", 0, ""), ("n_out", (1 << 17) + 1, ""), ("activation", -1, ""), ("activation", 4, ""),
                                   ("drop", -0.1, "probability"), ("drop", 1.0, "probability"), ("drop", float("nan"), "probability"), ("p", 1.0, "probability"),
                                   ("p", -1e-30, "probability"), ("n_classes", 0, ""), ("n_classes", (1 << 20) + 1, ""), ("n_tokens", -1, ""), ("n_tokens", 65, ""),
                                   ("n_top", -1, ""), ("n_top", 33, ""), ("n_top", 41, "n_top")]:
            if field not in [f[0] for f in kind._fields_]:
                continue
            bad = kind(*values)
            setattr(bad, field, value)
            _refused(lambda: query(ctypes.byref(bad)), text or field)
        big = kind(*values)
        big.n_replicas, big.n_rows = 1024, 1 << 15
        _refused(lambda: query(ctypes.byref(big)), "2^24")
    few = hadfl.HadflScores(2, 3, 4, 1, 5, 0)
    _refused(lambda: L.hadfl_scores_workspace(ctypes.byref(few), out), "n_top")
    _refused(lambda: L.hadfl_layer_workspace(ctypes.byref(descs[0][0]), 1, None), "bytes is null")
    _refused(lambda: L.hadfl_scores_workspace(ctypes.byref(descs[1][0]), None), "bytes is null")
    assert n.value == 7                            # nothing is written on an error


def test_tensors_of_a_layer_that_do_not_fit_are_refused():
    L = hadfl.lib()
    d = hadfl.HadflLayer(2, 3, 8, 16, 1, hadfl.ACTIVATIONS.index("gelu"), 0.25)
    x, w, y, b = R(GOOD, 24, 8), R(GOOD, 128, 16), R(GOOD, 48, 16), R(GOOD, 16, 0)

    def forward(x=x, w=w, bias=b, residual=y, draw=DRAW, pre=y, y=y, work=GOOD, d=d):
        return L.hadfl_layer_forward(ctypes.byref(d), *map(_p, (x, w, bias, residual, draw, pre, y)), work, None)

    for kw, text in ((dict(x=None), "x is null"), (dict(x=R(None, 24, 8)), "x has no data"), (dict(x=R(GOOD + 1, 24, 8)), "x is not aligned"), (dict(w=None), "w is null"),
                     (dict(w=R(GOOD, -1, 16)), "w: strides"), (dict(bias=R(GOOD + 2, 16, 0)), "bias is not"), (dict(residual=R(GOOD, 48, 1 << 41)), "residual: strides"),
                     (dict(draw=None), "draw is null"), (dict(draw=hadfl.HadflDraw(1, 2, GOOD + 4)), "counter"), (dict(pre=R(GOOD, 48, 15)), "pre: row_stride"),
                     (dict(y=None), "y is null"), (dict(y=R(GOOD, 47, 16)), "y: the replicas"), (dict(work=None), "work is null"), (dict(work=GOOD + 128), "work must be 256")):
        _refused(lambda: forward(**kw), text)

    def backward(dy=y, pre=y, x=x, packed=None, w=w, draw=DRAW, dx=x, dw=w, db=b, work=GOOD, d=d):
        return L.hadfl_layer_backward(ctypes.byref(d), *map(_p, (dy, pre, x, packed, w, draw, dx, dw, db)), work, None)

    for kw, text in ((dict(dy=None), "dy is null"), (dict(pre=None), "pre is null"), (dict(x=None), "x is null"), (dict(x=None, packed=GOOD + 16), "packed must be 256"),
                     (dict(w=None), "w is null"), (dict(draw=None), "draw is null"), (dict(dx=R(GOOD, 24, 7)), "dx: row_stride"), (dict(dw=R(GOOD, 0, 16)), "dw: the replicas"),
                     (dict(db=R(GOOD + 1, 16, 0)), "db is not"), (dict(work=GOOD + 1), "work must be")):
        _refused(lambda: backward(**kw), text)


def test_tensors_of_a_dropout_and_of_scores_that_do_not_fit_are_refused():
    L = hadfl.lib()
    d, x = hadfl.HadflDropout(2, 3, 8, 0, 0.5), R(GOOD, 24, 8)

    def drop(x=x, residual=x, draw=DRAW, y=x):
        return L.hadfl_dropout_rows(ctypes.byref(d), *map(_p, (x, residual, draw, y)), None)

    for kw, text in ((dict(x=None), "x is null"), (dict(residual=R(GOOD + 2, 24, 8)), "residual is not"), (dict(draw=None), "draw is null"), (dict(y=None), "y is null"),
                     (dict(y=R(GOOD, 24, 7)), "y: row_stride"), (dict(draw=hadfl.HadflDraw(1, 2, GOOD + 1)), "counter")):
        _refused(lambda: drop(**kw), text)
    s, z = hadfl.HadflScores(2, 3, 40, 2, 4, 0), R(GOOD, 120, 40)

    def forward(z=z, tokens=GOOD, logp=GOOD, entropy=GOOD, stats=GOOD, top=GOOD, top_logp=GOOD, work=GOOD):
        return L.hadfl_scores_forward(ctypes.byref(s), _p(z), tokens, logp, entropy, stats, top, top_logp, work, None)

    for kw, text in ((dict(z=None), "logits is null"), (dict(tokens=None), "tokens is null"), (dict(logp=GOOD + 2), "logp must be"), (dict(entropy=GOOD + 1), "entropy must be"),
                     (dict(stats=GOOD + 2), "stats must be"), (dict(top=None), "top is null"), (dict(top_logp=None), "top_logp is null"), (dict(work=None), "work is null")):
        _refused(lambda: forward(**kw), text)

    def backward(z=z, tokens=GOOD, stats=GOOD, dlogp=GOOD, dentropy=GOOD, dz=z):
        return L.hadfl_scores_backward(ctypes.byref(s), _p(z), tokens, stats, dlogp, dentropy, _p(dz), None)

    for kw, text in ((dict(z=None), "logits is null"), (dict(tokens=None), "tokens is null"), (dict(stats=None), "stats is null"), (dict(dlogp=None), "dlogp is null"),
                     (dict(dentropy=GOOD + 2), "dentropy must be"), (dict(dz=None), "dlogits is null"), (dict(dz=R(GOOD, 119, 40)), "dlogits: the replicas")):
        _refused(lambda: backward(**kw), text)


def test_the_working_memory_holds_what_both_calls_take():
    L = hadfl.lib()
    for n, rows, i, o in ((1, 0, 8, 8), (1, 1, 1, 1), (2, 64, 130, 257), (2, 65, 130, 257), (16, 1024, 512, 2048)):
        for bf16 in (0, 1):
            d = hadfl.HadflLayer(n, rows, i, o, bf16, 0, 0.0)
            assert _size(L.hadfl_layer_workspace, d, 1) >= _size(L.hadfl_layer_workspace, d, 0) > 0


@pytest.fixture
def machine(monkeypatch):
    real = hadfl.lib()
    m = Machine(monkeypatch)
    import sys
    fake = sys.modules["torch"]
    fake.int64 = "i64"
    for name in hadfl.EXPORTS:
        if name.startswith(("hadfl_layer", "hadfl_dropout", "hadfl_scores")):
            call = getattr(real, name) if name.endswith("workspace") else lambda *a, _name=name: (m.calls.append((_name, m.now, a)), 0)[1]
            setattr(hadfl._lib, name, call)
    Tensor.numel = lambda self: 1 if not self.shape else self.shape[0]
    yield m
    del Tensor.numel


def _plans(n=2, rows=3, i=8, o=16):
    return (hadfl.Dropout(n, rows, i, 0.5), hadfl.DenseLayer(n, rows, i, o, activation="relu"), hadfl.TokenScores(n, rows, o, n_tokens=2, n_top=3))


def _calls(device, n=2, rows=3, i=8, o=16):
    t = lambda *s, dtype="f32": Tensor(s, dtype, device)  # noqa: E731
    drop, dense, scores = _plans(n, rows, i, o)
    x, w, y, tokens, two = t(n, rows, i), t(n, i, o), t(n, rows, o), t(n, rows, 2, dtype="i32"), t(n, rows, 2)
    return [(drop.forward, (x,)), (drop.backward, (x,)), (dense.forward, (x, w)), (dense.backward, (y, x, w, y)), (dense.backward, (y, hadfl.PackedRows(n, rows, i), w, y)),
            (scores.forward, (y, tokens)), (scores.backward, (y, tokens, two))]


def test_calls_reach_the_device_and_stream_of_the_operator(machine):
    calls = _calls(machine.on(1))
    for call, args in calls:
        for now in (0, 1):
            machine.on(now)
            machine.calls.clear()
            call(*args)
            assert [d for _, d, _ in machine.calls] == [1] and machine.now == now, call
        call(*args, stream=Stream(7, Device("cuda", 1)))
        assert machine.calls[-1][2][-1] == 7
        with pytest.raises(hadfl.HadflError, match="stream"):
            call(*args, stream=Stream(7, Device("cuda", 0)))


def test_the_binding_refuses_what_the_library_cannot_see(machine):
    device = machine.on(0)
    t = lambda *s, dtype="f32", **k: Tensor(s, dtype, k.pop("device", device), **k)  # noqa: E731
    drop, dense, scores = _plans()
    x, w, y, tokens = t(2, 3, 8), t(2, 8, 16), t(2, 3, 16), t(2, 3, 2, dtype="i32")
    wrong = [lambda: drop.forward(t(2, 3, 9)), lambda: drop.forward(x, residual=t(2, 3, 8, dtype="bf16")), lambda: drop.forward(x, seed=-1), lambda: drop.forward(x, call=1 << 64),
             lambda: drop.forward(x, counter=t(1, dtype="i32")), lambda: drop.forward(x, counter=t(2, dtype="i64")), lambda: drop.forward(x, counter=t(1, dtype="i64", device=Device("cuda", 1))),
             lambda: dense.forward(x, t(2, 16, 8)), lambda: dense.forward(x, w, bias=t(2, 8)), lambda: dense.forward(x, w, pre=x), lambda: dense.backward(y, hadfl.PackedRows(2, 3, 9), w, y),
             lambda: scores.forward(y), lambda: scores.forward(y, t(2, 3, 2)), lambda: scores.forward(y, tokens, top=t(2, 3, 3)), lambda: scores.forward(y, tokens, stats=t(2, 3, 2)),
             lambda: hadfl.DenseLayer(2, 3, 8, 16, activation="tanh")]
    for call in wrong:
        with pytest.raises(hadfl.HadflError) as e:
            call()
        assert e.value.status == hadfl.EINVAL
    assert not machine.calls
    with pytest.raises(hadfl.HadflError, match="grad=False") as e:
        hadfl.DenseLayer(2, 3, 8, 16, grad=False).backward(y, x, w)
    assert e.value.status == hadfl.ESTATE
    for stats in (None, False):                               # no forward pass has left any
        with pytest.raises(hadfl.HadflError, match="forward") as e:
            scores.backward(y, tokens, t(2, 3, 2), stats=stats)
        assert e.value.status == hadfl.ESTATE
    scores.forward(y, tokens, stats=False)
    with pytest.raises(hadfl.HadflError, match="forward"):
        scores.backward(y, tokens, t(2, 3, 2))
    for size in ((1 << 32) + 2, -(1 << 32) + 2, 1 << 31):
        for make, sizes in ((hadfl.DenseLayer, 4), (hadfl.TokenScores, 5)):
            for k in range(sizes):
                with pytest.raises(hadfl.HadflError, match="32 bits"):
                    make(*[size if j == k else 2 for j in range(sizes)])
        with pytest.raises(hadfl.HadflError, match="32 bits"):
            hadfl.Dropout(2, size, 2, 0.5)


def test_inputs_that_ask_for_a_graph_are_refused_where_a_result_would_lack_it(machine):
    device = machine.on(0)
    drop, dense, scores = _plans()
    for which in range(4):
        t = lambda k, *s, dtype="f32": Tensor(s, dtype, device, requires_grad=k == which)  # noqa: E731
        ins = ((drop.forward, (t(0, 2, 3, 8), t(1, 2, 3, 8)), 2), (dense.forward, (t(0, 2, 3, 8), t(1, 2, 8, 16), t(2, 2, 16), t(3, 2, 3, 16)), 4),
               (scores.forward, (t(0, 2, 3, 16), Tensor((2, 3, 2), "i32", device)), 1))
        for call, args, inputs in ins:
            machine.grad_mode, before = True, len(machine.calls)
            if which < inputs:
                with pytest.raises(hadfl.HadflError, match="no_grad"):
                    call(*args)
                assert len(machine.calls) == before
            machine.grad_mode = False
            call(*args)
