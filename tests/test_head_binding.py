"""The binding's classes of the head's operators, on a CPU: what they pass to the library, on which device, and what they refuse.  torch's
device side and the library are stood in for; tensors are shapes, strides and addresses."""
import itertools
import types

import pytest

from paper_2111_08274_amd import hadfl


class Device:
    def __init__(self, kind, index):
        self.type, self.index = kind, index

    def __eq__(self, other):
        return (self.type, self.index) == (other.type, other.index)


class Tensor:
    def __init__(self, shape, dtype, device, requires_grad=False, at=1 << 20):
        self.shape, self.dtype, self.device, self.requires_grad, self.at = tuple(shape), dtype, device, requires_grad, at

    def stride(self):
        out, step = [], 1
        for s in reversed(self.shape):
            out.append(step)
            step *= s
        return tuple(reversed(out))

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.at

    def record_stream(self, s):
        pass


class Stream:
    def __init__(self, handle, device):
        self.cuda_stream, self.device = handle, device

    def __enter__(self):
        return self

    def __exit__(self, *a):
        pass


class Machine:
    """Two devices; the library writes down on which of them each call came, to which stream."""

    def __init__(self, monkeypatch):
        import torch
        self.now, self.calls, self.grad_mode = 0, [], True
        machine = self

        class Guard:
            def __init__(self, d):
                self.d = d if isinstance(d, int) else d.index

            def __enter__(self):
                self.before, machine.now = machine.now, self.d

            def __exit__(self, *a):
                machine.now = self.before

        fake = types.ModuleType("torch")
        fake.float32, fake.bfloat16, fake.uint8, fake.int32 = "f32", "bf16", "u8", "i32"
        fake.device = Device
        room = itertools.count(16 << 20, 1 << 20)
        fake.empty = lambda shape, dtype, device: Tensor(shape if isinstance(shape, tuple) else (shape,), dtype, device, at=next(room))
        fake.is_grad_enabled = lambda: machine.grad_mode
        fake._C = types.SimpleNamespace()
        fake.cuda = types.SimpleNamespace(current_device=lambda: machine.now, device=Guard, stream=lambda s: s,
                                          current_stream=lambda i=None: Stream(0, Device("cuda", machine.now if i is None else i if isinstance(i, int) else i.index)))
        real = hadfl.lib()
        entries = {name: (lambda *a, _name=name: (machine.calls.append((_name, machine.now, a)), 0)[1])
                   for name in hadfl.EXPORTS if name.startswith(("hadfl_norm_", "hadfl_pack", "hadfl_unpack", "hadfl_dense", "hadfl_loss"))}
        for name in ("hadfl_norm_workspace", "hadfl_packed_bytes", "hadfl_dense_workspace", "hadfl_loss_workspace", "hadfl_last_error"):
            entries[name] = getattr(real, name)
        monkeypatch.setattr(hadfl, "_lib", types.SimpleNamespace(**entries))
        monkeypatch.setitem(__import__("sys").modules, "torch", fake)
        assert torch is not fake

    def on(self, index):
        self.now = index
        return Device("cuda", index)


@pytest.fixture
def machine(monkeypatch):
    return Machine(monkeypatch)


def _calls(device, n=2, rows=3, f=8, v=16):
    """One call of every kind: (operator, method, arguments)"""
    t = lambda *s, dtype="f32": Tensor(s, dtype, device)  # noqa: E731
    norm, kept, dense, loss = hadfl.LayerNorm(n, rows, f), hadfl.PackedRows(n, rows, f), hadfl.DenseGrad(n, rows, f, v), hadfl.ClassLoss(n, rows, f, v)
    x, w, y, vec = t(n, rows, f), t(n, f, v), t(n, rows, dtype="i32"), t(n, f)
    return [(norm.forward, (x, vec, vec)), (norm.backward, (x, x, vec)), (kept.pack, (x,)), (kept.unpack, ()), (norm.backward, (x, kept, vec)),
            (dense.backward, (kept, t(n, rows, v))), (loss.loss, (x, w, y)), (loss.grad, (x, w, y))]


def test_calls_reach_the_device_of_the_operator(machine):
    # a stream's handle does not name its device (the default one is 0 on all): a call from a thread on another device
    calls = _calls(machine.on(1))
    for now in (0, 1):
        machine.on(now)
        for call, args in calls:
            machine.calls.clear()
            call(*args)
            assert [d for _, d, _ in machine.calls] == [1] and machine.now == now, call


def test_a_stream_of_another_device_is_refused(machine):
    calls = _calls(machine.on(1))
    for call, args in calls:
        machine.calls.clear()
        call(*args, stream=Stream(7, Device("cuda", 1)))
        with pytest.raises(hadfl.HadflError, match="stream"):
            call(*args, stream=Stream(7, Device("cuda", 0)))
        assert len(machine.calls) == 1


def test_a_checkpoint_of_another_device_or_shape_is_refused(machine):
    kept, other = hadfl.PackedRows(2, 3, 8), hadfl.PackedRows(2, 3, 9)
    device = machine.on(1)
    norm, dense = hadfl.LayerNorm(2, 3, 8), hadfl.DenseGrad(2, 3, 8, 16)
    for wrong in (kept, other):
        with pytest.raises(hadfl.HadflError, match="checkpoint"):
            norm.backward(Tensor((2, 3, 8), "f32", device), wrong, Tensor((2, 8), "f32", device))
        with pytest.raises(hadfl.HadflError, match="checkpoint"):
            dense.backward(wrong, Tensor((2, 3, 16), "f32", device))
    assert not machine.calls


@pytest.mark.parametrize("size", [(1 << 32) + 2, -(1 << 32) + 2, 1 << 31, (1 << 64) + 2])
def test_sizes_that_a_32_bit_field_cannot_hold_are_refused(machine, size):
    # ctypes would keep the low 32 bits: an operator of two rows for tensors of 2^32 + 2
    makers = [(hadfl.LayerNorm, 3), (hadfl.PackedRows, 3), (hadfl.DenseGrad, 4), (hadfl.ClassLoss, 4)]
    for make, sizes in makers:
        make(*[2] * sizes)
        for i in range(sizes + 1):
            args = [2] * sizes + [0]
            args[i] = size
            with pytest.raises(hadfl.HadflError, match="32 bits"):
                make(*args)


def test_a_db_that_is_given_is_written_without_a_bias_too(machine):
    device = machine.on(0)
    loss = hadfl.ClassLoss(2, 3, 8, 16)
    t = lambda *s, dtype="f32": Tensor(s, dtype, device)  # noqa: E731
    x, w, y, db = t(2, 3, 8), t(2, 8, 16), t(2, 3, dtype="i32"), t(2, 16)
    for kw, is_out in ((dict(), False), (dict(db=db), True), (dict(db=db, want=("dx", "dw")), False), (dict(bias=t(2, 16)), True)):
        machine.calls.clear()
        out = loss.grad(x, w, y, **kw)[4]
        passed = machine.calls[0][2][9]                       # the address of db's hadfl_rows
        assert (out is not None) == is_out == (passed is not None), kw
        assert "db" not in kw or out is None or out is db


def test_statistics_of_the_norm_are_the_forward_pass_s_own(machine):
    # by default the object's own; a pass that leaves none keeps the last ones; a pair of the caller's for passes in flight together
    device = machine.on(0)
    norm = hadfl.LayerNorm(2, 3, 8)
    x, vec = Tensor((2, 3, 8), "f32", device), Tensor((2, 8), "f32", device)
    mine = Tensor((2, 3), "f32", device, at=5 << 20), Tensor((2, 3), "f32", device, at=6 << 20)
    with pytest.raises(hadfl.HadflError, match="forward") as e:
        norm.backward(x, x, vec)
    assert e.value.status == hadfl.ESTATE
    norm.forward(x, vec, vec, stats=False)
    norm.forward(x, vec, vec, stats=mine)
    with pytest.raises(hadfl.HadflError, match="forward"):
        norm.backward(x, x, vec)
    norm.backward(x, x, vec, stats=mine)
    own = norm.mean.data_ptr(), norm.rstd.data_ptr()
    norm.forward(x, vec, vec)
    norm.backward(x, x, vec)
    got = [(name, a[5:7]) for name, _, a in machine.calls]
    f, b = "hadfl_norm_forward", "hadfl_norm_backward"
    assert got == [(f, (None, None)), (f, (5 << 20, 6 << 20)), (b, (5 << 20, 6 << 20)), (f, own), (b, own)]
    for wrong in ((mine[0], Tensor((2, 4), "f32", device)), (Tensor((2, 3), "bf16", device), mine[1]), (mine[0], Tensor((2, 3), "f32", Device("cuda", 1)))):
        with pytest.raises(hadfl.HadflError):
            norm.forward(x, vec, vec, stats=wrong)
        with pytest.raises(hadfl.HadflError):
            norm.backward(x, x, vec, stats=wrong)
    assert hadfl.LayerNorm(2, 0, 8).backward(Tensor((2, 0, 8), "f32", device), Tensor((2, 0, 8), "f32", device), vec)      # nothing to take from


def test_inputs_that_ask_for_a_graph_are_refused_where_a_result_would_lack_it(machine):
    # forward passes hand out tensors that autograd would take for constants; the gradient calls give the gradients themselves
    device = machine.on(0)
    norm, loss, kept, dense = hadfl.LayerNorm(2, 3, 8), hadfl.ClassLoss(2, 3, 8, 16), hadfl.PackedRows(2, 3, 8), hadfl.DenseGrad(2, 3, 8, 16)
    for which in range(4):
        t = lambda i, *s: Tensor(s, "f32", device, requires_grad=i == which)  # noqa: E731
        labels = Tensor((2, 3), "i32", device)
        norm_in, loss_in = (t(0, 2, 3, 8), t(1, 2, 8), t(2, 2, 8)), (t(0, 2, 3, 8), t(1, 2, 8, 16), labels, t(2, 2, 16))
        for call, args in ((norm.forward, norm_in), (loss.loss, loss_in)):
            machine.grad_mode, before = True, len(machine.calls)
            if which < 3:
                with pytest.raises(hadfl.HadflError, match="no_grad") as e:
                    call(*args)
                assert e.value.status == hadfl.EINVAL and len(machine.calls) == before
            else:
                call(*args)
            machine.grad_mode = False
            call(*args)
        machine.grad_mode = True
        norm.backward(norm_in[0], norm_in[0], norm_in[1])
        loss.grad(*loss_in)
        dense.backward(kept.pack(norm_in[0]), t(0, 2, 3, 16))
