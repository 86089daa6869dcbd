"""Calls of the head's operators read from standard input (JSON) on the stand-in for the HIP runtime (head_launches.cpp, already
built: first argument); writes the status, the text of an error, the working memory and the launches of each.  A process of its own: the stand-in
has to be loaded before the library and torch's HIP runtime must not be.  Tensors are addresses only: nothing reads them."""
import ctypes
import json
import sys
import types

fake = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
fake.check_trace.restype = fake.check_names.restype = ctypes.c_char_p
sys.modules["torch"] = types.ModuleType("torch")
from paper_2111_08274_amd import hadfl  # noqa: E402

AT = 1 << 40


def rows(strides, *shape, at=AT):
    """A tensor of this shape ([n][rows][cols] or [n][cols]), contiguous or with the strides [replica, row]."""
    rep, row = strides or (shape[-1] * (shape[1] if len(shape) == 3 else 1), shape[-1] if len(shape) == 3 else 0)
    return ctypes.byref(hadfl.HadflRows(at, rep, row))


def run(c):
    L, n, t, bf16, at = hadfl.lib(), c.get("n"), c.get("rows"), c.get("bf16", 0), c.get("at", AT)
    size = ctypes.c_size_t()
    fake.check_reset()
    if c["op"] == "dense":
        d = hadfl.HadflDense(n, t, c["inputs"], c["outputs"], bf16)
        status = L.hadfl_dense_workspace(ctypes.byref(d), ctypes.byref(size))
        status = status or L.hadfl_dense_grad_packed(ctypes.byref(d), AT, rows(c.get("dy"), n, t, c["outputs"], at=at), rows(None, n, c["inputs"], c["outputs"]),
                                                     rows(None, n, c["outputs"]), AT, None)
    elif c["op"] in ("pack", "unpack"):
        d = hadfl.HadflPack(n, t, c["features"], bf16)
        status = L.hadfl_packed_bytes(ctypes.byref(d), ctypes.byref(size))
        if c["op"] == "pack":
            status = status or L.hadfl_pack_rows(ctypes.byref(d), rows(c.get("x"), n, t, c["features"]), AT, None)
        else:
            status = status or L.hadfl_unpack_rows(ctypes.byref(d), AT, rows(None, n, t, c["features"]), None)
    elif c["op"] == "norm":
        d, x, v = hadfl.HadflNorm(n, t, c["features"], bf16, 1e-5), rows(c.get("x"), n, t, c["features"]), rows(None, n, c["features"])
        status = L.hadfl_norm_workspace(ctypes.byref(d), ctypes.byref(size))
        status = status or L.hadfl_norm_forward(ctypes.byref(d), x, v, v, rows(None, n, t, c["features"]), AT, AT, None)
        status = status or L.hadfl_norm_backward(ctypes.byref(d), x, x, None, v, AT, AT, rows(None, n, t, c["features"]), v, v, AT, None)
        status = status or L.hadfl_norm_backward(ctypes.byref(d), x, None, AT, v, AT, AT, rows(None, n, t, c["features"]), v, v, AT, None)
    elif c["op"] == "kernels":
        hadfl.lib()
        return fake.check_names().decode().split()
    else:
        d = hadfl.HadflLoss(n, t, c["features"], c["classes"], bf16)
        grad = int(c.get("grad", 1))
        status = L.hadfl_loss_workspace(ctypes.byref(d), grad, ctypes.byref(size))
        x, w = rows(c.get("x"), n, t, c["features"]), rows(c.get("w"), n, c["features"], c["classes"], at=at)
        bias = rows(None, n, c["classes"]) if c.get("bias") else None
        if grad:
            status = status or L.hadfl_loss_grad(ctypes.byref(d), x, w, bias, AT, AT, None, rows(None, n, t, c["features"]), rows(None, n, c["features"], c["classes"]),
                                                 bias, AT, None)
        else:
            status = status or L.hadfl_loss_forward(ctypes.byref(d), x, w, bias, AT, AT, None, AT, None)
    return dict(status=status, text=L.hadfl_last_error(None).decode() if status else "", work=size.value,
                launches=[line.split() for line in fake.check_trace().decode().splitlines()])


json.dump([run(c) for c in json.load(sys.stdin)], sys.stdout)
