"""Calls of the layers' operators read from standard input (JSON) on the stand-in for the HIP runtime (head_launches.cpp, already built: first
argument), as run_head.py does it for the head's; tensors are addresses only."""
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
    rep, row = strides or (shape[-1] * (shape[1] if len(shape) == 3 else 1), shape[-1] if len(shape) == 3 else 0)
    return ctypes.byref(hadfl.HadflRows(at, rep, row))


def run(c):
    L, n, t, bf16 = hadfl.lib(), c.get("n"), c.get("rows"), c.get("bf16", 0)
    size = ctypes.c_size_t()
    fake.check_reset()
    if c["op"] == "kernels":
        return fake.check_names().decode().split()
    draw = ctypes.byref(hadfl.HadflDraw(1, 2, None))
    if c["op"] == "drop":
        d = hadfl.HadflDropout(n, t, c["features"], bf16, 0.1)
        x = rows(c.get("x"), n, t, c["features"])
        status = L.hadfl_dropout_rows(ctypes.byref(d), x, x if c.get("residual") else None, draw, rows(None, n, t, c["features"]), None)
    elif c["op"] == "layer":
        i, o = c["inputs"], c["outputs"]
        d = hadfl.HadflLayer(n, t, i, o, bf16, c.get("act", 0), c.get("drop", 0.0))
        x, w, y = rows(c.get("x"), n, t, i), rows(c.get("w"), n, i, o), rows(c.get("y"), n, t, o)
        status = L.hadfl_layer_workspace(ctypes.byref(d), int(c.get("grad", 0)), ctypes.byref(size))
        if c.get("grad"):
            want = c.get("want", ["dx", "dw", "db"])
            status = status or L.hadfl_layer_backward(ctypes.byref(d), y, y, None if c.get("packed") else x, AT if c.get("packed") else None, w, draw,
                                                      rows(None, n, t, i) if "dx" in want else None, rows(None, n, i, o) if "dw" in want else None,
                                                      rows(None, n, o) if "db" in want else None, AT, None)
        else:
            status = status or L.hadfl_layer_forward(ctypes.byref(d), x, w, None, None, draw, None, rows(None, n, t, o), AT, None)
    else:
        d = hadfl.HadflScores(n, t, c["classes"], c.get("tokens", 1), c.get("top", 0), bf16)
        z = rows(c.get("z"), n, t, c["classes"])
        status = L.hadfl_scores_workspace(ctypes.byref(d), ctypes.byref(size))
        if c.get("grad"):
            status = status or L.hadfl_scores_backward(ctypes.byref(d), z, AT, AT, AT, AT, rows(None, n, t, c["classes"]), None)
        else:
            status = status or L.hadfl_scores_forward(ctypes.byref(d), z, AT, AT, AT, AT, AT, AT, AT, None)
    return dict(status=status, text=L.hadfl_last_error(None).decode() if status else "", work=size.value,
                launches=[line.split() for line in fake.check_trace().decode().splitlines()])


json.dump([run(c) for c in json.load(sys.stdin)], sys.stdout)
