"""Thin ctypes binding over libhadfl.so -- argument marshalling only; every step of the cycle runs in the
library's HIP kernels.  PyTorch supplies device memory and the stream.  There is no fallback: if the library
is not built, loading raises."""
import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libhadfl.so")

OK, EINVAL, ENOMEM, EDEVICE, ESTATE, EUNSUPPORTED = range(6)
STATUS_NAMES = ("HADFL_OK", "HADFL_EINVAL", "HADFL_ENOMEM", "HADFL_EDEVICE", "HADFL_ESTATE", "HADFL_EUNSUPPORTED")
NET_MLP, NET_CNN2, NET_RESNET18, NET_VGG16, NET_NONE, NET_CUSTOM = range(6)
NET_IDS = {"mlp": NET_MLP, "cnn2": NET_CNN2, "resnet18": NET_RESNET18, "vgg16": NET_VGG16, "none": NET_NONE,
           "custom": NET_CUSTOM}
KIND_NAMES = ("weight", "bias", "gamma", "beta", "running_mean", "running_var")


class HadflOp(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("type", "in0", "in1", "k", "stride", "pad", "cout", "bias")]


class HadflConfig(ctypes.Structure):
    _fields_ = [("n_replicas", ctypes.c_int32), ("n_select", ctypes.c_int32), ("net", ctypes.c_int32),
                ("bf16", ctypes.c_int32), ("batch", ctypes.c_int32), ("n_samples", ctypes.c_int32),
                ("in_dim", ctypes.c_int32 * 3), ("n_classes", ctypes.c_int32), ("lr", ctypes.c_float),
                ("momentum", ctypes.c_float), ("t_sync", ctypes.c_int32), ("steps_per_unit", ctypes.c_int32),
                ("weight_mode", ctypes.c_int32), ("n_custom_ops", ctypes.c_int32), ("seed", ctypes.c_uint64),
                ("m_none", ctypes.c_int64), ("custom_ops", ctypes.POINTER(HadflOp))]


class HadflTensorInfo(ctypes.Structure):
    _fields_ = [("offset", ctypes.c_int64), ("count", ctypes.c_int64), ("kind", ctypes.c_int32),
                ("fan_in", ctypes.c_int32)]


class HadflKernelTime(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 48), ("launches", ctypes.c_int64), ("total_ms", ctypes.c_double),
                ("flops", ctypes.c_double), ("bytes", ctypes.c_double)]


class HadflRows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("replica_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64)]


class HadflNorm(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_replicas", "n_rows", "n_features", "bf16")] + [("eps", ctypes.c_float)]


class HadflPack(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_replicas", "n_rows", "n_features", "bf16")]


class HadflDense(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_replicas", "n_rows", "n_in", "n_out", "bf16")]


class HadflLoss(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_replicas", "n_rows", "n_features", "n_classes", "bf16")]


class HadflDraw(ctypes.Structure):
    _fields_ = [("seed", ctypes.c_uint64), ("call", ctypes.c_uint64), ("counter", ctypes.c_void_p)]


class HadflDropout(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_replicas", "n_rows", "n_features", "bf16")] + [("p", ctypes.c_float)]


class HadflLayer(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_replicas", "n_rows", "n_in", "n_out", "bf16", "activation")] + [("drop", ctypes.c_float)]


class HadflScores(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_replicas", "n_rows", "n_classes", "n_tokens", "n_top", "bf16")]


OPT_SIDE_STREAM, OPT_TILE_HINT = 0, 1
ACTIVATIONS = ("none", "relu", "gelu", "silu")

EXPORTS = ("hadfl_param_count", "hadfl_param_layout", "hadfl_workspace_bytes", "hadfl_init_replicas",
           "hadfl_local_steps", "hadfl_select", "hadfl_aggregate", "hadfl_step_counts", "hadfl_steps_from_times",
           "hadfl_set_lr", "hadfl_set_steps", "hadfl_set_params", "hadfl_get_momentum", "hadfl_set_momentum",
           "hadfl_set_option", "hadfl_select_static",
           "hadfl_select_group", "hadfl_aggregate_group", "hadfl_predict_versions",
           "hadfl_select_real", "hadfl_get_predicted", "hadfl_get_steps", "hadfl_get_versions",
           "hadfl_get_selected", "hadfl_get_params", "hadfl_get_losses", "hadfl_profile_enable",
           "hadfl_profile_read", "hadfl_last_error", "hadfl_destroy",
           "hadfl_norm_workspace", "hadfl_norm_forward", "hadfl_norm_backward", "hadfl_packed_bytes", "hadfl_pack_rows",
           "hadfl_unpack_rows", "hadfl_dense_workspace", "hadfl_dense_grad_packed", "hadfl_loss_workspace",
           "hadfl_loss_forward", "hadfl_loss_grad", "hadfl_dropout_rows", "hadfl_layer_workspace", "hadfl_layer_forward",
           "hadfl_layer_backward", "hadfl_scores_workspace", "hadfl_scores_forward", "hadfl_scores_backward")

_lib = None


class HadflError(RuntimeError):
    def __init__(self, status, text):
        super().__init__("%s: %s" % (STATUS_NAMES[status] if 0 <= status < 6 else status, text))
        self.status = status


def lib():
    """Loads libhadfl.so (built in-tree by paper_2111_08274_amd.build).  Raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libhadfl.so is not built: run `python -m paper_2111_08274_amd.build`")
        # PyTorch ships its own HIP runtime; load it first so the library binds to the same runtime instance
        # that owns the tensors and streams handed to it (two runtimes in one process do not share devices).
        import torch  # noqa: F401
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64p = ctypes.c_void_p, ctypes.c_int32, ctypes.POINTER(ctypes.c_int64)
        cfgp = ctypes.POINTER(HadflConfig)
        L.hadfl_param_count.argtypes = [cfgp, i64p, i64p, i64p]
        L.hadfl_param_layout.argtypes = [cfgp, ctypes.POINTER(HadflTensorInfo), i32, ctypes.POINTER(i32)]
        L.hadfl_workspace_bytes.argtypes = [cfgp, ctypes.POINTER(ctypes.c_size_t), ctypes.POINTER(ctypes.c_size_t)]
        L.hadfl_init_replicas.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, vp, ctypes.POINTER(vp)]
        L.hadfl_local_steps.argtypes = [vp]
        L.hadfl_select.argtypes = [vp, vp, vp, ctypes.c_uint64]
        L.hadfl_aggregate.argtypes = [vp, i32]
        L.hadfl_set_steps.argtypes = [vp, vp]
        L.hadfl_step_counts.argtypes = [vp, i32, i32, i32, vp]
        L.hadfl_steps_from_times.argtypes = [vp, i32, i32, ctypes.c_double, i32, i32, vp]
        L.hadfl_set_params.argtypes = [vp, i32, vp, ctypes.c_size_t]
        L.hadfl_get_momentum.argtypes = [vp, i32, vp, ctypes.c_size_t]
        L.hadfl_set_momentum.argtypes = [vp, i32, vp, ctypes.c_size_t]
        L.hadfl_set_option.argtypes = [vp, i32, i32]
        L.hadfl_select_static.argtypes = [vp, vp, i32, i32, i32, ctypes.c_uint64, ctypes.c_uint64, vp, vp, vp, vp]
        L.hadfl_set_lr.argtypes = [vp, ctypes.c_float]
        L.hadfl_select_group.argtypes = [vp, vp, vp, i32, ctypes.c_uint64]
        L.hadfl_aggregate_group.argtypes = [vp, vp]
        L.hadfl_predict_versions.argtypes = [vp, vp, ctypes.c_double, i32]
        L.hadfl_select_real.argtypes = [vp, vp, vp, ctypes.c_uint64]
        L.hadfl_get_predicted.argtypes = [vp, vp]
        L.hadfl_get_steps.argtypes = [vp, vp]
        L.hadfl_get_versions.argtypes = [vp, vp, vp]
        L.hadfl_get_selected.argtypes = [vp, vp, ctypes.POINTER(i32), vp, vp]
        L.hadfl_get_params.argtypes = [vp, i32, vp, ctypes.c_size_t]
        L.hadfl_get_losses.argtypes = [vp, vp]
        L.hadfl_profile_enable.argtypes = [vp, i32]
        L.hadfl_profile_read.argtypes = [vp, ctypes.POINTER(HadflKernelTime), i32, ctypes.POINTER(i32)]
        # descriptors and tensors of the head's operators go by address (_Operator keeps the structs): converting typed
        # pointers costs about as much as a launch
        sizep = ctypes.POINTER(ctypes.c_size_t)
        L.hadfl_norm_workspace.argtypes = L.hadfl_packed_bytes.argtypes = L.hadfl_dense_workspace.argtypes = [vp, sizep]
        L.hadfl_loss_workspace.argtypes = [vp, i32, sizep]
        L.hadfl_norm_forward.argtypes = [vp] * 8
        L.hadfl_norm_backward.argtypes = [vp] * 12
        L.hadfl_pack_rows.argtypes = L.hadfl_unpack_rows.argtypes = [vp] * 4
        L.hadfl_dense_grad_packed.argtypes = [vp] * 7
        L.hadfl_loss_forward.argtypes = [vp] * 9
        L.hadfl_loss_grad.argtypes = [vp] * 12
        L.hadfl_dropout_rows.argtypes = [vp] * 6
        L.hadfl_layer_workspace.argtypes = [vp, i32, sizep]
        L.hadfl_layer_forward.argtypes = [vp] * 10
        L.hadfl_layer_backward.argtypes = [vp] * 12
        L.hadfl_scores_workspace.argtypes = [vp, sizep]
        L.hadfl_scores_forward.argtypes = [vp] * 10
        L.hadfl_scores_backward.argtypes = [vp] * 8
        L.hadfl_last_error.argtypes = [vp]
        L.hadfl_last_error.restype = ctypes.c_char_p
        L.hadfl_destroy.argtypes = [vp]
        L.hadfl_destroy.restype = None
        for name in EXPORTS:
            if name not in ("hadfl_last_error", "hadfl_destroy"):
                getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def make_config(n_replicas, n_select, net="none", bf16=0, batch=1, n_samples=1, in_shape=(1, 1, 1), n_classes=10,
                lr=0.01, momentum=0.0, t_sync=1, steps_per_unit=1, weight_mode=0, seed=2021, m_none=0,
                custom_ops=None):
    """custom_ops: rows (type, in0, in1, k, stride, pad, cout, bias)."""
    c = HadflConfig()
    c.n_replicas, c.n_select = int(n_replicas), int(n_select)
    c.net = NET_IDS[net] if isinstance(net, str) else int(net)
    c.bf16, c.batch, c.n_samples = int(bf16), int(batch), int(n_samples)
    c.in_dim[0], c.in_dim[1], c.in_dim[2] = (int(v) for v in in_shape)
    c.n_classes, c.lr, c.momentum = int(n_classes), float(lr), float(momentum)
    c.t_sync, c.steps_per_unit, c.weight_mode = int(t_sync), int(steps_per_unit), int(weight_mode)
    c.seed, c.m_none = int(seed), int(m_none)
    c._keep = None
    if custom_ops is not None:
        rows = np.asarray(custom_ops, dtype=np.int32).reshape(-1, 8)
        arr = (HadflOp * len(rows))()
        for i, r in enumerate(rows):
            arr[i] = HadflOp(*[int(v) for v in r])
        c._keep = arr
        c.custom_ops = ctypes.cast(arr, ctypes.POINTER(HadflOp))
        c.n_custom_ops = len(rows)
    return c


def _check(status, ctx=None):
    if status != OK:
        raise HadflError(status, lib().hadfl_last_error(ctx).decode())


def param_count(cfg):
    a, b, c = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
    _check(lib().hadfl_param_count(ctypes.byref(cfg), ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)))
    return a.value, b.value, c.value


def param_layout(cfg):
    n = ctypes.c_int32()
    _check(lib().hadfl_param_layout(ctypes.byref(cfg), None, 0, ctypes.byref(n)))
    rows = (HadflTensorInfo * n.value)()
    _check(lib().hadfl_param_layout(ctypes.byref(cfg), rows, n.value, ctypes.byref(n)))
    return [(r.offset, r.count, KIND_NAMES[r.kind], r.fan_in) for r in rows]


def workspace_bytes(cfg):
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().hadfl_workspace_bytes(ctypes.byref(cfg), ctypes.byref(a), ctypes.byref(b)))
    return a.value, b.value


def _np_ptr(a):
    return a.ctypes.data_as(ctypes.c_void_p)


def step_counts(ratio, t_sync=1, steps_per_unit=1):
    """The step-count rule from computing-power ratios (host only) -> int32[n]."""
    r = np.ascontiguousarray(ratio, dtype=np.int32)
    out = np.zeros(r.size, dtype=np.int32)
    _check(lib().hadfl_step_counts(_np_ptr(r), int(r.size), int(t_sync), int(steps_per_unit), _np_ptr(out)))
    return out


def steps_from_times(times, e_warmup, quantum, t_sync=1, steps_per_unit=1):
    """Step counts from measured warm-up times (host only) -> int32[n]."""
    t = np.ascontiguousarray(times, dtype=np.float64)
    out = np.zeros(t.size, dtype=np.int32)
    _check(lib().hadfl_steps_from_times(_np_ptr(t), int(t.size), int(e_warmup), float(quantum), int(t_sync),
                                        int(steps_per_unit), _np_ptr(out)))
    return out


def select_static(versions, n_select, seed, cycle, selected, flag, weights, avail=None, weight_mode=0, stream=None):
    """hadfl_select_static on torch device tensors the CALLER has allocated: versions int32[n], avail uint8[n] or None;
    outputs selected int32[n_select], flag uint8[n], weights float32[n].  The library allocates nothing."""
    import torch
    n = versions.numel()
    assert versions.dtype == torch.int32 and versions.is_cuda and versions.is_contiguous()
    assert selected.dtype == torch.int32 and selected.numel() >= n_select and selected.is_cuda
    assert flag.dtype == torch.uint8 and flag.numel() >= n and flag.is_cuda
    assert weights.dtype == torch.float32 and weights.numel() >= n and weights.is_cuda
    if avail is not None:
        assert avail.dtype == torch.uint8 and avail.numel() == n and avail.is_cuda
    st = (torch.cuda.current_stream() if stream is None else stream).cuda_stream
    _check(lib().hadfl_select_static(versions.data_ptr(), avail.data_ptr() if avail is not None else None, int(n),
                                     int(n_select), int(weight_mode), int(seed), int(cycle), selected.data_ptr(),
                                     flag.data_ptr(), weights.data_ptr(), st))


class Context:
    """One set of replicas on the current torch device.  Holds the torch tensors the library works in."""

    def __init__(self, cfg, ratio, w0=None, x=None, y=None, replicas=None, stream=None, options=None):
        import torch
        self.cfg = cfg
        self.m_train, self.m_total, self.row_stride = param_count(cfg)
        pb, sb = workspace_bytes(cfg)
        dev = torch.device("cuda", torch.cuda.current_device())
        if replicas is None:
            replicas = torch.empty(pb // 4, dtype=torch.float32, device=dev)
        assert replicas.numel() * 4 >= pb and replicas.is_contiguous()
        self.replicas = replicas
        self.scratch = torch.empty(sb, dtype=torch.uint8, device=dev)
        self.w0 = None if w0 is None else torch.as_tensor(w0, dtype=torch.float32).to(dev).contiguous()
        self.x = None if x is None else (x if hasattr(x, "data_ptr") else torch.as_tensor(x)).to(dev).contiguous()
        self.y = None if y is None else (y if hasattr(y, "data_ptr") else torch.as_tensor(y)).to(dev).to(torch.int32).contiguous()
        if self.w0 is not None:
            assert self.w0.numel() == self.m_total
        self.stream = torch.cuda.current_stream() if stream is None else stream
        ratio = np.ascontiguousarray(ratio, dtype=np.int32)
        assert len(ratio) == cfg.n_replicas
        h = ctypes.c_void_p()
        torch.cuda.synchronize()
        _check(lib().hadfl_init_replicas(ctypes.byref(cfg), self.w0.data_ptr() if self.w0 is not None else None,
                                         self.replicas.data_ptr(), self.scratch.data_ptr(),
                                         self.x.data_ptr() if self.x is not None else None,
                                         self.y.data_ptr() if self.y is not None else None,
                                         _np_ptr(ratio), self.stream.cuda_stream, ctypes.byref(h)))
        self.h = h
        for opt, value in (options or {}).items():
            self.set_option(opt, value)

    def set_option(self, option, value):
        _check(lib().hadfl_set_option(self.h, int(option), int(value)), self.h)

    def set_params(self, replica, values):
        v = np.ascontiguousarray(values, dtype=np.float32)
        _check(lib().hadfl_set_params(self.h, int(replica), _np_ptr(v), v.size), self.h)

    def momentum(self, replica, n=None):
        out = np.zeros(self.m_train if n is None else n, dtype=np.float32)
        _check(lib().hadfl_get_momentum(self.h, int(replica), _np_ptr(out), out.size), self.h)
        return out

    def set_momentum(self, replica, values):
        v = np.ascontiguousarray(values, dtype=np.float32)
        _check(lib().hadfl_set_momentum(self.h, int(replica), _np_ptr(v), v.size), self.h)

    def close(self):
        if getattr(self, "h", None):
            lib().hadfl_destroy(self.h)
            self.h = None

    def __del__(self):
        # at interpreter shutdown module globals may already be gone; the process is ending anyway
        try:
            self.close()
        except TypeError:
            pass

    def local_steps(self):
        _check(lib().hadfl_local_steps(self.h), self.h)

    def select(self, cycle, versions=None, avail=None):
        """versions: torch int32 device tensor or None; avail: host array of bytes or None."""
        av = None if avail is None else np.ascontiguousarray(avail, dtype=np.uint8)
        if versions is not None:
            assert versions.dtype.__str__() == "torch.int32" and versions.is_cuda and versions.numel() == self.cfg.n_replicas
        _check(lib().hadfl_select(self.h, versions.data_ptr() if versions is not None else None,
                                  _np_ptr(av) if av is not None else None, int(cycle)), self.h)

    def set_lr(self, lr):
        _check(lib().hadfl_set_lr(self.h, float(lr)), self.h)

    def set_steps(self, steps):
        st = np.ascontiguousarray(steps, dtype=np.int32)
        assert st.size == self.cfg.n_replicas
        _check(lib().hadfl_set_steps(self.h, _np_ptr(st)), self.h)

    def predict_versions(self, alpha, horizon=1, versions=None):
        """versions: torch int32 device tensor or None (the counters of the last local_steps)."""
        if versions is not None:
            assert versions.dtype.__str__() == "torch.int32" and versions.is_cuda and versions.numel() == self.cfg.n_replicas
        _check(lib().hadfl_predict_versions(self.h, versions.data_ptr() if versions is not None else None,
                                            float(alpha), int(horizon)), self.h)

    def select_real(self, cycle, versions=None, avail=None):
        """versions: torch float64 device tensor or None (the forecast of predict_versions)."""
        av = None if avail is None else np.ascontiguousarray(avail, dtype=np.uint8)
        if versions is not None:
            assert versions.dtype.__str__() == "torch.float64" and versions.is_cuda and versions.numel() == self.cfg.n_replicas
        _check(lib().hadfl_select_real(self.h, versions.data_ptr() if versions is not None else None,
                                       _np_ptr(av) if av is not None else None, int(cycle)), self.h)

    def predicted(self):
        out = np.zeros(self.cfg.n_replicas, dtype=np.float64)
        _check(lib().hadfl_get_predicted(self.h, _np_ptr(out)), self.h)
        return out

    def select_group(self, cycle, members, n_select, versions=None):
        mb = np.ascontiguousarray(members, dtype=np.uint8)
        assert mb.size == self.cfg.n_replicas
        if versions is not None:
            assert versions.dtype.__str__() == "torch.int32" and versions.is_cuda and versions.numel() == self.cfg.n_replicas
        _check(lib().hadfl_select_group(self.h, versions.data_ptr() if versions is not None else None, _np_ptr(mb),
                                        int(n_select), int(cycle)), self.h)

    def aggregate_group(self, members):
        mb = np.ascontiguousarray(members, dtype=np.uint8)
        assert mb.size == self.cfg.n_replicas
        _check(lib().hadfl_aggregate_group(self.h, _np_ptr(mb)), self.h)

    def aggregate(self, resync=True):
        _check(lib().hadfl_aggregate(self.h, int(bool(resync))), self.h)

    def steps(self):
        out = np.zeros(self.cfg.n_replicas, dtype=np.int32)
        _check(lib().hadfl_get_steps(self.h, _np_ptr(out)), self.h)
        return out

    def versions(self):
        v = np.zeros(self.cfg.n_replicas, dtype=np.int32)
        c = np.zeros(self.cfg.n_replicas, dtype=np.int64)
        _check(lib().hadfl_get_versions(self.h, _np_ptr(v), _np_ptr(c)), self.h)
        return v, c

    def selected(self):
        sel = np.zeros(self.cfg.n_select, dtype=np.int32)
        cnt = ctypes.c_int32()
        flag = np.zeros(self.cfg.n_replicas, dtype=np.uint8)
        w = np.zeros(self.cfg.n_replicas, dtype=np.float32)
        _check(lib().hadfl_get_selected(self.h, _np_ptr(sel), ctypes.byref(cnt), _np_ptr(flag), _np_ptr(w)), self.h)
        return sel[:cnt.value], flag, w

    def params(self, replica, n=None):
        n = self.m_total if n is None else n
        out = np.zeros(n, dtype=np.float32)
        _check(lib().hadfl_get_params(self.h, int(replica), _np_ptr(out), n), self.h)
        return out

    def losses(self):
        out = np.zeros(self.cfg.n_replicas, dtype=np.float32)
        _check(lib().hadfl_get_losses(self.h, _np_ptr(out)), self.h)
        return out

    def profile(self, on):
        _check(lib().hadfl_profile_enable(self.h, int(on)), self.h)

    def profile_read(self):
        n = ctypes.c_int32()
        rows = (HadflKernelTime * 4096)()
        _check(lib().hadfl_profile_read(self.h, rows, 4096, ctypes.byref(n)), self.h)
        return {rows[i].name.decode(): dict(launches=rows[i].launches, ms=rows[i].total_ms, flops=rows[i].flops,
                                            bytes=rows[i].bytes) for i in range(min(n.value, 4096))}


# ---- operators of a language model's head ----------------------------------------------------------------------------
def _int32(*values):
    """The sizes as the library's structs hold them; ctypes would keep the low 32 bits of any number."""
    out = [int(v) for v in values]
    if any(not -2 ** 31 <= v < 2 ** 31 for v in out):
        raise HadflError(EINVAL, "%s: a size must fit 32 bits" % (values,))
    return out


class _Operator:
    """Sizes, types and working memory of one operator on the current torch device.  Its tensors are torch device tensors
    [replica, row, column] (or [replica, column] for vectors) whose columns are contiguous; other strides are free.  Calls go
    to `stream` or to the device's current one, and the tensors have to be ready there; calls of one object share its working memory
    and must not overlap in time.  Outputs that are not given are allocated, as memory of the stream the call goes to.  autograd records none of the
    calls: a forward pass of tensors that require a gradient is refused in grad mode (an autograd.Function runs outside of it)."""

    def __init__(self, desc, bf16, workspace=None):
        import torch
        self.torch, self.desc = torch, desc
        self.device = torch.device("cuda", torch.cuda.current_device())
        self.dtype = torch.bfloat16 if bf16 else torch.float32
        self._ref = ctypes.addressof(desc)
        self._structs = {}
        # the handle itself where torch offers it; the object around it takes longer to make than a kernel to launch
        self._current = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
        self._device_now = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        self._home, self._own = self._current(self.device.index), []
        self.work = None if workspace is None else self._bytes(workspace)

    def _bytes(self, query):
        n = ctypes.c_size_t()
        _check(query(self._ref, ctypes.byref(n)))
        return self._keep(self.torch.empty(n.value, dtype=self.torch.uint8, device=self.device))

    def _keep(self, t):
        self._own.append(t)
        return t

    def _rows(self, name, t, shape, dtype):
        """The address of the hadfl_rows of a tensor, checked; None stays None."""
        if t is None:
            return None
        if t.dtype != dtype or t.device != self.device or t.shape != shape:
            raise HadflError(EINVAL, "%s must be %s %s on %s, not %s %s on %s" % (name, dtype, shape, self.device, t.dtype, tuple(t.shape), t.device))
        st = t.stride()
        if st[-1] != 1 and shape[-1] > 1:
            raise HadflError(EINVAL, "%s: the columns must be contiguous" % name)
        got = self._structs.get(name)
        if got is None:
            r = HadflRows()
            got = self._structs[name] = (r, ctypes.addressof(r))
        r = got[0]
        r.data, r.replica_stride, r.row_stride = t.data_ptr() or None, st[0], (st[1] if len(st) == 3 else 0)
        return got[1]

    def _plain(self, name, t, shape, dtype):
        """The address of a contiguous tensor, checked."""
        if t is None:
            return None
        if t.dtype != dtype or t.device != self.device or t.shape != shape or not t.is_contiguous():
            raise HadflError(EINVAL, "%s must be contiguous %s %s on %s" % (name, dtype, shape, self.device))
        return t.data_ptr() or None

    def _no_graph(self, *inputs):
        for t in inputs:
            if t is not None and t.requires_grad and self.torch.is_grad_enabled():
                raise HadflError(EINVAL, "an input requires a gradient, which the result would not pass on: call under torch.no_grad()")

    def _kept(self, packed, shape):
        """The address of a checkpoint, checked."""
        if packed.shape != shape or packed.device != self.device:
            raise HadflError(EINVAL, "the checkpoint holds %s on %s, not %s on %s" % (packed.shape, packed.device, shape, self.device))
        return packed.data.data_ptr()

    def _out(self, t, shape, dtype, stream=None):
        if t is not None:
            return t
        if stream is not None:
            with self.torch.cuda.stream(stream):
                return self.torch.empty(shape, dtype=dtype, device=self.device)
        return self.torch.empty(shape, dtype=dtype, device=self.device)

    def _stream(self, stream, *others):
        """The handle of the stream a call goes to.  Away from the stream this object was made on, the allocator is told that
        its memory (and that of the other operators that the call uses) is in use there."""
        if stream is not None and stream.device != self.device:
            raise HadflError(EINVAL, "the stream is one of %s, not of %s" % (stream.device, self.device))
        h = self._current(self.device.index) if stream is None else stream.cuda_stream
        for o in (self,) + others:
            if h != o._home:
                for t in o._own:
                    t.record_stream(self.torch.cuda.current_stream(self.device) if stream is None else stream)
        return h

    def _call(self, entry, *args):
        """A call of the library with the operator's device current, which a stream's handle does not name: the default one is 0 on all."""
        if self._device_now() == self.device.index:
            return _check(entry(self._ref, *args))
        with self.torch.cuda.device(self.device):
            return _check(entry(self._ref, *args))


class LayerNorm(_Operator):
    """Layer norm of [n_replicas, n_rows, n_features] with gamma, beta [n_replicas, n_features] (32-bit), and its gradient.
    backward() takes the rows' statistics that forward() left, in `mean` and `rstd` of this object, which hold those of its last pass, or in a
    pair of the caller's: stats=(mean, rstd), 32-bit [n_replicas, n_rows], given to both.  forward(stats=False) leaves none and keeps what is
    there (an evaluation between a forward pass and its gradient)."""

    def __init__(self, n_replicas, n_rows, n_features, bf16=0, eps=1e-5):
        n, rows, features, bf16 = _int32(n_replicas, n_rows, n_features, bf16)
        super().__init__(HadflNorm(n, rows, features, bf16, float(eps)), bf16, lib().hadfl_norm_workspace)
        self.shape, self.vector = (n, rows, features), (n, features)
        f32 = self.torch.float32
        self.mean = self._keep(self.torch.empty(self.shape[:2], dtype=f32, device=self.device))
        self.rstd = self._keep(self.torch.empty(self.shape[:2], dtype=f32, device=self.device))
        self._left = rows == 0                                # statistics are there

    def _stats(self, stats):
        if stats is None:
            return self.mean.data_ptr() or None, self.rstd.data_ptr() or None
        if stats is False:
            return None, None
        mean, rstd = stats
        return self._plain("mean", mean, self.shape[:2], self.torch.float32), self._plain("rstd", rstd, self.shape[:2], self.torch.float32)

    def forward(self, x, gamma, beta, y=None, stream=None, stats=None):
        f32 = self.torch.float32
        self._no_graph(x, gamma, beta)
        y = self._out(y, self.shape, self.dtype, stream)
        self._call(lib().hadfl_norm_forward, self._rows("x", x, self.shape, self.dtype), self._rows("gamma", gamma, self.vector, f32),
                   self._rows("beta", beta, self.vector, f32), self._rows("y", y, self.shape, self.dtype), *self._stats(stats), self._stream(stream))
        self._left = self._left or stats is None
        return y

    def backward(self, dy, x, gamma, dx=None, dgamma=None, dbeta=None, stream=None, stats=None):
        """x: the tensor given to forward() or the PackedRows that holds it.  -> dx, dgamma, dbeta"""
        f32 = self.torch.float32
        dx, dgamma, dbeta = self._out(dx, self.shape, self.dtype, stream), self._out(dgamma, self.vector, f32, stream), self._out(dbeta, self.vector, f32, stream)
        packed, others = None, ()
        if isinstance(x, PackedRows):
            others, packed, x = (x,), self._kept(x, self.shape), None
        if stats is None and not self._left:
            raise HadflError(ESTATE, "no forward() of this LayerNorm has left its statistics")
        self._call(lib().hadfl_norm_backward, self._rows("dy", dy, self.shape, self.dtype), self._rows("x", x, self.shape, self.dtype),
                   packed, self._rows("gamma", gamma, self.vector, f32), *self._stats(stats), self._rows("dx", dx, self.shape, self.dtype),
                   self._rows("dgamma", dgamma, self.vector, f32), self._rows("dbeta", dbeta, self.vector, f32),
                   self.work.data_ptr(), self._stream(stream, *others))
        return dx, dgamma, dbeta


class PackedRows(_Operator):
    """An activation checkpoint in 8 bits of [n_replicas, n_rows, n_features]; bf16: the type that pack() reads and unpack()
    writes."""

    def __init__(self, n_replicas, n_rows, n_features, bf16=0):
        n, rows, features, bf16 = _int32(n_replicas, n_rows, n_features, bf16)
        super().__init__(HadflPack(n, rows, features, bf16), bf16)
        self.shape = (n, rows, features)
        self.data = self._bytes(lib().hadfl_packed_bytes)

    def pack(self, x, stream=None):
        self._call(lib().hadfl_pack_rows, self._rows("x", x, self.shape, self.dtype), self.data.data_ptr(), self._stream(stream))
        return self

    def unpack(self, out=None, stream=None):
        out = self._out(out, self.shape, self.dtype, stream)
        self._call(lib().hadfl_unpack_rows, self.data.data_ptr(), self._rows("out", out, self.shape, self.dtype), self._stream(stream))
        return out


class DenseGrad(_Operator):
    """dW [n_replicas, n_in, n_out] and db [n_replicas, n_out] (32-bit) of a dense layer from its input's PackedRows and dy
    [n_replicas, n_rows, n_out]."""

    def __init__(self, n_replicas, n_rows, n_in, n_out, bf16=0):
        self.n, self.rows, self.n_in, self.n_out, bf16 = _int32(n_replicas, n_rows, n_in, n_out, bf16)
        super().__init__(HadflDense(self.n, self.rows, self.n_in, self.n_out, bf16), bf16, lib().hadfl_dense_workspace)

    def backward(self, packed, dy, dw=None, db=None, bias=True, stream=None):
        """-> dw, db; bias=False leaves db out (None)"""
        f32 = self.torch.float32
        kept = self._kept(packed, (self.n, self.rows, self.n_in))
        dw = self._out(dw, (self.n, self.n_in, self.n_out), f32, stream)
        db = self._out(db, (self.n, self.n_out), f32, stream) if bias else None
        self._call(lib().hadfl_dense_grad_packed, kept, self._rows("dy", dy, (self.n, self.rows, self.n_out), self.dtype),
                   self._rows("dw", dw, (self.n, self.n_in, self.n_out), f32),
                   self._rows("db", db, (self.n, self.n_out), f32), self.work.data_ptr(), self._stream(stream, packed))
        return dw, db


class ClassLoss(_Operator):
    """Softmax cross entropy of a last dense layer over many classes, whose logits are formed in the working memory, a piece of the
    vocabulary at a time: x [n_replicas, n_rows, n_features], w [n_replicas, n_features, n_classes], bias [n_replicas, n_classes]
    (32-bit) or None, labels [n_replicas, n_rows] int32; a label outside [0, n_classes) marks a row that takes no part."""

    def __init__(self, n_replicas, n_rows, n_features, n_classes, bf16=0, grad=True):
        self.n, self.rows, self.features, self.classes, bf16 = _int32(n_replicas, n_rows, n_features, n_classes, bf16)
        self.with_grad, query = bool(grad), lib().hadfl_loss_workspace
        super().__init__(HadflLoss(self.n, self.rows, self.features, self.classes, bf16), bf16, lambda ref, out: query(ref, int(self.with_grad), out))

    def _inputs(self, x, w, labels, bias, row_loss, loss):
        f32, i32 = self.torch.float32, self.torch.int32
        return (self._rows("x", x, (self.n, self.rows, self.features), self.dtype),
                self._rows("w", w, (self.n, self.features, self.classes), self.dtype), self._rows("bias", bias, (self.n, self.classes), f32),
                self._plain("labels", labels, (self.n, self.rows), i32), self._plain("loss", loss, (self.n,), f32),
                self._plain("row_loss", row_loss, (self.n, self.rows), f32))

    def loss(self, x, w, labels, bias=None, loss=None, row_loss=None, stream=None):
        """-> loss [n_replicas] (mean over the labelled rows), row_loss [n_replicas, n_rows]"""
        f32 = self.torch.float32
        self._no_graph(x, w, bias)
        loss, row_loss = self._out(loss, (self.n,), f32, stream), self._out(row_loss, (self.n, self.rows), f32, stream)
        self._call(lib().hadfl_loss_forward, *self._inputs(x, w, labels, bias, row_loss, loss), self.work.data_ptr(), self._stream(stream))
        return loss, row_loss

    def grad(self, x, w, labels, bias=None, loss=None, row_loss=None, dx=None, dw=None, db=None, want=("dx", "dw", "db"), stream=None):
        """-> loss, row_loss, dx, dw, db of the mean losses; what `want` leaves out is None, and so is db where neither it nor a bias is given"""
        if not self.with_grad:
            raise HadflError(ESTATE, "this ClassLoss was made with grad=False")
        f32 = self.torch.float32
        loss, row_loss = self._out(loss, (self.n,), f32, stream), self._out(row_loss, (self.n, self.rows), f32, stream)
        dx = self._out(dx, (self.n, self.rows, self.features), self.dtype, stream) if "dx" in want else None
        dw = self._out(dw, (self.n, self.features, self.classes), self.dtype, stream) if "dw" in want else None
        db = self._out(db, (self.n, self.classes), f32, stream) if "db" in want and (bias is not None or db is not None) else None
        self._call(lib().hadfl_loss_grad, *self._inputs(x, w, labels, bias, row_loss, loss),
                   self._rows("dx", dx, (self.n, self.rows, self.features), self.dtype),
                   self._rows("dw", dw, (self.n, self.features, self.classes), self.dtype),
                   self._rows("db", db, (self.n, self.classes), f32), self.work.data_ptr(), self._stream(stream))
        return loss, row_loss, dx, dw, db


# ---- operators of a next-word model's layers and answers --------------------------------------------------------------
class _Drawing(_Operator):
    """An operator that drops values: which ones is decided by seed and call, whole numbers below 2^64, and a counter, a device
    tensor of one int64 whose value is added to call when the kernels run (one that a captured graph counts up, say)."""

    def _draw(self, seed, call, counter):
        if not self.drops:
            return None
        at = None
        if counter is not None:
            if counter.dtype != self.torch.int64 or counter.device != self.device or counter.numel() != 1:
                raise HadflError(EINVAL, "counter must be one int64 on %s" % (self.device,))
            at = counter.data_ptr()
        if not (0 <= seed < 2 ** 64 and 0 <= call < 2 ** 64):
            raise HadflError(EINVAL, "seed and call must be in [0, 2^64)")
        got = self._structs.get("draw")
        if got is None:
            d = HadflDraw()
            got = self._structs["draw"] = (d, ctypes.addressof(d))
        d = got[0]
        d.seed, d.call, d.counter = int(seed), int(call), at
        return got[1]


class Dropout(_Drawing):
    """Dropout of [n_replicas, n_rows, n_features] with probability p (a multiple of 2^-16, rounded to it), onto a residual if one is
    given.  The mask is never stored: backward() with the forward pass's seed, call and counter draws it again."""

    def __init__(self, n_replicas, n_rows, n_features, p, bf16=0):
        n, rows, features, bf16 = _int32(n_replicas, n_rows, n_features, bf16)
        super().__init__(HadflDropout(n, rows, features, bf16, float(p)), bf16)
        self.shape, self.drops = (n, rows, features), float(p) != 0

    def _run(self, x, residual, y, draw, stream, names=("x", "y")):
        y = self._out(y, self.shape, self.dtype, stream)
        self._call(lib().hadfl_dropout_rows, self._rows(names[0], x, self.shape, self.dtype), self._rows("residual", residual, self.shape, self.dtype),
                   draw, self._rows(names[1], y, self.shape, self.dtype), self._stream(stream))
        return y

    def forward(self, x, residual=None, y=None, seed=0, call=0, counter=None, stream=None):
        """y may be x or the residual"""
        self._no_graph(x, residual)
        return self._run(x, residual, y, self._draw(seed, call, counter), stream)

    def backward(self, dy, dx=None, seed=0, call=0, counter=None, stream=None):
        """-> dx, which may be dy; the residual's gradient is dy"""
        return self._run(dy, None, dx, self._draw(seed, call, counter), stream, ("dy", "dx"))


class DenseLayer(_Drawing):
    """y = residual + dropout(activation(x w + bias)): x [n_replicas, n_rows, n_in], w [n_replicas, n_in, n_out], bias [n_replicas, n_out]
    (32-bit) or None, residual and y [n_replicas, n_rows, n_out]; activation one of ACTIVATIONS ("gelu" is the tanh form, z (1 +
    tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2, not the one of the error function), drop the probability of dropping.  What backward() needs of the forward pass is `pre`, a tensor like y for x w + bias, and the same seed, call and counter."""

    def __init__(self, n_replicas, n_rows, n_in, n_out, bf16=0, activation="none", drop=0.0, grad=True):
        self.n, self.rows, self.n_in, self.n_out, bf16 = _int32(n_replicas, n_rows, n_in, n_out, bf16)
        if activation not in ACTIVATIONS:
            raise HadflError(EINVAL, "activation must be one of %s" % (ACTIVATIONS,))
        self.with_grad, self.drops, query = bool(grad), float(drop) != 0, lib().hadfl_layer_workspace
        super().__init__(HadflLayer(self.n, self.rows, self.n_in, self.n_out, bf16, ACTIVATIONS.index(activation), float(drop)), bf16,
                         lambda ref, out: query(ref, int(self.with_grad), out))

    def forward(self, x, w, bias=None, residual=None, pre=None, y=None, seed=0, call=0, counter=None, stream=None):
        """-> y, which may be the residual; x w + bias is left in `pre` if that is given"""
        self._no_graph(x, w, bias, residual)
        out = (self.n, self.rows, self.n_out)
        y = self._out(y, out, self.dtype, stream)
        self._call(lib().hadfl_layer_forward, self._rows("x", x, (self.n, self.rows, self.n_in), self.dtype),
                   self._rows("w", w, (self.n, self.n_in, self.n_out), self.dtype), self._rows("bias", bias, (self.n, self.n_out), self.torch.float32),
                   self._rows("residual", residual, out, self.dtype), self._draw(seed, call, counter), self._rows("pre", pre, out, self.dtype),
                   self._rows("y", y, out, self.dtype), self.work.data_ptr(), self._stream(stream))
        return y

    def backward(self, dy, x, w, pre=None, dx=None, dw=None, db=None, want=("dx", "dw", "db"), seed=0, call=0, counter=None, stream=None):
        """x: the tensor given to forward() or the PackedRows that holds it (None without dw; w None without dx).  -> dx, dw, db; what
        `want` leaves out is None.  The residual's gradient is dy."""
        if not self.with_grad:
            raise HadflError(ESTATE, "this DenseLayer was made with grad=False")
        rows, weights, out = (self.n, self.rows, self.n_in), (self.n, self.n_in, self.n_out), (self.n, self.rows, self.n_out)
        dx = self._out(dx, rows, self.dtype, stream) if "dx" in want else None
        dw = self._out(dw, weights, self.dtype, stream) if "dw" in want else None
        db = self._out(db, (self.n, self.n_out), self.torch.float32, stream) if "db" in want else None
        packed, others = None, ()
        if isinstance(x, PackedRows):
            others, packed, x = (x,), self._kept(x, rows), None
        self._call(lib().hadfl_layer_backward, self._rows("dy", dy, out, self.dtype), self._rows("pre", pre, out, self.dtype),
                   self._rows("x", x, rows, self.dtype), packed, self._rows("w", w, weights, self.dtype), self._draw(seed, call, counter),
                   self._rows("dx", dx, rows, self.dtype), self._rows("dw", dw, weights, self.dtype),
                   self._rows("db", db, (self.n, self.n_out), self.torch.float32), self.work.data_ptr(), self._stream(stream, *others))
        return dx, dw, db


class TokenScores(_Operator):
    """What logits [n_replicas, n_rows, n_classes] say: log probabilities of tokens [n_replicas, n_rows, n_tokens] int32 (one outside
    [0, n_classes) has none: 0), entropy [n_replicas, n_rows] and the n_top largest, [n_replicas, n_rows, n_top], ties to the lowest
    index.  backward() takes the rows' statistics that forward() left, in `stats` of this object, which holds those of its last pass, or
    in a tensor of the caller's, 32-bit [n_replicas, n_rows, 3], given to both.  forward(stats=False) leaves none and keeps what is there."""

    def __init__(self, n_replicas, n_rows, n_classes, n_tokens=1, n_top=0, bf16=0):
        self.n, self.rows, self.classes, self.tokens, self.top, bf16 = _int32(n_replicas, n_rows, n_classes, n_tokens, n_top, bf16)
        super().__init__(HadflScores(self.n, self.rows, self.classes, self.tokens, self.top, bf16), bf16, lib().hadfl_scores_workspace)
        self.stats = self._keep(self.torch.empty((self.n, self.rows, 3), dtype=self.torch.float32, device=self.device))
        self._left = self.rows == 0                           # statistics are there

    def _stats(self, stats):
        return self.stats.data_ptr() or None if stats is None else None if stats is False else self._plain("stats", stats, (self.n, self.rows, 3), self.torch.float32)

    def forward(self, logits, tokens=None, logp=None, entropy=None, top=None, top_logp=None, stats=None, stream=None):
        """-> logp (None without tokens), entropy, top (int32) and top_logp (None without alternatives)"""
        f32, i32 = self.torch.float32, self.torch.int32
        self._no_graph(logits)
        given, best = (self.n, self.rows, self.tokens), (self.n, self.rows, self.top)
        if self.tokens and tokens is None:
            raise HadflError(EINVAL, "tokens is None")
        logp = self._out(logp, given, f32, stream) if self.tokens else None
        entropy = self._out(entropy, given[:2], f32, stream)
        top, top_logp = (self._out(top, best, i32, stream), self._out(top_logp, best, f32, stream)) if self.top else (None, None)
        self._call(lib().hadfl_scores_forward, self._rows("logits", logits, (self.n, self.rows, self.classes), self.dtype),
                   self._plain("tokens", tokens if self.tokens else None, given, i32), self._plain("logp", logp, given, f32),
                   self._plain("entropy", entropy, given[:2], f32), self._stats(stats), self._plain("top", top, best, i32),
                   self._plain("top_logp", top_logp, best, f32), self.work.data_ptr(), self._stream(stream))
        self._left = self._left or stats is None
        return logp, entropy, top, top_logp

    def backward(self, logits, tokens, dlogp, dentropy=None, dlogits=None, stats=None, stream=None):
        """tokens, dlogp: None without tokens.  -> dlogits, which may be the logits"""
        f32, given, rows = self.torch.float32, (self.n, self.rows, self.tokens), (self.n, self.rows, self.classes)
        if self.tokens and (tokens is None or dlogp is None):
            raise HadflError(EINVAL, "tokens and dlogp must be given")
        if stats is False or (stats is None and not self._left):
            raise HadflError(ESTATE, "no forward() of this TokenScores has left its statistics")
        dlogits = self._out(dlogits, rows, self.dtype, stream)
        self._call(lib().hadfl_scores_backward, self._rows("logits", logits, rows, self.dtype),
                   self._plain("tokens", tokens if self.tokens else None, given, self.torch.int32), self._stats(stats),
                   self._plain("dlogp", dlogp if self.tokens else None, given, f32), self._plain("dentropy", dentropy, given[:2], f32),
                   self._rows("dlogits", dlogits, rows, self.dtype), self._stream(stream))
        return dlogits
