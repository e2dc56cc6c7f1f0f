"""Thin Python binding of the C ABI in include/aet.h (same names, marshalling only).

torch supplies device memory, pinned host memory and the stream; every step of
the method runs inside the library's kernels and host scheduler.
"""
from __future__ import annotations

import ctypes as C

import numpy as np

from . import _lib
from ._lib import AetConfig, AetEvent, AetStats, AetSummary, NEVER_WAIT, STATUS_NAMES  # noqa: F401

FLAG_BORROW_DATA, FLAG_DEBUG_CHECKS, FLAG_KEEP_UPDATE_SUMS, FLAG_STEPWISE_RECURRENCE = 1, 2, 4, 8   # AET_FLAG_*


class AetError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else status}: {message}")
        self.status = status


def make_config(cfg: dict) -> AetConfig:
    """A workload dict (see workloads.CONFIGS) as the library's aet_config."""
    c = AetConfig()
    c.struct_size = C.sizeof(AetConfig)
    dims = list(cfg["dims"])
    c.n_layers = len(dims) - 1
    for i, d in enumerate(dims):
        c.dims[i] = d
    for name, _ in AetConfig._fields_:
        if name in ("struct_size", "n_layers", "dims", "flags", "split_mode", "topology", "client_shares"):
            continue
        setattr(c, name, cfg[name])
    c.flags = int(cfg.get("flags", 0))
    c.split_mode = int(cfg.get("split_mode", 0))
    c.topology = int(cfg.get("topology", 0))
    shares = cfg.get("client_shares")
    if shares:
        arr = (C.c_uint32 * len(shares))(*[int(v) for v in shares])
        c.client_shares = C.cast(arr, C.POINTER(C.c_uint32))
        c._shares_keepalive = arr      # the library copies them in aet_create; until then they live here
    return c


def _ptr(buf):
    """Address of a torch tensor, numpy array or raw int; None -> null."""
    if buf is None:
        return None
    if isinstance(buf, int):
        return C.c_void_p(buf)
    if isinstance(buf, np.ndarray):
        assert buf.flags["C_CONTIGUOUS"]
        return C.c_void_p(buf.ctypes.data)
    assert buf.is_contiguous()
    return C.c_void_p(buf.data_ptr())


def _stream(stream):
    if stream is None:
        import torch
        return C.c_void_p(torch.cuda.current_stream().cuda_stream)
    return C.c_void_p(stream if isinstance(stream, int) else stream.cuda_stream)


def _check(handle, status):
    if status != 0:
        msg = _lib.load().aet_last_error(handle)
        raise AetError(status, msg.decode() if msg else "")


def aet_create(cfg) -> C.c_void_p:
    conf = cfg if isinstance(cfg, AetConfig) else make_config(cfg)
    h = C.c_void_p()
    _check(None, _lib.load().aet_create(C.byref(conf), C.byref(h)))
    return h


def aet_destroy(h):
    _check(h, _lib.load().aet_destroy(h))


def aet_release_memory():
    """Device memory kept from destroyed handles, and pinned blocks, back to the driver."""
    _check(None, _lib.load().aet_release_memory())


def aet_reset(h, stream=None):
    _check(h, _lib.load().aet_reset(h, _stream(stream)))


def aet_set_global_model(h, w0, stream=None):
    _check(h, _lib.load().aet_set_global_model(h, _ptr(w0), w0.size if isinstance(w0, np.ndarray) else w0.numel(),
                                               _stream(stream)))


def _kind(a, kind, what: str):
    """Held to a type (or one of several)."""
    kinds = (kind,) if isinstance(kind, str) else kind
    if str(a.dtype).rsplit(".", 1)[-1] not in kinds:
        raise AetError(1, f"{what}: {a.dtype}, expected {kinds[0]}")


def _u32(v: int, what: str) -> int:
    """Held to what the library's 32-bit arguments can say (ctypes would cut it off)."""
    if not 0 <= v < 1 << 32:
        raise AetError(1, f"{what}: {v} is not a number of 32 bits")
    return v


def _rows(a, kind, n: int, width: int, what: str):
    """Held to its type and size, n rows of `width` values: the library gets an address and reads or writes that much behind it."""
    _kind(a, kind, what)
    _u32(n, "rows")
    if a.shape[0] != n or (a.size if isinstance(a, np.ndarray) else a.numel()) != n * width:
        raise AetError(1, f"{what}: {tuple(a.shape)}, expected {n} rows of {width}")


def aet_load_client_data(h, client: int, x, y, stream=None):
    n = x.shape[0]
    _rows(x, "float32", n, aet_n_inputs(h), "x")
    _rows(y, ("int32", "uint32"), n, 1, "y")          # (classes are not negative: the same bits)
    _check(h, _lib.load().aet_load_client_data(h, client, _ptr(x), _ptr(y), n, _stream(stream)))


def aet_run_rounds(h, n_rounds: int, stream=None):
    _check(h, _lib.load().aet_run_rounds(h, n_rounds, _stream(stream)))


def aet_prepare_rounds(h, n_rounds: int):
    """Start the host-side schedule and launch plan of the next aet_run_rounds(h, n_rounds) on a library thread."""
    _check(h, _lib.load().aet_prepare_rounds(h, n_rounds))


def aet_n_params(h) -> int:
    return int(_lib.load().aet_n_params(h))


def aet_n_inputs(h) -> int:
    """Values in a row of the model's inputs."""
    return int(_lib.load().aet_n_inputs(h))


def aet_n_classes(h) -> int:
    return int(_lib.load().aet_n_classes(h))


def aet_get_global_model(h, out=None, stream=None):
    if out is None:
        out = np.empty(aet_n_params(h), dtype=np.float32)
    n = out.size if isinstance(out, np.ndarray) else out.numel()
    _check(h, _lib.load().aet_get_global_model(h, _ptr(out), n, _stream(stream)))
    return out


def aet_get_node_model(h, node: int, out=None, stream=None):
    if out is None:
        out = np.empty(aet_n_params(h), dtype=np.float32)
    n = out.size if isinstance(out, np.ndarray) else out.numel()
    _check(h, _lib.load().aet_get_node_model(h, node, _ptr(out), n, _stream(stream)))
    return out


def aet_get_update_sum(h, seq: int, out=None, stream=None):
    if out is None:
        out = np.empty(aet_n_params(h), dtype=np.float32)
    n = out.size if isinstance(out, np.ndarray) else out.numel()
    _check(h, _lib.load().aet_get_update_sum(h, seq, _ptr(out), n, _stream(stream)))
    return out


def _here(a, what: str):
    """An array of the host or of the current device: the evaluation's kernels read and write a device array where it is."""
    if isinstance(a, np.ndarray) or not a.is_cuda:
        return
    import torch
    if a.get_device() != torch.cuda.current_device():
        raise AetError(1, f"{what} has to be on the host or on the current CUDA device, not on {a.device}")


def aet_predict(h, node: int, x, logits=None, classes=None, stream=None):
    """Logits [n, classes] of a node's model for the rows of x; host or device arrays (without `logits` a numpy array of `classes` columns)."""
    if logits is None:
        if classes is None:
            raise AetError(1, "either logits or classes is needed")
        logits = np.empty((x.shape[0], classes), dtype=np.float32)
    n = x.shape[0]
    _rows(x, "float32", n, aet_n_inputs(h), "x")
    _rows(logits, "float32", n, aet_n_classes(h), "logits")
    _here(x, "x")
    _here(logits, "logits")
    _check(h, _lib.load().aet_predict(h, _u32(node, "node"), _ptr(x), n, _ptr(logits), _stream(stream)))
    return logits


def aet_evaluate(h, node: int, x, y, dropout=None, gradient=None, stream=None):
    """(loss, rows the model gets right) of a node's model on rows x with classes y; gradient: where the loss's gradient goes."""
    n = x.shape[0]
    _rows(x, "float32", n, aet_n_inputs(h), "x")
    _rows(y, "int32", n, 1, "y")
    _here(x, "x")
    _here(y, "y")
    if gradient is not None:
        _kind(gradient, "float32", "gradient")
        if (gradient.size if isinstance(gradient, np.ndarray) else gradient.numel()) != aet_n_params(h):
            raise AetError(1, "gradient: as many values as the model has parameters are expected")
    loss, right = C.c_double(), C.c_uint64()
    _check(h, _lib.load().aet_evaluate(h, _u32(node, "node"), _ptr(x), _ptr(y), n, None if dropout is None else C.addressof(dropout),
                                       C.addressof(loss), C.addressof(right), _ptr(gradient), _stream(stream)))
    return float(loss.value), int(right.value)


def _events_from(arr, n):
    names = [f for f, _ in AetEvent._fields_]
    return [{f: int(getattr(arr[k], f)) for f in names} for k in range(n)]


def _summary_from(s):
    return {f: int(getattr(s, f)) for f, _ in AetSummary._fields_}


def aet_get_event_log(h, raw: bool = False):
    """(events, summary); events as dicts, or the raw 64-byte records if raw."""
    lib = _lib.load()
    n = C.c_size_t()
    _check(h, lib.aet_get_event_log(h, None, 0, C.byref(n), None))
    arr = (AetEvent * max(1, n.value))()
    s = AetSummary()
    _check(h, lib.aet_get_event_log(h, arr, n.value, C.byref(n), C.byref(s)))
    if raw:
        return bytes(memoryview(arr))[:64 * n.value], _summary_from(s)
    return _events_from(arr, n.value), _summary_from(s)


def aet_debug_run_client_round(h, client: int, rnd: int, w_in, U_out=None, w_out=None, stream=None):
    P = aet_n_params(h)
    if U_out is None:
        U_out = np.empty(P, dtype=np.float32)
    if w_out is None:
        w_out = np.empty(P, dtype=np.float32)
    _check(h, _lib.load().aet_debug_run_client_round(h, client, rnd, _ptr(w_in), _ptr(U_out), _ptr(w_out),
                                                     _stream(stream)))
    return U_out, w_out


def aet_round_no_alloc(cfg, client: int, rnd: int, x, y, w_in, U_out, w_out, stream=None):
    """One round-task from caller-owned DEVICE buffers, using only the scratch
    array built into the library: for callers that may not allocate device
    memory while they run.  Asynchronous on the stream; calls that could overlap
    on the GPU race on the shared scratch."""
    conf = cfg if isinstance(cfg, AetConfig) else make_config(cfg)
    _check(None, _lib.load().aet_round_no_alloc(C.byref(conf), client, rnd, _ptr(x), _ptr(y), x.shape[0],
                                                _ptr(w_in), _ptr(U_out), _ptr(w_out), _stream(stream)))


def aet_debug_wait_probe(h, max_polls: int = 1 << 12, stream=None):
    """Makes a bounded device wait run out on purpose; raises AetError(AET_ERR_TIMEOUT)."""
    _check(h, _lib.load().aet_debug_wait_probe(h, max_polls, _stream(stream)))


def aet_set_kernel_timing(h, enable: bool):
    _check(h, _lib.load().aet_set_kernel_timing(h, int(enable)))


def aet_get_stats(h) -> dict:
    s = AetStats()
    _check(h, _lib.load().aet_get_stats(h, C.byref(s)))
    return dict(waves=int(s.waves), launches=[int(v) for v in s.launches],
                kernel_ms=[float(v) for v in s.kernel_ms], plan_ms=float(s.plan_ms))


def aet_schedule_only(cfg, n_rounds: int, raw: bool = False):
    """Host only: the event log a fresh run of n_rounds would produce."""
    lib = _lib.load()
    conf = cfg if isinstance(cfg, AetConfig) else make_config(cfg)
    n = C.c_size_t()
    _check(None, lib.aet_schedule_only(C.byref(conf), n_rounds, None, 0, C.byref(n), None))
    arr = (AetEvent * max(1, n.value))()
    s = AetSummary()
    _check(None, lib.aet_schedule_only(C.byref(conf), n_rounds, arr, n.value, C.byref(n), C.byref(s)))
    if raw:
        return bytes(memoryview(arr))[:64 * n.value], _summary_from(s)
    return _events_from(arr, n.value), _summary_from(s)


def aet_debug_regression_kernel(n_tasks, longest, by_value, at_once):
    """(kernel, CTAs per round-task) of a launch of regression round-tasks; at_once[n]: clusters of n CTAs the device runs at once."""
    got = _lib.load().aet_debug_regression_kernel(n_tasks, longest, int(by_value), (C.c_uint32 * 9)(*at_once))
    return ("relay", "chain", "block", "crowded")[got // 16], got % 16


def aet_debug_draw(seed, stream_id, client, counter) -> int:
    return int(_lib.load().aet_debug_draw(seed, stream_id, client, counter))


def aet_debug_delay_ticks(dist, draw, p0, p1=0) -> int:
    return int(_lib.load().aet_debug_delay_ticks(dist, draw, p0, p1))


def aet_debug_plan_waves(cfg, n_rounds) -> int:
    conf = cfg if isinstance(cfg, AetConfig) else make_config(cfg)
    return int(_lib.load().aet_debug_plan_waves(C.byref(conf), n_rounds))


def aet_debug_plan_layout(cfg, n_rounds) -> dict:
    """Host only: the launch plan of a fresh run (see include/aet.h)."""
    conf = cfg if isinstance(cfg, AetConfig) else make_config(cfg)
    E = conf.n_clients * n_rounds
    u32 = lambda: np.zeros(max(E, 1), dtype=np.uint32)
    out = dict(task_seq=u32(), task_wave=u32(), task_snap_slot=u32(), u_row=u32(),
               snap_slot_after=np.zeros(max(E, 1), dtype=np.int32), apply_upto=u32())
    counts = np.zeros(3, dtype=np.uint32)
    _check(None, _lib.load().aet_debug_plan_layout(C.byref(conf), n_rounds, *[_ptr(v) for v in out.values()], _ptr(counts)))
    out = {k: v[:E] for k, v in out.items()}
    out["apply_upto"] = out["apply_upto"][:int(counts[0])]
    out.update(waves=int(counts[0]), n_u_rows=int(counts[1]), n_snap=int(counts[2]))
    return out


# ---- layers: torch tensors on the current CUDA device ----------------------------------------------------------------------

ACTS = dict(none=0, relu=1, gelu=2, silu=3)           # AET_ACT_*
DENSE_ANY_ADDRESS, DENSE_ACCUMULATE = 1, 2            # AET_DENSE_*
_dtypes = {}


def _dtype(t) -> int:
    """AET_F32, AET_BF16 or AET_F16 of a torch dtype."""
    if not _dtypes:
        import torch
        _dtypes.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    try:
        return _dtypes[t]
    except KeyError:
        raise AetError(1, f"element type {t} is not float32, bfloat16 or float16") from None


_cuda = None


def _stream_of(dev: int, t, stream):
    """The stream given, or the current one, of the current device, which the tensors have to be on.

    torch.cuda.current_device() and current_stream() take longer than a whole call here; this is what they ask."""
    global _cuda
    if _cuda is None:
        import torch
        _cuda = torch._C
    if dev < 0 or dev != _cuda._cuda_getDevice():
        raise AetError(1, f"tensors have to be on the current CUDA device, not on {t.device}")
    if stream is None:
        return _cuda._cuda_getCurrentRawStream(dev)
    return stream if isinstance(stream, int) else stream.cuda_stream


def _at(t, dtype, dev, shape, what, ld):
    """Address of a matrix of rows `ld` elements apart, or (ld None) of a vector (t None: null)."""
    if t is None:
        return None
    if t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.stride() == ((ld, 1) if ld else (1,)):
        return t.data_ptr()
    s = t.stride()
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev:
        raise AetError(1, f"{what}: {tuple(t.shape)} of {t.dtype} on {t.device}, expected {tuple(shape)} of {dtype} on CUDA device {dev}")
    if t.numel() and ((shape[-1] > 1 and s[-1] != 1) or (ld and shape[0] > 1 and s[0] != ld)):   # (what an index of one value strides by does not matter)
        raise AetError(1, f"{what}: strides {s}, expected rows {ld} elements apart of neighbouring elements")
    return t.data_ptr()


def _row_major(t, dtype, dev, shape, what):
    """Address and ld of a matrix whose rows may be any distance apart."""
    if t is None:
        return None, 0
    ld = t.stride(0) if shape[0] > 1 and len(t.shape) == 2 else shape[1]
    at = _at(t, dtype, dev, shape, what, ld)
    if ld < shape[1]:       # (a broadcast tensor's rows are 0 apart, which the library would take for no gaps)
        raise AetError(1, f"{what}: strides {t.stride()}, expected rows {shape[1]} or more elements apart")
    return at, ld


def aet_dropout_spec(seed: int, client: int = 0, counter: int = 0, rate: float = 0.0):
    return _lib.AetDropoutSpec(seed=seed, client=_u32(client, "client"), counter=counter, rate=rate)


def aet_dropout(drop, x, y, residual=None, stream=None):
    """y = residual + dropout(x); see include/aet.h for which elements a (seed, client, counter) drops."""
    shape, dtype, dev = x.shape, x.dtype, x.get_device()
    if len(shape) != 2:
        raise AetError(1, "x: a matrix is expected")
    px, ld_x = _row_major(x, dtype, dev, shape, "x")
    pr, ld_r = _row_major(residual, dtype, dev, shape, "residual")
    py, ld_y = _row_major(y, dtype, dev, shape, "y")
    _check(None, _lib.load().aet_dropout(_dtype(dtype), shape[0], _u32(shape[1], "columns"), C.addressof(drop), px, ld_x, pr, ld_r, py, ld_y, _stream_of(dev, x, stream)))


def aet_cross_entropy(logits, labels, loss=None, dlogits=None, top=None, weight=None, scale: float = 1.0, stream=None):
    """Softmax cross-entropy of each row, its gradient times `scale` (and `weight`), and the lowest index of its maximum."""
    import torch
    shape, dtype, dev = logits.shape, logits.dtype, logits.get_device()
    if len(shape) != 2:
        raise AetError(1, "logits: a matrix is expected")
    one = shape[:1]
    pz, ld_z = _row_major(logits, dtype, dev, shape, "logits")
    pg, ld_g = _row_major(dlogits, dtype, dev, shape, "dlogits")
    _check(None, _lib.load().aet_cross_entropy(
        _dtype(dtype), shape[0], _u32(shape[1], "classes"), pz, ld_z, _at(labels, torch.int32, dev, one, "labels", None),
        _at(weight, torch.float32, dev, one, "weight", None), scale, _at(loss, torch.float32, dev, one, "loss", None), pg, ld_g,
        _at(top, torch.int32, dev, one, "top", None), _stream_of(dev, logits, stream)))


def aet_dense(n_in: int, n_out: int, dtype=None, act: str = "none", dropout=None, ld_in: int = 0, ld_out: int = 0, ld_w: int = 0, flags: int = 0, **lds):
    """Descriptor of a dense layer.  dtype: a torch dtype (float32).  ld_in: rows of x and dx, ld_out: of y, residual, pre and dy,
    ld_w: of W and dW; ld_x=, ld_dw= and so on for one alone; 0: no gaps."""
    d = _lib.AetDenseDesc()
    d.struct_size = C.sizeof(_lib.AetDenseDesc)
    d.dtype = 0 if dtype is None else _dtype(dtype)
    if act not in ACTS:
        raise AetError(1, f"activation {act!r} is not one of {', '.join(ACTS)}")
    d.act, d.n_in, d.n_out, d.flags = ACTS[act], _u32(n_in, "n_in"), _u32(n_out, "n_out"), _u32(flags, "flags")
    d.ld_x = d.ld_dx = ld_in or n_in
    d.ld_w = d.ld_dw = ld_w or n_out
    d.ld_y = d.ld_residual = d.ld_pre = d.ld_dy = ld_out or n_out
    for k, v in lds.items():
        if not k.startswith("ld_") or not hasattr(d, k):
            raise AetError(1, f"unknown argument {k}")
        setattr(d, k, v or (n_in if k in ("ld_x", "ld_dx") else n_out))
    if dropout is not None:
        d.drop = dropout
    return d


def aet_dense_workspace(d, rows: int, backward: bool = False) -> int:
    """Bytes of workspace a call on so many rows needs."""
    n = C.c_size_t()
    _check(None, _lib.load().aet_dense_workspace(C.addressof(d), rows, int(backward), C.addressof(n)))
    return int(n.value)


def _space(workspace, dev):
    if workspace is None:
        return None, 0
    if workspace.get_device() != dev or not workspace.is_contiguous():
        raise AetError(1, "workspace: a contiguous tensor on the layer's device is expected")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _rows_of(d, x, cols, what):
    if len(x.shape) != 2 or x.shape[1] != cols or _dtype(x.dtype) != d.dtype:
        raise AetError(1, f"{what}: {tuple(x.shape)} of {x.dtype} does not fit the descriptor")
    return x.shape[0], x.dtype, x.get_device()


def aet_dense_forward(d, x, w, bias, y, residual=None, pre=None, workspace=None, stream=None):
    """y = residual + dropout(act(x w + bias)); pre: where x w + bias goes for the backward pass."""
    n_in, n_out = d.n_in, d.n_out
    rows, t, dev = _rows_of(d, x, n_in, "x")
    out = (rows, n_out)
    ws, size = _space(workspace, dev)
    _check(None, _lib.load().aet_dense_forward(
        C.addressof(d), rows, _at(x, t, dev, (rows, n_in), "x", d.ld_x), _at(w, t, dev, (n_in, n_out), "w", d.ld_w), _at(bias, t, dev, (n_out,), "bias", None),
        _at(residual, t, dev, out, "residual", d.ld_residual), _at(y, t, dev, out, "y", d.ld_y), _at(pre, t, dev, out, "pre", d.ld_pre), ws, size,
        _stream_of(dev, x, stream)))


def aet_debug_dense_lost_copies(d, x, w, y, workspace, stages: int, wait_us: int, stream=None):
    """y = dropout(act(x w)) on the tensor cores as if the first CTA's copies from stage `stages` on never came."""
    rows, t, dev = _rows_of(d, x, d.n_in, "x")
    ws, size = _space(workspace, dev)
    _check(None, _lib.load().aet_debug_dense_lost_copies(
        C.addressof(d), rows, _at(x, t, dev, (rows, d.n_in), "x", d.ld_x), _at(w, t, dev, (d.n_in, d.n_out), "w", d.ld_w),
        _at(y, t, dev, (rows, d.n_out), "y", d.ld_y), ws, size, _u32(stages, "stages"), _u32(wait_us, "wait_us"), _stream_of(dev, x, stream)))


def aet_dense_backward(d, x, w, dy, pre=None, dx=None, dw=None, db=None, workspace=None, stream=None):
    """dx, dw and db (any of them None) of the layer from dy."""
    n_in, n_out = d.n_in, d.n_out
    rows, t, dev = _rows_of(d, dy, n_out, "dy")
    out, into, weights = (rows, n_out), (rows, n_in), (n_in, n_out)
    ws, size = _space(workspace, dev)
    _check(None, _lib.load().aet_dense_backward(
        C.addressof(d), rows, _at(x, t, dev, into, "x", d.ld_x), _at(w, t, dev, weights, "w", d.ld_w), _at(pre, t, dev, out, "pre", d.ld_pre),
        _at(dy, t, dev, out, "dy", d.ld_dy), _at(dx, t, dev, into, "dx", d.ld_dx), _at(dw, t, dev, weights, "dw", d.ld_dw),
        _at(db, t, dev, (n_out,), "db", None), ws, size, _stream_of(dev, dy, stream)))


class Session:
    """Convenience wrapper: create, load every client's data, run, read back."""

    def __init__(self, cfg: dict, data, w0=None, stream=None):
        self.cfg = cfg
        self.h = aet_create(cfg)
        self.stream = stream
        try:
            if w0 is not None:
                aet_set_global_model(self.h, w0, stream)
            for c, (x, y) in enumerate(data):
                aet_load_client_data(self.h, c, x, y, stream)
        except Exception:
            self.close()
            raise

    def run(self, n_rounds=None):
        aet_run_rounds(self.h, self.cfg["n_rounds"] if n_rounds is None else n_rounds, self.stream)

    def reset(self):
        aet_reset(self.h, self.stream)

    def model(self):
        return aet_get_global_model(self.h, stream=self.stream)

    def predict(self, x, node=0):
        return aet_predict(self.h, node, x, classes=self.cfg["dims"][-1], stream=self.stream)

    def evaluate(self, x, y, node=0, dropout=None, gradient=None):
        return aet_evaluate(self.h, node, x, y, dropout, gradient, self.stream)

    def log(self, raw=False):
        return aet_get_event_log(self.h, raw)

    def close(self):
        if self.h is not None:
            aet_destroy(self.h)
            self.h = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


def aet_debug_lost_copies(h, client: int, rnd: int, cta: int, w_in, U_out, w_out, max_polls: int = 1 << 12, stream=None):
    """One round-task as if the copies of one CTA of its cluster never came; raises AetError(AET_ERR_TIMEOUT), with U_out written."""
    _check(h, _lib.load().aet_debug_lost_copies(h, client, rnd, cta, max_polls, _ptr(w_in), _ptr(U_out), _ptr(w_out),
                                                _stream(stream)))
