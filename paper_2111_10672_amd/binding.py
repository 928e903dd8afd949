"""ctypes binding of libspb.so.  Same names as the C ABI; no arithmetic happens here."""
from __future__ import annotations

import array
import ctypes as C
import os
import struct

HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(HERE, "libspb.so")
_lib = None

SPB_MAX_DIMS, SPB_MAX_STAGES, SPB_NAME_LEN = 64, 8, 48
SPB_OK = 0
ERRORS = {-1: "SPB_ERR_INVALID_ARG", -2: "SPB_ERR_DEPTH_RANGE", -3: "SPB_ERR_STATE",
          -4: "SPB_ERR_WORKSPACE", -5: "SPB_ERR_HIP", -6: "SPB_ERR_UNSUPPORTED"}
FAMILIES = {"mlp": 0, "resnet_basic": 1, "resnet_bottleneck": 2, "encoder": 3}
DTYPES = {"f32": 0, "bf16": 1}


class SpbError(RuntimeError):
    def __init__(self, code, message):
        super().__init__(f"{ERRORS.get(code, code)}: {message}")
        self.code = code


class spb_model_desc(C.Structure):
    _fields_ = [("family", C.c_int32), ("dtype", C.c_int32), ("batch", C.c_int32),
                ("n_dims", C.c_int32), ("dims", C.c_int32 * SPB_MAX_DIMS),
                ("image_h", C.c_int32), ("image_w", C.c_int32), ("image_c", C.c_int32),
                ("stem_kernel", C.c_int32), ("stem_stride", C.c_int32), ("stem_pad", C.c_int32),
                ("stem_pool", C.c_int32), ("stem_width", C.c_int32),
                ("n_stages", C.c_int32), ("stage_blocks", C.c_int32 * SPB_MAX_STAGES),
                ("stage_widths", C.c_int32 * SPB_MAX_STAGES), ("classes", C.c_int32),
                ("seq", C.c_int32), ("layers", C.c_int32), ("hidden", C.c_int32), ("heads", C.c_int32),
                ("ffn", C.c_int32), ("vocab", C.c_int32), ("loss_rows", C.c_int32)]


class spb_tensor_info(C.Structure):
    _fields_ = [("name", C.c_char * SPB_NAME_LEN), ("unit", C.c_int32), ("dtype", C.c_int32),
                ("ndim", C.c_int32), ("shape", C.c_int64 * 4), ("numel", C.c_int64)]


class spb_grad_view(C.Structure):
    _fields_ = [("param_index", C.c_int32), ("unit", C.c_int32), ("data", C.c_void_p), ("numel", C.c_int64)]


class spb_buffer_view(C.Structure):
    _fields_ = [("offset", C.c_int64), ("rows", C.c_int64), ("cols", C.c_int64), ("pitch", C.c_int64),
                ("dtype", C.c_int32), ("relu_applied", C.c_int32)]


class spb_kernel_time(C.Structure):
    _fields_ = [("name", C.c_char * SPB_NAME_LEN), ("launches", C.c_int64), ("total_ms", C.c_double),
                ("flops", C.c_double), ("bytes", C.c_double)]


class spb_sched_job(C.Structure):
    _fields_ = [("arrival", C.c_double), ("model_size", C.c_double), ("iterations", C.c_int32), ("workers", C.c_int32),
                ("durations", C.POINTER(C.c_double)), ("resources", C.POINTER(C.c_double))]


class spb_sched_task(C.Structure):
    _fields_ = [("job", C.c_int32), ("iteration", C.c_int32), ("worker", C.c_int32), ("machine", C.c_int32),
                ("moved", C.c_int32), ("start", C.c_double), ("end", C.c_double), ("held_until", C.c_double)]


_F32 = DTYPES["f32"]
SPB_MAX_HEAD_DIM, SPB_MAX_PAIRS, SPB_MAX_AXES, SPB_MAX_MATRIX_SIDE = 256, 128, 4, 65536


class spb_rotary(C.Structure):
    _fields_ = [("pairs", C.c_int32), ("interleaved", C.c_int32), ("axes", C.c_int32), ("reserved", C.c_int32),
                ("axis", C.c_int32 * SPB_MAX_PAIRS), ("freq", C.c_double * SPB_MAX_PAIRS)]


class spb_heads_desc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("batch", C.c_int32), ("seq", C.c_int32), ("heads_q", C.c_int32), ("heads_k", C.c_int32),
                ("head_dim", C.c_int32), ("norm", C.c_int32), ("eps", C.c_float), ("x_stride", C.c_int64 * 3), ("y_stride", C.c_int64 * 3),
                ("dx_stride", C.c_int64 * 3), ("rotary", spb_rotary)]


class spb_muon_tensor(C.Structure):
    _fields_ = [("w", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("grads", C.POINTER(C.c_void_p)), ("rows", C.c_int64), ("cols", C.c_int64),
                ("rate_scale", C.c_double), ("count", C.c_int32), ("dtype", C.c_int32), ("blocks", C.c_int32), ("reserved", C.c_int32)]


class spb_muon_config(C.Structure):
    _fields_ = [("lr", C.c_double), ("rms", C.c_double), ("momentum", C.c_double), ("ns_eps", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double),
                ("adam_eps", C.c_double), ("weight_decay", C.c_double), ("step", C.c_int64), ("nesterov", C.c_int32), ("ns_steps", C.c_int32)]


_TASK = struct.Struct("<4i?7x3d")     # spb_sched_task; `moved` is 0 or 1, so its lowest byte says it
assert _TASK.size == C.sizeof(spb_sched_task)


EXPORTS = {
    "spb_last_error": (C.c_char_p, []),
    "spb_model_create": (C.c_int, [C.POINTER(spb_model_desc), C.POINTER(C.c_void_p)]),
    "spb_model_destroy": (C.c_int, [C.c_void_p]),
    "spb_num_units": (C.c_int, [C.c_void_p, C.POINTER(C.c_int32)]),
    "spb_param_count": (C.c_int, [C.c_void_p, C.POINTER(C.c_int32)]),
    "spb_param_info": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(spb_tensor_info)]),
    "spb_bind_params": (C.c_int, [C.c_void_p, C.POINTER(C.c_void_p), C.c_int32]),
    "spb_bind_grads": (C.c_int, [C.c_void_p, C.POINTER(C.c_void_p), C.c_int32]),
    "spb_workspace_size": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(C.c_size_t)]),
    "spb_forward": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                              C.c_size_t, C.c_void_p, C.c_void_p]),
    "spb_forward_static": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]),
    "spb_backward_truncated": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p]),
    "spb_grad_buffers": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(spb_grad_view), C.c_int32, C.POINTER(C.c_int32)]),
    "spb_unit_io": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.POINTER(spb_buffer_view), C.POINTER(spb_buffer_view)]),
    "spb_zero_absent_grads": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p]),
    "spb_worker_depth": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.POINTER(C.c_int32)]),
    "spb_aggregate_update": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(C.c_int32), C.POINTER(C.c_void_p), C.POINTER(C.c_void_p),
                                       C.c_float, C.c_float, C.c_float, C.c_int32, C.c_void_p]),
    "spb_rotary_sections": (C.c_int, [C.POINTER(spb_rotary), C.c_int32, C.c_void_p, C.c_double, C.c_int32, C.c_int32]),
    "spb_heads_forward": (C.c_int, [C.POINTER(spb_heads_desc), C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]),
    "spb_heads_workspace_size": (C.c_int, [C.POINTER(spb_heads_desc), C.POINTER(C.c_size_t)]),
    "spb_heads_backward": (C.c_int, [C.POINTER(spb_heads_desc), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_void_p,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "spb_encoder_heads": (C.c_int, [C.c_void_p, C.POINTER(spb_rotary), C.c_void_p, C.c_int64, C.c_int64, C.c_int32, C.c_float]),
    "spb_muon_workspace_size": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(C.c_size_t)]),
    "spb_muon_step": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(spb_muon_config), C.c_void_p, C.c_size_t, C.c_void_p]),
    "spb_aggregate_muon_workspace_size": (C.c_int, [C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_size_t)]),
    "spb_aggregate_muon": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(C.c_int32), C.POINTER(C.c_void_p), C.POINTER(C.c_int32), C.POINTER(C.c_void_p),
                                     C.POINTER(C.c_void_p), C.POINTER(spb_muon_config), C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]),
    "spb_set_kernel_timing": (C.c_int, [C.c_void_p, C.c_int32]),
    "spb_replay_kernel": (C.c_int, [C.c_void_p, C.c_char_p, C.c_int32, C.c_void_p]),
    "spb_read_kernel_timing": (C.c_int, [C.c_void_p, C.POINTER(spb_kernel_time), C.c_int32, C.POINTER(C.c_int32)]),
    "spb_schedule_tasks": (C.c_int, [C.POINTER(spb_sched_job), C.c_int32, C.c_int32, C.c_double, C.c_double, C.c_int32,
                                     C.POINTER(spb_sched_task), C.c_int64, C.POINTER(C.c_int64), C.POINTER(C.c_double)]),
}


def library_path() -> str:
    return _LIB_PATH


def lib():
    """Load libspb.so; build it first only if it does not exist.  No fallback: raises if it cannot load."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            from .build import build_library
            build_library()
        handle = C.CDLL(_LIB_PATH)
        for name, (res, args) in EXPORTS.items():
            fn = getattr(handle, name)
            fn.restype, fn.argtypes = res, args
        _lib = handle
    return _lib


def spb_last_error() -> str:
    return lib().spb_last_error().decode()


def _check(code):
    if code != SPB_OK:
        raise SpbError(code, spb_last_error())


def desc_from_config(cfg: dict) -> spb_model_desc:
    d = spb_model_desc()
    d.family, d.dtype, d.batch = FAMILIES[cfg["family"]], DTYPES[cfg["dtype"]], cfg["batch"]
    if cfg["family"] == "mlp":
        d.n_dims = len(cfg["dims"])
        for i, w in enumerate(cfg["dims"]):
            d.dims[i] = w
    elif cfg["family"].startswith("resnet"):
        d.image_h, d.image_w, d.image_c = cfg["image"]
        st = cfg["stem"]
        d.stem_kernel, d.stem_stride, d.stem_pad = st["kernel"], st["stride"], st["pad"]
        d.stem_pool, d.stem_width = int(st["pool"]), st["width"]
        d.n_stages = len(cfg["stage_blocks"])
        for i, (b, w) in enumerate(zip(cfg["stage_blocks"], cfg["stage_widths"])):
            d.stage_blocks[i], d.stage_widths[i] = b, w
        d.classes = cfg["classes"]
    else:
        for key in ("seq", "layers", "hidden", "heads", "ffn", "vocab", "loss_rows"):
            setattr(d, key, cfg[key])
    return d


def _ptr(t):
    """Device (or null) pointer of a torch tensor / int / None."""
    if t is None:
        return None
    if isinstance(t, int):
        return C.c_void_p(t)
    return C.c_void_p(t.data_ptr())


def spb_model_create(desc: spb_model_desc) -> C.c_void_p:
    out = C.c_void_p()
    _check(lib().spb_model_create(C.byref(desc), C.byref(out)))
    out.batch, out.seq = desc.batch, desc.seq      # what tensors per token are compared with
    return out


def spb_model_destroy(m):
    _check(lib().spb_model_destroy(m))


def spb_num_units(m) -> int:
    n = C.c_int32()
    _check(lib().spb_num_units(m, C.byref(n)))
    return n.value


def spb_param_count(m) -> int:
    n = C.c_int32()
    _check(lib().spb_param_count(m, C.byref(n)))
    return n.value


def spb_param_info(m, index: int) -> dict:
    info = spb_tensor_info()
    _check(lib().spb_param_info(m, index, C.byref(info)))
    return {"name": info.name.decode(), "unit": info.unit, "dtype": "f32" if info.dtype == 0 else "bf16",
            "shape": tuple(info.shape[i] for i in range(info.ndim)), "numel": info.numel}


def _ptr_array(tensors):
    arr = (C.c_void_p * len(tensors))()
    for i, t in enumerate(tensors):
        arr[i] = None if t is None else (t if isinstance(t, int) else t.data_ptr())
    return arr


def spb_bind_params(m, tensors):
    _check(lib().spb_bind_params(m, _ptr_array(tensors), len(tensors)))


def spb_bind_grads(m, tensors):
    _check(lib().spb_bind_grads(m, _ptr_array(tensors), len(tensors)))


def spb_workspace_size(m, k: int) -> int:
    n = C.c_size_t()
    _check(lib().spb_workspace_size(m, k, C.byref(n)))
    return n.value


def spb_forward(m, x, labels, loss_rows, k, workspace, workspace_bytes, loss_out, stream):
    _check(lib().spb_forward(m, _ptr(x), _ptr(labels), _ptr(loss_rows), k, _ptr(workspace),
                             workspace_bytes, _ptr(loss_out), C.c_void_p(stream)))


SPB_STATIC_WORKSPACE_BYTES = 8 << 20


def spb_forward_static(m, x, labels, loss_rows, k, loss_out, stream):
    _check(lib().spb_forward_static(m, _ptr(x), _ptr(labels), _ptr(loss_rows), k, _ptr(loss_out), C.c_void_p(stream)))


def spb_backward_truncated(m, k, stream):
    _check(lib().spb_backward_truncated(m, k, C.c_void_p(stream)))


def spb_grad_buffers(m, k, cap=None):
    cap = spb_param_count(m) if cap is None else cap
    views = (spb_grad_view * max(cap, 1))()
    n = C.c_int32()
    _check(lib().spb_grad_buffers(m, k, views, cap, C.byref(n)))
    return [{"param_index": v.param_index, "unit": v.unit, "data": v.data, "numel": v.numel} for v in views[:n.value]]


SPB_VIEW_CALLER_INPUT, SPB_VIEW_NONE = -1, -2


def spb_unit_io(m, k: int, unit: int):
    """(input view, output-gradient view) of a unit as dicts; see spb.h."""
    a, b = spb_buffer_view(), spb_buffer_view()
    _check(lib().spb_unit_io(m, k, unit, C.byref(a), C.byref(b)))
    as_dict = lambda v: {"offset": v.offset, "rows": v.rows, "cols": v.cols, "pitch": v.pitch,
                         "dtype": {0: "f32", 1: "bf16", 2: "i32"}[v.dtype], "relu_applied": bool(v.relu_applied)}
    return as_dict(a), as_dict(b)


def spb_zero_absent_grads(m, k, stream):
    _check(lib().spb_zero_absent_grads(m, k, C.c_void_p(stream)))


def spb_worker_depth(m, j: int, n_workers: int) -> int:
    k = C.c_int32()
    _check(lib().spb_worker_depth(m, j, n_workers, C.byref(k)))
    return k.value


def spb_aggregate_update(m, depths, worker_grads, velocity, lr, momentum, weight_decay, scale_lr, stream):
    """worker_grads: one list per worker, each with one tensor (or None) per parameter; velocity: one tensor per parameter."""
    n = len(depths)
    d = (C.c_int32 * n)(*depths)
    flat = [g for per_worker in worker_grads for g in per_worker]
    _check(lib().spb_aggregate_update(m, n, d, _ptr_array(flat), _ptr_array(velocity), lr, momentum, weight_decay,
                                      int(bool(scale_lr)), C.c_void_p(stream)))


_COUNTS = [struct.Struct(f"<{n}i") for n in range(SPB_MAX_AXES + 2)]      # (one more than there are axes: refused in C)


def spb_rotary_sections(sections, base=10000.0, own_ladder=False, interleaved=False) -> spb_rotary:
    """Rotary description: sections[a] pairs for axis a; see spb.h for the frequencies."""
    out, n = spb_rotary(), len(sections)
    counts = _COUNTS[n].pack(*sections) if n < len(_COUNTS) else b""
    code = lib().spb_rotary_sections(out, n, counts, base, 1 if own_ladder else 0, 1 if interleaved else 0)
    if code:
        _check(code)
    return out


_STORED, _TYPES, _INT32 = None, {}, None      # torch's type -> dtype code, the other way round, torch's int32 (torch is imported by whoever has a tensor)


def _stored():
    global _STORED, _INT32
    if _STORED is None:
        import torch
        _STORED, _INT32 = {torch.float32: DTYPES["f32"], torch.bfloat16: DTYPES["bf16"]}, torch.int32
        _TYPES.update((code, t) for t, code in _STORED.items())
    return _STORED


def _dtype_code(t) -> int:
    code = _stored().get(t.dtype)
    if code is None:
        raise ValueError(f"{t.dtype}: only float32 and bfloat16 are stored")
    return code


# Filled in C in one go: field by field through ctypes a description took 12 us, twice the small kernels behind it.
_HEADS = struct.Struct("<7if9q")       # spb_heads_desc up to its rotary
_HEADS_READ = struct.Struct("<7if9q4i")    # and the rotary's pairs, interleaved, axes and reserved
assert _HEADS.size == spb_heads_desc.rotary.offset


def heads_desc(x, heads_q, y=None, dx=None, norm=False, eps=1e-5, rotary=None) -> spb_heads_desc:
    """Description of a spb_heads_forward call on x and y, or a spb_heads_backward call on x, dy (passed as y) and dx: tensors
    [batch, seq, heads, head_dim] of one dtype and any strides but that of the head's elements.  The first heads_q heads are queries, the
    rest keys.  y and dx default to x's strides."""
    d = spb_heads_desc()
    shape, dtype, sx = x.shape, x.dtype, x.stride()
    batch, seq, heads, dim = shape
    sy = sd = sx
    if y is not None:
        if y.shape != shape or y.dtype is not dtype:
            raise ValueError(f"y: {tuple(y.shape)} of {y.dtype}, x is {tuple(shape)} of {dtype}")
        sy = y.stride()
    if dx is not None:
        if dx.shape != shape or dx.dtype is not dtype:
            raise ValueError(f"dx: {tuple(dx.shape)} of {dx.dtype}, x is {tuple(shape)} of {dtype}")
        sd = dx.stride()
    if dim > 1 and not sx[3] == sy[3] == sd[3] == 1:
        raise ValueError("the elements of a head must be contiguous")
    code = _stored().get(dtype)
    if code is None:
        _dtype_code(x)                 # says what is stored
    _HEADS.pack_into(d, 0, code, batch, seq, heads_q, heads - heads_q, dim, 1 if norm else 0, eps, sx[0], sx[1], sx[2], sy[0], sy[1], sy[2],
                     sd[0], sd[1], sd[2])
    if rotary is not None:
        d.rotary = rotary
    return d


def _on(t, device, name):
    """Address of a tensor that has to lie on the GPU `device`, or None, or an address as it is."""
    if t is None or isinstance(t, int):
        return t
    if t.get_device() != device or device < 0:
        raise ValueError(f"{name} is on {t.device}, not on {'GPU ' + str(device) if device >= 0 else 'a GPU'}")
    return t.data_ptr()


def _described(f, device, *tensors):
    """Raises unless every (tensor, where its strides are in the description, name) is what the description f says, on the GPU `device`; a stride that nothing steps by may be another."""
    _stored()
    shape, dtype = (f[1], f[2], f[3] + f[4], f[5]), _TYPES.get(f[0])
    for t, at, name in tensors:
        steps = (*f[at:at + 3], 1)
        if t.shape != shape or t.dtype is not dtype or any(n > 1 and a != b for n, a, b in zip(shape, t.stride(), steps)):
            raise ValueError(f"{name}: {tuple(t.shape)} of {t.dtype} with strides {t.stride()}, described are {shape} of {dtype} with strides {steps}")
    for t, _at, name in sorted(tensors, key=lambda t: t[0].get_device()):      # (host memory first)
        _on(t, device, name)


def _positions(axes, batch, seq, pos):
    """(address, axis stride, batch stride) of positions [axes, batch, seq], int32; a batch dimension of 1 serves every sequence."""
    shape, stride = pos.shape, pos.stride()
    if len(shape) != 3 or _stored() and pos.dtype is not _INT32:
        raise ValueError(f"positions are int32 [axes, batch, seq], not {pos.dtype} {tuple(shape)}")
    has, by, long = shape
    if has < axes or (by != 1 and by != batch) or long != seq or (stride[2] != 1 and seq > 1):
        raise ValueError(f"positions {tuple(shape)} (last stride {stride[2]}) for {axes} axes of {batch} x {seq} tokens")
    return pos.data_ptr(), stride[0], 0 if by == 1 else stride[1]


def _weights(t, shape, code, device, name):
    """Address of a [rows of weights, head_dim] tensor, dense."""
    if t is None:
        return None
    if t.shape != shape or t.dtype is not _TYPES.get(code) or not t.is_contiguous():
        raise ValueError(f"{name}: {tuple(t.shape)} of {t.dtype}, contiguous {shape} of {_TYPES.get(code)} wanted")
    if t.get_device() != device:
        _on(t, device, name)
    return t.data_ptr()


def _workspace(t, size, device):
    """Address of a workspace tensor of at least `size` bytes."""
    if t is None or isinstance(t, int):
        return t
    if t.nbytes < size:
        raise ValueError(f"the workspace has {t.nbytes} bytes, not {size}")
    if t.get_device() != device:
        _on(t, device, "the workspace")
    return t.data_ptr()


_NOWHERE = None, 0, 0


def spb_heads_forward(desc, x, y, pos, gamma, beta, stream):
    """x and y as described (see heads_desc), all on one GPU."""
    f, device, sx, sy = _HEADS_READ.unpack_from(desc), x.get_device(), x.stride(), y.stride()
    if not (x.shape == y.shape == (f[1], f[2], f[3] + f[4], f[5]) and sx[:3] == f[8:11] and sy[:3] == f[11:14] and sx[3] == sy[3] == 1 and y.get_device() == device >= 0
            and x.dtype is y.dtype is _TYPES.get(f[0])):
        _described(f, device, (x, 8, "x"), (y, 11, "y"))
    if pos is None:
        where, by_axis, by_batch = _NOWHERE
    else:
        where, by_axis, by_batch = _positions(f[19], f[1], f[2], pos)
        if pos.get_device() != device:
            _on(pos, device, "positions")
    rc = lib().spb_heads_forward(desc, x.data_ptr(), y.data_ptr(), where, by_axis, by_batch, None if gamma is None else _weights(gamma, (2 if f[4] else 1, f[5]), f[0], device, "gamma"),
                                 None if beta is None else _weights(beta, (2 if f[4] else 1, f[5]), f[0], device, "beta"), stream)
    if rc:
        _check(rc)


def spb_heads_workspace_size(desc) -> int:
    n = C.c_size_t()
    rc = lib().spb_heads_workspace_size(desc, n)
    if rc:
        _check(rc)
    return n.value


def spb_heads_backward(desc, x, dy, dx, pos, gamma, dgamma, dbeta, workspace, workspace_bytes, stream):
    """x, dy and dx as described (see heads_desc), all on one GPU; x is not looked at without norm."""
    f, device, sy, sd = _HEADS_READ.unpack_from(desc), dy.get_device(), dy.stride(), dx.stride()
    fine = (dy.shape == dx.shape == (f[1], f[2], f[3] + f[4], f[5]) and sy[:3] == f[11:14] and sd[:3] == f[14:17] and sy[3] == sd[3] == 1
            and dx.get_device() == device >= 0 and dy.dtype is dx.dtype is _TYPES.get(f[0]))
    if not f[6] or x is None:
        if not fine:
            _described(f, device, (dy, 11, "dy"), (dx, 14, "dx"))
        x = None
    else:
        sx = x.stride()
        if not (fine and x.shape == dy.shape and sx[:3] == f[8:11] and sx[3] == 1 and x.get_device() == device and x.dtype is dy.dtype):
            _described(f, device, (x, 8, "x"), (dy, 11, "dy"), (dx, 14, "dx"))
        x = x.data_ptr()
    if pos is None:
        where, by_axis, by_batch = _NOWHERE
    else:
        where, by_axis, by_batch = _positions(f[19], f[1], f[2], pos)
        if pos.get_device() != device:
            _on(pos, device, "positions")
    shape = 2 if f[4] else 1, f[5]
    rc = lib().spb_heads_backward(desc, x, dy.data_ptr(), dx.data_ptr(), where, by_axis, by_batch, _weights(gamma, shape, f[0], device, "gamma"),
                                  _weights(dgamma, shape, _F32, device, "dgamma"), _weights(dbeta, shape, _F32, device, "dbeta"), _workspace(workspace, workspace_bytes, device),
                                  workspace_bytes, stream)
    if rc:
        _check(rc)


def spb_encoder_heads(m, rotary, pos, norm=False, eps=1e-5):
    """pos: [axes, batch or 1, seq] int32 on the device, for the model's batch and seq, which must outlive its passes; see spb.h."""
    where, by_axis, by_batch = None, 0, 0
    if pos is not None:
        if len(pos.shape) != 3:
            raise ValueError(f"positions are int32 [axes, batch, seq], not {pos.dtype} {tuple(pos.shape)}")
        # (seq 0: no encoder, which the call below says)
        batch, seq = (m.batch, m.seq) if getattr(m, "seq", 0) else pos.shape[1:]
        where, by_axis, by_batch = _positions(rotary.axes if rotary is not None else 0, batch, seq, pos)
    _check(lib().spb_encoder_heads(m, C.byref(rotary) if rotary is not None else None, where, by_axis, by_batch, int(bool(norm)), eps))


def muon_config(lr, rms=0.2, momentum=0.95, nesterov=True, ns_steps=5, ns_eps=1e-7, beta1=0.9, beta2=0.95, adam_eps=1e-8, weight_decay=0.0,
                step=1) -> spb_muon_config:
    return spb_muon_config(lr, rms, momentum, ns_eps, beta1, beta2, adam_eps, weight_decay, step, int(bool(nesterov)), ns_steps)


_MUON = struct.Struct("<4Q2qd4i")      # spb_muon_tensor
assert _MUON.size == C.sizeof(spb_muon_tensor)
_MUON_LAYOUT = "m, v and gradients are contiguous float32 tensors of the parameter's shape, which is contiguous too, all on one GPU"


def _muon_tensors(tensors, pointers=True):
    """List of tensors given as dict(w, m, v=None, grads=[...], blocks=0, rate_scale=1.0) as C lays it out, what keeps the arrays it points to
    alive, and their GPU.  A stack [blocks, rows, cols] is its matrices' rows one after the other; any other tensor has its first dimension as rows.  Without
    pointers: shapes only."""
    stored, packed = _stored(), []
    device = tensors[0]["w"].get_device() if tensors and pointers else 0
    held = array.array("Q", [g.data_ptr() for t in tensors for g in t["grads"]]) if pointers else None
    at = held.buffer_info()[0] if pointers else 0
    for t in tensors:
        w, blocks = t["w"], t.get("blocks", 0)
        shape, code = w.shape, stored.get(w.dtype)
        if code is None:
            _dtype_code(w)                 # says what is stored
        pw = pm = pv = pg = count = 0
        if pointers:
            m, v, grads = t["m"], t.get("v"), t["grads"]
            for x in (m, *grads) if v is None else (m, v, *grads):
                if stored.get(x.dtype) != _F32 or x.shape != shape or not x.is_contiguous() or x.get_device() != device:
                    raise ValueError(_MUON_LAYOUT)
            if not w.is_contiguous() or w.get_device() != device or device < 0:
                raise ValueError(_MUON_LAYOUT)
            pw, pm, pv, pg, count = w.data_ptr(), m.data_ptr(), 0 if v is None else v.data_ptr(), at, len(grads)
            at += 8 * count
        dims = len(shape)
        rows = shape[0] * shape[1] if dims == 3 and blocks >= 1 and shape[0] == blocks else shape[0] if dims else 1
        packed.append(_MUON.pack(pw, pm, pv, pg, rows, w.numel() // rows if rows else 0, t.get("rate_scale", 1.0), count, code, blocks, 0))
    return b"".join(packed), held, device


def spb_muon_workspace_size(tensors) -> int:
    """Shapes, types and blocks of the tensors are all it looks at."""
    n = C.c_size_t()
    _check(lib().spb_muon_workspace_size(_muon_tensors(tensors, pointers=False)[0], len(tensors), n))
    return n.value


def spb_muon_step(tensors, config: spb_muon_config, workspace, workspace_bytes, stream):
    listed, _held, device = _muon_tensors(tensors)
    _check(lib().spb_muon_step(listed, len(tensors), config, _workspace(workspace, workspace_bytes, device), workspace_bytes, stream))


def _one_per_parameter(m, *lists):
    n = spb_param_count(m)
    if any(len(x) != n for x in lists):
        raise ValueError(f"lists of {sorted({len(x) for x in lists})} entries for {n} parameters")


def spb_aggregate_muon_workspace_size(m, blocks) -> int:
    n = C.c_size_t()
    _one_per_parameter(m, blocks)
    _check(lib().spb_aggregate_muon_workspace_size(m, (C.c_int32 * len(blocks))(*blocks), C.byref(n)))
    return n.value


def spb_aggregate_muon(m, depths, worker_grads, blocks, first, second, config: spb_muon_config, scale_lr, workspace, workspace_bytes, stream):
    """worker_grads as in spb_aggregate_update; blocks, first, second: one entry per parameter (second: None for matrices)."""
    n = len(depths)
    if len(worker_grads) != n:
        raise ValueError(f"gradients of {len(worker_grads)} workers, depths of {n}")
    _one_per_parameter(m, blocks, first, second, *worker_grads)
    flat = [g for per_worker in worker_grads for g in per_worker]
    held = workspace is None or isinstance(workspace, int)
    _check(lib().spb_aggregate_muon(m, n, (C.c_int32 * n)(*depths), _ptr_array(flat), (C.c_int32 * len(blocks))(*blocks), _ptr_array(first),
                                    _ptr_array(second), C.byref(config), int(bool(scale_lr)),
                                    workspace if held else _workspace(workspace, workspace_bytes, max(workspace.get_device(), 0)), workspace_bytes, C.c_void_p(stream)))


def spb_set_kernel_timing(m, enable: bool):
    _check(lib().spb_set_kernel_timing(m, int(enable)))


def spb_replay_kernel(m, name: str, count: int, stream):
    _check(lib().spb_replay_kernel(m, name.encode(), count, C.c_void_p(stream)))


def spb_read_kernel_timing(m, cap=1024):
    recs = (spb_kernel_time * cap)()
    n = C.c_int32()
    _check(lib().spb_read_kernel_timing(m, recs, cap, C.byref(n)))
    return [{"name": r.name.decode(), "launches": r.launches, "total_ms": r.total_ms, "flops": r.flops,
             "bytes": r.bytes} for r in recs[:n.value]]


def spb_schedule_tasks(jobs, n_machines: int, gamma: float = 0.0, capacity: float = 1.0, gang: bool = False):
    """jobs: list of dict(arrival, iterations, model_size, durations[w], resources[w]) -> (placements, makespan),
    placements as dicts in the order the library placed them (host computation, no GPU)."""
    arr = (spb_sched_job * max(1, len(jobs)))()
    keep = []
    total = 0
    for a, job in zip(arr, jobs):
        w = len(job["durations"])
        if len(job["resources"]) != w:
            raise ValueError("one duration and one resource per worker")
        d = (C.c_double * max(1, w))(*[float(v) for v in job["durations"]])
        r = (C.c_double * max(1, w))(*[float(v) for v in job["resources"]])
        keep += [d, r]
        a.arrival, a.model_size, a.iterations, a.workers = float(job["arrival"]), float(job["model_size"]), int(job["iterations"]), w
        a.durations, a.resources = d, r
        total += w * max(0, int(job["iterations"]))
    out = (spb_sched_task * max(1, total))()
    n, makespan = C.c_int64(), C.c_double()
    _check(lib().spb_schedule_tasks(arr, len(jobs), int(n_machines), float(gamma), float(capacity), int(bool(gang)), out, total,
                                    C.byref(n), C.byref(makespan)))
    # one record per task, unpacked in C (reading the fields through ctypes took 0.9 us a task, twice the placement itself)
    return ([{"job": j, "iteration": i, "worker": w, "machine": m, "start": start, "end": end, "held_until": held, "moved": moved}
             for j, i, w, m, moved, start, end, held in _TASK.iter_unpack(memoryview(out).cast("B")[:n.value * _TASK.size])], makespan.value)


class SpbModel:
    """Convenience holder: a model handle plus the torch tensors bound to it (memory and stream plumbing only)."""

    def __init__(self, cfg: dict, params: dict, device="cuda:0", positions=None):
        """An encoder's cfg may hold rotary=dict(sections, base, own_ladder, interleaved) and qk_norm=eps (see spb_encoder_heads); positions:
        int32 [axes, batch or 1, seq] of its tokens."""
        import torch
        self.torch = torch
        self.cfg = cfg
        self.device = torch.device(device)
        if self.device.type != "cuda" or not torch.cuda.is_available():
            raise RuntimeError("the SPB path needs a GPU; there is no host fallback")
        self.handle = spb_model_create(desc_from_config(cfg))
        if cfg.get("rotary") or cfg.get("qk_norm"):
            rotary = spb_rotary_sections(**cfg["rotary"]) if cfg.get("rotary") else None
            if positions is not None and (positions.shape[1] not in (1, cfg["batch"]) or positions.shape[2] != cfg["seq"]):
                raise ValueError(f"positions {tuple(positions.shape)} for {cfg['batch']} x {cfg['seq']} tokens")
            self.positions = None if positions is None else positions.to(self.device, torch.int32).contiguous()
            spb_encoder_heads(self.handle, rotary, self.positions, norm=bool(cfg.get("qk_norm")), eps=cfg.get("qk_norm") or 1e-5)
        self.n_units = spb_num_units(self.handle)
        self.infos = [spb_param_info(self.handle, i) for i in range(spb_param_count(self.handle))]
        self.params, self.grads = [], []
        for info in self.infos:
            src = params[info["name"]]
            if tuple(src.shape) != info["shape"]:
                raise ValueError(f"{info['name']}: shape {tuple(src.shape)} != {info['shape']}")
            self.params.append(src.to(self.device).contiguous())
            self.grads.append(torch.empty(info["shape"], dtype=torch.float32, device=self.device))
        spb_bind_params(self.handle, self.params)
        spb_bind_grads(self.handle, self.grads)
        self.loss = torch.zeros(1, dtype=torch.float32, device=self.device)
        self.workspace = None
        self.workspace_bytes = 0

    def reserve(self, k: int):
        need = spb_workspace_size(self.handle, k)
        if need > self.workspace_bytes:
            self.workspace = self.torch.empty(need, dtype=self.torch.uint8, device=self.device)
            self.workspace_bytes = need
        return need

    def stream(self) -> int:
        return self.torch.cuda.current_stream(self.device).cuda_stream

    def forward(self, batch: dict, k: int):
        self.reserve(k)
        spb_forward(self.handle, batch["x"], batch["labels"], batch.get("loss_rows"), k, self.workspace,
                    self.workspace_bytes, self.loss, self.stream())

    def forward_static(self, batch: dict, k: int):
        """The forward pass on the library's own fixed-size workspace (allocates nothing)."""
        spb_forward_static(self.handle, batch["x"], batch["labels"], batch.get("loss_rows"), k, self.loss, self.stream())

    def backward(self, k: int):
        spb_backward_truncated(self.handle, k, self.stream())

    def step(self, batch: dict, k: int):
        self.forward(batch, k)
        self.backward(k)

    def grad_dict(self, k: int) -> dict:
        """name -> float32 tensor view of the buffers spb_grad_buffers lists at depth k."""
        out = {}
        for v in spb_grad_buffers(self.handle, k):
            g = self.grads[v["param_index"]]
            assert g.data_ptr() == v["data"] and g.numel() == v["numel"]
            out[self.infos[v["param_index"]]["name"]] = g
        return out

    def read_view(self, view: dict, batch: dict = None):
        """The tensor a spb_unit_io view describes, copied out of the workspace as a float64 (ids: int64) CPU tensor
        [rows, cols]; None for SPB_VIEW_NONE."""
        torch = self.torch
        if view["offset"] == SPB_VIEW_NONE:
            return None
        if view["offset"] == SPB_VIEW_CALLER_INPUT:
            x = batch["x"].detach().cpu()
            return x.reshape(view["rows"], -1).long() if view["dtype"] == "i32" else x.reshape(view["rows"], -1).double()
        tdtype, size = {"f32": (torch.float32, 4), "bf16": (torch.bfloat16, 2)}[view["dtype"]]
        nbytes = ((view["rows"] - 1) * view["pitch"] + view["cols"]) * size
        raw = self.workspace[view["offset"]:view["offset"] + nbytes].view(tdtype)
        return torch.as_strided(raw, (view["rows"], view["cols"]), (view["pitch"], 1)).double().cpu()

    def close(self):
        if self.handle is not None:
            spb_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
