"""Binding of the C ABI in include/qlora.h.  Same names, same argument order; tensors are passed as their device pointers and
`stream=None` means torch's current CUDA stream.  No arithmetic happens here.  The calls of a training or generation loop go
through the C extension of csrc/pycall.cpp, the others through ctypes."""
from __future__ import annotations

import ctypes
import os

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG_DIR, "libqlora_b200.so")
_lib = None
_calls = None


class QloraError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where} failed: {qlora_status_string(status)} ({status})")


class _Desc(ctypes.Structure):
    _fields_ = [("bits", ctypes.c_int), ("group_size", ctypes.c_int), ("K", ctypes.c_int), ("N", ctypes.c_int),
                ("r", ctypes.c_int), ("alpha", ctypes.c_float)]


class _AdamwTensor(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in ("param", "master", "grad", "m", "v", "m_scale", "v_scale")] + [("n", ctypes.c_longlong)]


class _AdamwDesc(ctypes.Structure):
    _fields_ = [("n_tensors", ctypes.c_int), ("tensors", ctypes.POINTER(_AdamwTensor)), ("param_type", ctypes.c_int), ("grad_type", ctypes.c_int),
                ("state_type", ctypes.c_int), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double)]


class _AdaptersDesc(ctypes.Structure):
    _fields_ = [("K", ctypes.c_int), ("N", ctypes.c_int), ("r", ctypes.c_int), ("n_adapters", ctypes.c_int)]


def desc(bits: int, group_size: int, K: int, N: int, r: int, alpha: float) -> _Desc:
    """Layer descriptor (qlora_desc)."""
    return _Desc(int(bits), int(group_size), int(K), int(N), int(r), float(alpha))


def adapters_desc(K: int, N: int, r: int, n_adapters: int) -> _AdaptersDesc:
    """Descriptor (qlora_adapters_desc) of the adapters of one projection."""
    return _AdaptersDesc(int(K), int(N), int(r), int(n_adapters))


def library_path() -> str:
    return _LIB_PATH


def library() -> ctypes.CDLL:
    """Load the CUDA library (built in-tree by paper_2306_08162_b200.build).  Raises if it is not there."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2306_08162_b200.build` "
                           "(there is no fallback path)")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    dp = ctypes.POINTER(_Desc)
    lib.qlora_status_string.restype = ctypes.c_char_p
    lib.qlora_status_string.argtypes = [i32]
    lib.qlora_workspace_bytes.argtypes = [dp, i32, ctypes.POINTER(sz)]
    lib.qlora_fwd.argtypes = [dp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.qlora_bwd_input.argtypes = [dp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.qlora_bwd_lora.argtypes = [dp, i32, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp]
    lib.qlora_bwd_input_db_on_producers.argtypes = [dp, i32]
    lib.qlora_bwd_input_db_on_producers.restype = i32
    lib.qlora_bwd_input_db.argtypes = [dp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp]
    f32 = ctypes.c_float
    lib.qlora_fwd_dropout.argtypes = [dp, i32, vp, vp, f32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.qlora_bwd_input_dropout.argtypes = [dp, i32, vp, vp, f32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.qlora_bwd_lora_dropout.argtypes = [dp, i32, vp, vp, f32, vp, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp]
    lib.qlora_bwd_lora_static.argtypes = [dp, i32, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp]
    lib.qlora_pack.argtypes = [i32, i32, i32, vp, vp, vp]
    lib.qlora_unpack.argtypes = [i32, i32, i32, vp, vp, vp]
    lib.qlora_dequant.argtypes = [dp, vp, vp, vp, vp, vp]
    lib.qlora_quantize_rtn.argtypes = [dp, vp, vp, vp, vp, vp]
    lib.qlora_gather_columns.argtypes = [i32, i32, i32, vp, vp, vp, vp]
    lib.qlora_lrec_loss.argtypes = [i32, i32, vp, vp, vp, ctypes.c_float, ctypes.c_float, ctypes.c_float, vp, vp, vp]
    i64, f64, ap = ctypes.c_longlong, ctypes.c_double, ctypes.POINTER(_AdamwDesc)
    lib.qlora_token_logprobs.argtypes = [i32, i32, i64, i32, vp, vp, f32, i32, vp, vp, vp, vp, vp, vp]
    lib.qlora_token_logprobs_bwd.argtypes = [i32, i32, i64, i32, vp, vp, f32, vp, vp, vp, i64, vp, vp]
    lib.qlora_grad_norm.argtypes = [ap, f32, f32, vp, vp, sz, vp]
    lib.qlora_adamw.argtypes = [ap, f64, i32, vp, vp, vp, vp]
    dd = ctypes.POINTER(_AdaptersDesc)
    lib.qlora_adapters_workspace_bytes.argtypes = [dd, i32, ctypes.POINTER(sz)]
    lib.qlora_adapters_fwd.argtypes = [dd, i32] + [vp] * 9 + [sz, vp]
    lib.qlora_adapters_bwd_input.argtypes = [dd, i32] + [vp] * 9 + [sz, vp]
    lib.qlora_adapters_bwd_lora.argtypes = [dd, i32] + [vp] * 10 + [i32, vp, sz, vp]
    lib.qlora_head_loss_workspace_bytes.argtypes = [i32, i32, i32, i32, ctypes.POINTER(sz)]
    lib.qlora_head_loss.argtypes = [i32, i32, i32] + [vp] * 7 + [sz, vp]
    lib.qlora_device_status.argtypes = [ctypes.POINTER(ctypes.c_uint), i32]
    lib.qlora_selftest_bounded_wait.argtypes = [i32, vp]
    for name in ("qlora_workspace_bytes", "qlora_fwd", "qlora_bwd_input", "qlora_bwd_input_db", "qlora_bwd_lora", "qlora_bwd_lora_static", "qlora_fwd_dropout", "qlora_bwd_input_dropout",
                 "qlora_bwd_lora_dropout", "qlora_pack",
                 "qlora_unpack", "qlora_dequant", "qlora_quantize_rtn", "qlora_gather_columns", "qlora_lrec_loss", "qlora_device_status", "qlora_selftest_bounded_wait",
                 "qlora_token_logprobs", "qlora_token_logprobs_bwd", "qlora_grad_norm", "qlora_adamw",
                 "qlora_adapters_workspace_bytes", "qlora_adapters_fwd", "qlora_adapters_bwd_input", "qlora_adapters_bwd_lora",
                 "qlora_head_loss_workspace_bytes", "qlora_head_loss"):
        getattr(lib, name).restype = i32
    _lib = lib
    return lib


def _native():
    """The C extension with the calls of the hot path (built in-tree together with the library)."""
    global _calls
    if _calls is None:
        library()
        from . import _pycall
        _pycall.set_desc_types((_Desc, _AdamwDesc, _AdaptersDesc))
        _calls = _pycall
    return _calls


def _ptr(t):
    """Device pointer of a torch tensor; None -> NULL; an int is passed through (tests of the error paths)."""
    if t is None:
        return None
    if isinstance(t, int):
        return ctypes.c_void_p(t)
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous (dense row-major)")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        import torch
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    if isinstance(stream, int):
        return ctypes.c_void_p(stream)
    return ctypes.c_void_p(stream.cuda_stream)


def _check(status: int, where: str):
    if status != 0:
        raise QloraError(status, where)


def qlora_status_string(status: int) -> str:
    return library().qlora_status_string(int(status)).decode()


def qlora_workspace_bytes(d: _Desc, M: int) -> int:
    out = ctypes.c_size_t(0)
    _check(library().qlora_workspace_bytes(ctypes.byref(d), int(M), ctypes.byref(out)), "qlora_workspace_bytes")
    return int(out.value)


def qlora_fwd(d, M, X, Q, scales, zeros, A, B, Y, H_out, workspace, stream=None, workspace_bytes=None):
    rc = _native().qlora_fwd(d, M, X, Q, scales, zeros, A, B, Y, H_out, workspace, workspace_bytes, stream)
    if rc != 0:
        raise QloraError(rc, "qlora_fwd")


def qlora_bwd_input(d, M, dY, Q, scales, zeros, A, B, dX, G_out, workspace, stream=None, workspace_bytes=None):
    rc = _native().qlora_bwd_input(d, M, dY, Q, scales, zeros, A, B, dX, G_out, workspace, workspace_bytes, stream)
    if rc != 0:
        raise QloraError(rc, "qlora_bwd_input")


def qlora_bwd_input_db(d, M, dY, Q, scales, zeros, A, B, H, dX, G_out, dB, accumulate, workspace, stream=None, workspace_bytes=None):
    rc = _native().qlora_bwd_input_db(d, M, dY, Q, scales, zeros, A, B, H, dX, G_out, dB, accumulate, workspace, workspace_bytes, stream)
    if rc != 0:
        raise QloraError(rc, "qlora_bwd_input_db")


def qlora_bwd_input_db_on_producers(d, M) -> bool:
    rc = library().qlora_bwd_input_db_on_producers(ctypes.byref(d), int(M))
    if rc < 0:
        _check(rc, "qlora_bwd_input_db_on_producers")
    return rc == 1


def qlora_bwd_lora(d, M, X, dY, A, B, H, G, dA, dB, accumulate, workspace, stream=None, workspace_bytes=None):
    rc = _native().qlora_bwd_lora(d, M, X, dY, A, B, H, G, dA, dB, accumulate, workspace, workspace_bytes, stream)
    if rc != 0:
        raise QloraError(rc, "qlora_bwd_lora")


def qlora_fwd_dropout(d, M, X, mask, keep_scale, Q, scales, zeros, A, B, Y, H_out, workspace, stream=None, workspace_bytes=None):
    rc = _native().qlora_fwd_dropout(d, M, X, mask, keep_scale, Q, scales, zeros, A, B, Y, H_out, workspace, workspace_bytes, stream)
    if rc != 0:
        raise QloraError(rc, "qlora_fwd_dropout")


def qlora_bwd_input_dropout(d, M, dY, mask, keep_scale, Q, scales, zeros, A, B, dX, G_out, workspace, stream=None,
                            workspace_bytes=None):
    rc = _native().qlora_bwd_input_dropout(d, M, dY, mask, keep_scale, Q, scales, zeros, A, B, dX, G_out, workspace, workspace_bytes, stream)
    if rc != 0:
        raise QloraError(rc, "qlora_bwd_input_dropout")


def qlora_bwd_lora_dropout(d, M, X, mask, keep_scale, dY, A, B, H, G, dA, dB, accumulate, workspace, stream=None,
                           workspace_bytes=None):
    rc = _native().qlora_bwd_lora_dropout(d, M, X, mask, keep_scale, dY, A, B, H, G, dA, dB, accumulate, workspace, workspace_bytes, stream)
    if rc != 0:
        raise QloraError(rc, "qlora_bwd_lora_dropout")


STATIC_SCRATCH_BYTES = 16 << 20   # QLORA_STATIC_SCRATCH_BYTES


def qlora_bwd_lora_static(d, M, X, dY, A, B, H, G, dA, dB, accumulate, stream=None):
    """qlora_bwd_lora for callers that may not allocate device memory: no workspace argument, the scratch is an array
    inside the library (STATIC_SCRATCH_BYTES).  Raises QloraError(-7) when the shape needs more than that."""
    _check(library().qlora_bwd_lora_static(ctypes.byref(d), int(M), _ptr(X), _ptr(dY), _ptr(A), _ptr(B), _ptr(H), _ptr(G),
                                           _ptr(dA), _ptr(dB), int(accumulate), _stream(stream)),
           "qlora_bwd_lora_static")


def qlora_pack(bits, K, N, codes, Q, stream=None):
    _check(library().qlora_pack(int(bits), int(K), int(N), _ptr(codes), _ptr(Q), _stream(stream)), "qlora_pack")


def qlora_unpack(bits, K, N, Q, codes, stream=None):
    _check(library().qlora_unpack(int(bits), int(K), int(N), _ptr(Q), _ptr(codes), _stream(stream)), "qlora_unpack")


def qlora_lrec_loss(student_logits, teacher_logits, labels, lambda_kl, lambda_ce, grad_scale, loss_tokens, dlogits, stream=None):
    """Fused KL + cross-entropy loss of the error-correction objective and its gradient; logits bf16 [T, V]."""
    T, V = student_logits.shape
    rc = _native().qlora_lrec_loss(T, V, student_logits, teacher_logits, labels, lambda_kl, lambda_ce, grad_scale, loss_tokens, dlogits, stream)
    if rc != 0:
        raise QloraError(rc, "qlora_lrec_loss")


_torch = None
_TYPES = {}                      # torch dtype -> QLORA_BF16, QLORA_FP16, QLORA_FP32, QLORA_E4M3
_LOGIT_TYPES = (0, 1, 2)


def _load_torch():
    """torch and the element types, at the first call that needs them (the package itself can be imported without)."""
    global _torch
    if _torch is None:
        import torch
        _TYPES.update({torch.bfloat16: 0, torch.float16: 1, torch.float32: 2, torch.float8_e4m3fn: 3})
        _torch = torch
    return _torch


def _type_of(t, where: str, allowed) -> int:
    code = _TYPES.get(t.dtype, -1)
    if code not in allowed:
        raise ValueError(f"{where}: {t.dtype} is not supported here")
    return code


def _current_device(where: str) -> int:
    """The current CUDA device, on which the library works: a tensor of another one, or of the host, in a kernel's hands would be a fault."""
    if _torch.cuda.is_initialized():
        return _torch._C._cuda_getDevice()
    if not _torch.cuda.is_available():
        raise ValueError(f"{where}: tensors must be on the current CUDA device, and there is none")
    return _torch.cuda.current_device()


def _rows(t, where: str):
    """Shape and row stride of a 2-D tensor whose rows are dense (they may lie apart and begin anywhere)."""
    if t.dim() != 2:
        raise ValueError(f"{where}: a 2-D tensor with dense rows is needed")
    (T, V), (stride, step) = t.shape, t.stride()
    if step != 1 and V > 1:
        raise ValueError(f"{where}: a 2-D tensor with dense rows is needed")
    return T, V, stride if T > 1 else V


def _operands(where: str, device: int, *wanted):
    """The operands beside the logits: each None or of the type, the size and on the device that the library will assume."""
    for t, dtype, shape in wanted:
        if t is not None and (t.dtype is not dtype or t.shape != shape or t.get_device() != device):
            if t.dtype is not dtype or t.shape != shape:
                raise ValueError(f"{where}: {dtype} {list(shape)} is needed, got {t.dtype} {list(t.shape)}")
            raise ValueError(f"{where}: tensors must be on the current CUDA device, got {t.device}")


def qlora_token_logprobs(logits, tokens, inv_temperature, logprobs, entropy=None, top_ids=None, top_logprobs=None, stats=None, stream=None):
    """Log probabilities of `tokens` (int32 [T], or None) under logits [T, V] (bf16, fp16 or fp32; rows may lie apart), the entropy of each
    row and its k most likely places (k = top_ids.shape[1]); stats fp32 [T, 3] is what the backward call reads.  Outputs may be None."""
    where = "qlora_token_logprobs"
    torch = _torch or _load_torch()
    T, V, stride = _rows(logits, where)
    dtype = _type_of(logits, where, _LOGIT_TYPES)
    f32, i32, row, k = torch.float32, torch.int32, (T,), 0
    if top_ids is not None or top_logprobs is not None:
        top = top_ids if top_ids is not None else top_logprobs
        if top.dim() != 2:
            raise ValueError(f"{where}: the alternatives are [T, k]")
        k = top.shape[1]
    device = logits.get_device()
    _operands(where, device, (tokens, i32, row), (logprobs, f32, row), (entropy, f32, row), (top_ids, i32, (T, k)), (top_logprobs, f32, (T, k)), (stats, f32, (T, 3)))
    if device != _current_device(where):
        raise ValueError(f"{where}: tensors must be on the current CUDA device, got {logits.device}")
    rc = _native().qlora_token_logprobs(T, V, stride, dtype, logits.data_ptr(), tokens, inv_temperature, k, logprobs, entropy, top_ids, top_logprobs,
                                        stats, stream)
    if rc != 0:
        raise QloraError(rc, where)


def qlora_token_logprobs_bwd(logits, tokens, inv_temperature, stats, d_logprobs, d_entropy, dlogits, stream=None):
    """Gradient of qlora_token_logprobs with respect to the logits, into dlogits [T, V] (the logits' type; rows may lie apart; may be the
    logits themselves)."""
    where = "qlora_token_logprobs_bwd"
    torch = _torch or _load_torch()
    T, V, stride = _rows(logits, where)
    dtype = _type_of(logits, where, _LOGIT_TYPES)
    Tg, Vg, grad_stride = _rows(dlogits, where)
    if Tg != T or Vg != V or dlogits.dtype is not logits.dtype:
        raise ValueError(f"{where}: dlogits has the shape and the type of logits")
    f32, row, device = torch.float32, (T,), logits.get_device()
    _operands(where, device, (tokens, torch.int32, row), (stats, f32, (T, 3)), (d_logprobs, f32, row), (d_entropy, f32, row), (dlogits, logits.dtype, (T, V)))
    if device != _current_device(where):
        raise ValueError(f"{where}: tensors must be on the current CUDA device, got {logits.device}")
    rc = _native().qlora_token_logprobs_bwd(T, V, stride, dtype, logits.data_ptr(), tokens, inv_temperature, stats, d_logprobs, d_entropy, grad_stride,
                                            dlogits.data_ptr(), stream)
    if rc != 0:
        raise QloraError(rc, where)


GRAD_NORM_WORKSPACE_BYTES = 8192   # QLORA_GRAD_NORM_WORKSPACE_BYTES


def adamw_desc(params, grads, m, v, master=None, m_scale=None, v_scale=None, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0) -> _AdamwDesc:
    """Descriptor (qlora_adamw_desc) of the optimizer step over a list of parameters: made once, used every step.  All lists have one tensor
    per parameter.  m and v are fp32, or float8_e4m3fn with m_scale and v_scale (fp32, one for every 256 elements, rounded up); master
    (fp32) or None.  The descriptor holds the tensors' addresses and keeps the tensors alive: a gradient that is allocated anew needs a
    new descriptor."""
    import bisect
    where = "adamw_desc"
    _load_torch()
    lists = dict(param=params, master=master, grad=grads, m=m, v=v, m_scale=m_scale, v_scale=v_scale)
    lists = {name: list(ts) for name, ts in lists.items() if ts is not None}
    n = len(lists["param"])
    for name, ts in lists.items():
        if len(ts) != n:
            raise ValueError(f"{where}: {len(ts)} tensors in {name}, {n} parameters")
    d = _AdamwDesc(n_tensors=n, param_type=2, grad_type=2, state_type=2, beta1=beta1, beta2=beta2, eps=eps, weight_decay=weight_decay)
    d.keep, d.device = lists, None
    if n == 0:
        return d
    d.param_type, d.grad_type, d.state_type = (_type_of(lists[name][0], f"{where}: {name}", allowed)
                                               for name, allowed in (("param", _LOGIT_TYPES), ("grad", _LOGIT_TYPES), ("m", (2, 3))))
    eight = d.state_type == 3
    if ("m_scale" in lists, "v_scale" in lists) != (eight, eight):
        raise ValueError(f"{where}: m_scale and v_scale go with states in 8 bits, and only with those")
    if "master" in lists and d.param_type == 2:
        raise ValueError(f"{where}: fp32 parameters have no master weights")
    sizes = [t.numel() for t in lists["param"]]
    blocks = [-(-size // 256) for size in sizes]
    columns, written, read, devices = {}, [], [], set()
    for name, ts in lists.items():
        kind = {"param": d.param_type, "grad": d.grad_type, "m": d.state_type, "v": d.state_type}.get(name, 2)
        wanted = blocks if name.endswith("_scale") else sizes
        for dtype in {t.dtype for t in ts}:
            if _TYPES.get(dtype) != kind:
                raise ValueError(f"{where}: {dtype} is not supported as {name} here (one call, one type)")
        found = [t.numel() for t in ts]
        if found != wanted:
            j = next(j for j in range(n) if found[j] != wanted[j])
            raise ValueError(f"{where}: {name}[{j}] has {found[j]} elements for a parameter of {sizes[j]}")
        if not all(t.is_contiguous() for t in ts):
            raise ValueError(f"{where}: tensors must be contiguous (dense)")
        columns[name] = at = [t.data_ptr() for t in ts]
        bytes_each = ts[0].element_size()
        (read if name == "grad" else written).extend((a, a + size * bytes_each) for a, size in zip(at, found) if size)
        devices.update(t.get_device() for t in ts)
    written.sort()
    for (_, end), (begin, _) in zip(written, written[1:]):
        if begin < end:
            raise ValueError(f"{where}: two of the tensors that the step writes overlap (the same one twice?)")
    for begin, end in read:
        at = bisect.bisect_left(written, (end,))                      # the last written range that begins before this one ends
        if at > 0 and written[at - 1][1] > begin:
            raise ValueError(f"{where}: a gradient overlaps a tensor that the step writes")
    if len(devices) != 1 or min(devices) < 0:
        raise ValueError(f"{where}: tensors must be on one CUDA device")
    # the structures' fields in order, all of them 64 bits wide
    none = [0] * n
    fields = [columns.get(name, none) for name, _ in _AdamwTensor._fields_[:-1]] + [sizes]
    array = (ctypes.c_longlong * (len(fields) * n))(*(value for tensor in zip(*fields) for value in tensor))
    d.tensors, d.device = ctypes.cast(array, ctypes.POINTER(_AdamwTensor)), devices.pop()
    d.keep = (array, lists)
    return d


def _desc_device(d, where: str) -> int:
    if not isinstance(d, _AdamwDesc):
        raise TypeError(f"{where}: the optimizer descriptor must come from adamw_desc()")
    if _torch is None:
        _load_torch()
    device = _current_device(where)
    if d.device is not None and d.device != device:
        raise ValueError(f"{where}: the descriptor's tensors are on device {d.device}, the current one is {device}")
    return device


def qlora_grad_norm(d, prescale, max_norm, out, workspace, stream=None, workspace_bytes=None):
    """out fp32 [2]: the norm of prescale times all gradients of the descriptor, and the factor for qlora_adamw that clips it to max_norm."""
    where = "qlora_grad_norm"
    device = _desc_device(d, where)
    _operands(where, device, (out, _torch.float32, (2,)))
    if workspace is not None and workspace.get_device() != device:
        raise ValueError(f"{where}: tensors must be on the current CUDA device, got {workspace.device}")
    rc = _native().qlora_grad_norm(d, prescale, max_norm, out, workspace, workspace_bytes, stream)
    if rc != 0:
        raise QloraError(rc, where)


def qlora_adamw(d, lr, step, norm=None, stream=None):
    """One AdamW step over the descriptor's tensors.  lr: a number or an fp32 tensor [1]; step: an int from 1 or an int32 tensor [1] (device
    memory that a captured step reads at replay); norm: fp32 [2] from qlora_grad_norm or None."""
    where = "qlora_adamw"
    device = _desc_device(d, where)
    lr_dev = step_dev = None
    if not isinstance(lr, float) and hasattr(lr, "data_ptr"):
        lr, lr_dev = 0.0, lr
    if not isinstance(step, int) and hasattr(step, "data_ptr"):
        step, step_dev = 0, step
    _operands(where, device, (lr_dev, _torch.float32, (1,)), (step_dev, _torch.int32, (1,)), (norm, _torch.float32, (2,)))
    rc = _native().qlora_adamw(d, lr, step, lr_dev, step_dev, norm, stream)
    if rc != 0:
        raise QloraError(rc, where)


def qlora_adapters_workspace_bytes(d: _AdaptersDesc, M: int) -> int:
    out = ctypes.c_size_t(0)
    _check(library().qlora_adapters_workspace_bytes(ctypes.byref(d), int(M), ctypes.byref(out)), "qlora_adapters_workspace_bytes")
    return int(out.value)


def _adapters_operands(where, d, M, adapter_of, A, B, scales, workspace, *more):
    if not isinstance(d, _AdaptersDesc):
        raise TypeError(f"{where}: the adapters' descriptor must come from adapters_desc()")
    torch = _torch or _load_torch()
    device, bf16, L, r = _current_device(where), torch.bfloat16, d.n_adapters, d.r
    _operands(where, device, (adapter_of, torch.int32, (M,)), (A, bf16, (L, r, d.K)), (B, bf16, (L, d.N, r)), (scales, torch.float32, (L,)),
              *((t, torch.float32 if low else bf16, shape) for t, low, shape in more))
    if workspace is not None and workspace.get_device() != device:
        raise ValueError(f"{where}: tensors must be on the current CUDA device, got {workspace.device}")


def qlora_adapters_fwd(d, M, X, adapter_of, A, B, scales, Y_base, Y, H_out, workspace, stream=None, workspace_bytes=None):
    """Y[t] = Y_base[t] + scales[a] (X[t] A_a^T) B_a^T with a = adapter_of[t] (none outside [0, n_adapters)); Y may be Y_base, H_out may be None."""
    where = "qlora_adapters_fwd"
    _adapters_operands(where, d, M, adapter_of, A, B, scales, workspace, (X, False, (M, d.K)), (Y_base, False, (M, d.N)), (Y, False, (M, d.N)),
                       (H_out, True, (M, d.r)))
    rc = _native().qlora_adapters_fwd(d, M, X, adapter_of, A, B, scales, Y_base, Y, H_out, workspace, workspace_bytes, stream)
    if rc != 0:
        raise QloraError(rc, where)


def qlora_adapters_bwd_input(d, M, dY, adapter_of, A, B, scales, dX_base, dX, G_out, workspace, stream=None, workspace_bytes=None):
    """dX[t] = dX_base[t] + scales[a] (dY[t] B_a) A_a; dX may be dX_base, G_out may be None."""
    where = "qlora_adapters_bwd_input"
    _adapters_operands(where, d, M, adapter_of, A, B, scales, workspace, (dY, False, (M, d.N)), (dX_base, False, (M, d.K)), (dX, False, (M, d.K)),
                       (G_out, True, (M, d.r)))
    rc = _native().qlora_adapters_bwd_input(d, M, dY, adapter_of, A, B, scales, dX_base, dX, G_out, workspace, workspace_bytes, stream)
    if rc != 0:
        raise QloraError(rc, where)


def qlora_adapters_bwd_lora(d, M, X, dY, adapter_of, A, B, scales, H, G, dA, dB, accumulate, workspace, stream=None, workspace_bytes=None):
    """dA fp32 [n_adapters, r, K] and dB fp32 [n_adapters, N, r] of every adapter; H and G as the calls above left them, or None (recomputed)."""
    where = "qlora_adapters_bwd_lora"
    _adapters_operands(where, d, M, adapter_of, A, B, scales, workspace, (X, False, (M, d.K)), (dY, False, (M, d.N)), (H, True, (M, d.r)), (G, True, (M, d.r)),
                       (dA, True, (d.n_adapters, d.r, d.K)), (dB, True, (d.n_adapters, d.N, d.r)))
    rc = _native().qlora_adapters_bwd_lora(d, M, X, dY, adapter_of, A, B, scales, H, G, dA, dB, accumulate, workspace, workspace_bytes, stream)
    if rc != 0:
        raise QloraError(rc, where)


def qlora_head_loss_workspace_bytes(T: int, V: int, D: int, gradient: bool) -> int:
    out = ctypes.c_size_t(0)
    _check(library().qlora_head_loss_workspace_bytes(int(T), int(V), int(D), 1 if gradient else 0, ctypes.byref(out)), "qlora_head_loss_workspace_bytes")
    return int(out.value)


def qlora_head_loss(hidden, head, labels, loss_tokens, workspace, d_loss=None, d_hidden=None, stream=None, workspace_bytes=None):
    """Cross entropy of labels (int32 [T]; outside [0, V): none) under softmax(hidden head^T), hidden bf16 [T, D], head bf16 [V, D], into loss_tokens fp32 [T];
    with d_loss (fp32 [T]) and d_hidden (bf16 [T, D], may be hidden itself) also its gradient with respect to hidden."""
    where = "qlora_head_loss"
    torch = _torch or _load_torch()
    if hidden.dim() != 2 or head.dim() != 2:
        raise ValueError(f"{where}: hidden is [T, D] and head [V, D]")
    (T, D), V = hidden.shape, head.shape[0]
    device, bf16, f32 = _current_device(where), torch.bfloat16, torch.float32
    _operands(where, device, (hidden, bf16, (T, D)), (head, bf16, (V, D)), (labels, torch.int32, (T,)), (loss_tokens, f32, (T,)), (d_loss, f32, (T,)),
              (d_hidden, bf16, (T, D)))
    if workspace is not None and workspace.get_device() != device:
        raise ValueError(f"{where}: tensors must be on the current CUDA device, got {workspace.device}")
    rc = _native().qlora_head_loss(T, V, D, hidden, head, labels, d_loss, loss_tokens, d_hidden, workspace, workspace_bytes, stream)
    if rc != 0:
        raise QloraError(rc, where)


def qlora_gather_columns(inp, perm, out, stream=None):
    """out[m, j] = inp[m, perm[j]] for 2-D bf16 / fp16 / fp32 tensors; perm int32 [cols]."""
    rows, cols = inp.shape
    rc = _native().qlora_gather_columns(inp.element_size(), rows, cols, inp, perm, out, stream)
    if rc != 0:
        raise QloraError(rc, "qlora_gather_columns")


def qlora_dequant(d, Q, scales, zeros, W, stream=None):
    _check(library().qlora_dequant(ctypes.byref(d), _ptr(Q), _ptr(scales), _ptr(zeros), _ptr(W), _stream(stream)),
           "qlora_dequant")


def qlora_quantize_rtn(d, W, Q, scales, zeros, stream=None):
    """Min-max round-to-nearest quantization of W fp32 [N, K] into packed Q, fp16 scales and zeros [K/g, N]."""
    rc = _native().qlora_quantize_rtn(d, W, Q, scales, zeros, stream)
    if rc != 0:
        raise QloraError(rc, "qlora_quantize_rtn")


def qlora_selftest_bounded_wait(limit_us: int, stream=None):
    """Enqueue a wait that is known to run out after limit_us microseconds (sets the device's sticky status word)."""
    _check(library().qlora_selftest_bounded_wait(int(limit_us), _stream(stream)), "qlora_selftest_bounded_wait")


def qlora_device_status(clear: bool = True) -> int:
    """Synchronise the device and return its sticky health word (0 = healthy).  Raises QloraError on a recorded timeout."""
    out = ctypes.c_uint(0)
    rc = library().qlora_device_status(ctypes.byref(out), 1 if clear else 0)
    if rc != 0:
        raise QloraError(rc, f"qlora_device_status (word {out.value:#x})")
    return int(out.value)
