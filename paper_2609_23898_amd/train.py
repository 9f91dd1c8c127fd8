"""Python binding of the training step around the all-reduce
(include/cerar_train.h): block-scaled 8-bit matrices and their products, the
gradient norm, and the AdamW step.  Argument marshalling only, as in
``cerar``: every call checks its tensors and enqueues the library's HIP
kernels on `stream` (default: torch's current stream).
"""

import ctypes
import functools
import math

from . import cerar as C
from .cerar import CerarError  # noqa: F401  (the errors these calls raise)

_P, _SZ, _I, _F, _D = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_float, ctypes.c_double
_U64 = ctypes.c_uint64

BLOCK = 128
F32, BF16 = 0, 1


class TensorDesc(ctypes.Structure):
    """cerar_tensor"""
    _fields_ = [("n", _SZ), ("grad", _P), ("param", _P), ("m", _P), ("v", _P), ("m_scale", _P), ("v_scale", _P),
                ("copy", _P), ("grad_type", _I), ("param_type", _I), ("lr_scale", _F), ("weight_decay", _F)]


class AdamWDesc(ctypes.Structure):
    """cerar_adamw"""
    _fields_ = [("lr", _D), ("beta1", _D), ("beta2", _D), ("eps", _D), ("grad_scale", _D), ("step", _U64), ("seed", _U64)]


class AdamWValues(ctypes.Structure):
    """cerar_adamw_values"""
    _fields_ = [("beta1", _D), ("rest1", _D), ("beta2", _D), ("rest2", _D), ("key", _U64), ("lr", _F), ("eps", _F),
                ("grad_scale", _F), ("step_size", _F), ("root2", _F), ("unused", _F)]


class BlocksDesc(ctypes.Structure):
    """cerar_blocks"""
    _fields_ = [("codes", _P), ("scales", _P), ("rows", _SZ), ("cols", _SZ), ("format", _I)]


_BP = ctypes.POINTER(BlocksDesc)

# name -> (restype, argtypes); mirrors include/cerar_train.h
SIGNATURES = {
    "cerar_tensors_create": (_I, [_I, ctypes.POINTER(TensorDesc), _I, ctypes.POINTER(_P)]),
    "cerar_tensors_destroy": (None, [_P]),
    "cerar_grad_norm": (_I, [_P, _F, _F, _P, _P]),
    "cerar_adamw_pack": (_I, [ctypes.POINTER(AdamWDesc), ctypes.POINTER(AdamWValues)]),
    "cerar_adamw_step": (_I, [_P, ctypes.POINTER(AdamWDesc), _P, _P, _P]),
    "cerar_quantize_blocks": (_I, [_P, _I, _SZ, _SZ, _SZ, _I, _BP, _BP, _P]),
    "cerar_matmul_workspace_bytes": (_I, [_SZ, _SZ, _SZ, _I, ctypes.POINTER(_SZ)]),
    "cerar_matmul_blocks": (_I, [_BP, _BP, _P, _I, _SZ, _I, _I, _P, _P]),
    "cerar_linear_blocks": (_I, [_P, _I, _SZ, _SZ, _BP, _P, _I, _SZ, _I, _P, _P]),
}

_lib = None


def lib():
    """The loaded libcerar.so with these calls declared (raises if it was not built)."""
    global _lib
    handle = C.lib()
    if _lib is not handle:
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


_raw = None


def _queue(stream, current):
    """The HIP stream to enqueue on: `stream`, else torch's current one on the device
    `current`, which the caller has looked up (C._stream looks it up again: 0.5 us)."""
    global _raw
    if stream is not None:
        return stream.cuda_stream
    if _raw is None:
        import torch
        _raw = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda _: C._stream(None))
    return _raw(current)


_bump = None


def _written(tensors):
    """Counts a write to each of a list of tensors, as torch's own in-place operations do: a
    backward pass that has saved one of them then raises instead of using the new values.
    (0.15 us for one; the public call that it is behind takes 0.3.)"""
    global _bump
    if _bump is None:
        import torch
        _bump = getattr(torch._C, "_increment_version", None) or torch.autograd.graph.increment_version
    _bump(tensors)


_types = {}


def _type(t, name):
    """F32 or BF16 of a tensor's entries."""
    kind = _types.get(t.dtype)
    if kind is None:
        import torch
        _types.update({torch.float32: F32, torch.bfloat16: BF16})
        kind = _types.get(t.dtype)
    if kind is None:
        raise ValueError(f"{name} must be float32 or bfloat16, not {t.dtype}")
    return kind


# --- gradients and states of many tensors -------------------------------------------

def _flat(t, name, n=None, dtype=None):
    """t's address; it must be contiguous on the current device, of n entries of dtype."""
    C._on_device(t, name)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if n is not None and t.numel() != n:
        raise ValueError(f"{name} has {t.numel()} entries, {n} are needed")
    if dtype is not None and t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    return t.data_ptr() if t.numel() else None


def _each(value, count, name):
    """One number for each tensor, from a number or a list."""
    if isinstance(value, (int, float)):
        return [float(value)] * count
    if len(value) != count:
        raise ValueError(f"{name} has {len(value)} entries for {count} tensors")
    return [float(v) for v in value]


class _Set:
    """A cerar_tensors handle and the tensors that it holds the addresses of."""

    def _create(self, descs, bits, keep):
        self._h = _P()
        self._keep = keep
        table = (TensorDesc * len(descs))(*descs)
        C._check(lib().cerar_tensors_create(len(descs), table, bits, ctypes.byref(self._h)))

    @property
    def handle(self):
        return self._h

    def close(self):
        if getattr(self, "_h", None):
            lib().cerar_tensors_destroy(self._h)
            self._h = _P()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class GradSet(_Set):
    """Gradients (float32 or bfloat16, contiguous, on the current device) whose
    common norm is taken: cerar_tensors_create with state_bits = 0."""

    def __init__(self, grads):
        grads = list(grads)
        descs = [TensorDesc(n=g.numel(), grad=_flat(g, f"grads[{i}]"), grad_type=_type(g, f"grads[{i}]"))
                 for i, g in enumerate(grads)]
        self._create(descs, 0, grads)


class TensorSet(_Set):
    """Parameters, gradients and AdamW states that are stepped together.

    params, grads   lists of contiguous float32 or bfloat16 tensors of equal sizes.
                    The set keeps their addresses: gradients are written
                    into the same tensors at every step (rows of an
                    all-reduce's output, for example)
    state_bits      32: m and v in float32; 8: float8_e4m3fn and float8_e5m2
                    codes with one scale byte for each 128 entries
    copies          optional bfloat16 tensors that receive the stepped parameters
    lr_scale, weight_decay   a number, or one for each tensor
    states          {"m": [...], "v": [...]}, with "m_scale" and "v_scale" for
                    8 bits, to go on from (a checkpoint's); made here, zero, if
                    absent
    """

    def __init__(self, params, grads, state_bits=32, copies=None, lr_scale=1.0, weight_decay=0.0, states=None):
        import torch
        params, grads = list(params), list(grads)
        count = len(params)
        if len(grads) != count or (copies is not None and len(copies) != count):
            raise ValueError(f"{count} params, {len(grads)} grads" + ("" if copies is None else f", {len(copies)} copies"))
        if state_bits not in (8, 32):
            raise ValueError(f"state_bits={state_bits} is neither 8 nor 32")
        kinds = ({"m": torch.float32, "v": torch.float32} if state_bits == 32 else
                 {"m": torch.float8_e4m3fn, "v": torch.float8_e5m2, "m_scale": torch.uint8, "v_scale": torch.uint8})

        def length(name, n):
            return -(-n // BLOCK) if name.endswith("scale") else n

        made = states is None
        if made:
            states = {name: [torch.zeros(length(name, p.numel()), dtype=dt, device=p.device) for p in params]
                      for name, dt in kinds.items()}
        if set(states) != set(kinds) or any(len(states[name]) != count for name in kinds):
            raise ValueError(f"states must hold {sorted(kinds)}, {count} tensors each")
        lr_scale, weight_decay = _each(lr_scale, count, "lr_scale"), _each(weight_decay, count, "weight_decay")
        descs = []
        for i, (p, g) in enumerate(zip(params, grads)):
            n = p.numel()
            d = TensorDesc(n=n, param=_flat(p, f"params[{i}]"), grad=_flat(g, f"grads[{i}]", n),
                           param_type=_type(p, f"params[{i}]"), grad_type=_type(g, f"grads[{i}]"),
                           lr_scale=lr_scale[i], weight_decay=weight_decay[i])
            for name, dt in kinds.items():
                setattr(d, name, _flat(states[name][i], f"{name}[{i}]", length(name, n), dt))
            if copies is not None:
                d.copy = _flat(copies[i], f"copies[{i}]", n, torch.bfloat16)
            descs.append(d)
        self.state_bits = state_bits
        self.states = states
        # one tensor for each count of writes: the views of a tensor share its
        counted = {id(t if t._base is None else t._base): t for t in params + list(copies or [])}
        self._stepped = list(counted.values())
        self._create(descs, state_bits, (params, grads, copies, states))
        if made:
            torch.cuda.current_stream().synchronize()    # they are zero before a step on any stream


def _clip(clip):
    """The address of grad_norm's result, on the current device."""
    if _types.get(clip.dtype) != F32 or not clip.is_contiguous() or clip.numel() < 2:
        raise ValueError("clip must be a contiguous float32 tensor of 2 entries")
    return clip.data_ptr()


def grad_norm(tensors, clip, grad_scale=1.0, max_norm=math.inf, stream=None):
    """clip[0] = the norm of all gradients of a GradSet or TensorSet times
    grad_scale, clip[1] = the factor that brings it down to max_norm
    (cerar_grad_norm)."""
    current = C._on_device(clip, "clip")
    C._check(lib().cerar_grad_norm(tensors.handle, grad_scale, max_norm, _clip(clip), _queue(stream, current)))


def _settings(lr, beta1, beta2, eps, grad_scale, step, seed):
    """cerar_adamw; a negative step would wrap to a large one (a seed may)."""
    if step < 0:
        raise ValueError(f"step={step}: the first step is 1")
    return AdamWDesc(lr, beta1, beta2, eps, grad_scale, step, seed)


def adamw_values(step, lr, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, seed=0):
    """What one step reads of its settings, as a uint8 host tensor: a program
    that replays a captured step copies the next one's into the device tensor
    that it gave as `values`."""
    import torch
    values = AdamWValues()
    C._check(lib().cerar_adamw_pack(ctypes.byref(_settings(lr, beta1, beta2, eps, grad_scale, step, seed)),
                                    ctypes.byref(values)))
    return torch.frombuffer(bytearray(values), dtype=torch.uint8)


def adamw_step(tensors, step=None, lr=None, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, clip=None, seed=0,
               values=None, stream=None):
    """One AdamW step over a TensorSet (cerar_adamw_step).  `clip` is
    grad_norm's result: its factor multiplies the gradients, and a norm that is
    not finite makes the step change nothing.  `values`: a device copy of
    adamw_values, in place of step, lr and the others."""
    hyper, dev, current = None, None, None
    if values is not None:
        if step is not None or lr is not None:
            raise ValueError("values holds the step and lr: give either")
        current = C._bytes(values, "values", ctypes.sizeof(AdamWValues))
        dev = values.data_ptr()
        if dev % 8:
            raise ValueError("values must be 8-byte aligned")
    else:
        if step is None or lr is None:
            raise ValueError("step and lr are needed")
        hyper = ctypes.byref(_settings(lr, beta1, beta2, eps, grad_scale, step, seed))
    if clip is not None:
        current = C._on_device(clip, "clip", current)
        clip = _clip(clip)
    C._check(lib().cerar_adamw_step(tensors.handle, hyper, dev, clip,
                                    C._stream(stream) if current is None else _queue(stream, current)))
    _written(tensors._stepped)


# --- block-scaled 8-bit matrices --------------------------------------------------------

_FORMATS = {"e4m3": 0, "e5m2": 1}


def _up(n, m):
    return -(-n // m) * m


class Blocks:
    """A matrix (rows x cols) in the block format of cerar_train.h.

    codes    (rows, cols up to a multiple of 128), float8_e4m3fn or float8_e5m2
    scales   (groups of four blocks, rows, 4), uint8 exponents with bias 127
    """

    def __init__(self, codes, scales, cols):
        import torch
        self.rows, self.cols = codes.shape[0], cols
        self.fmt = {torch.float8_e4m3fn: "e4m3", torch.float8_e5m2: "e5m2"}.get(codes.dtype)
        if self.fmt is None:
            raise ValueError(f"codes must be float8_e4m3fn or float8_e5m2, not {codes.dtype}")
        ld = _up(cols, BLOCK)
        groups = -(-ld // (4 * BLOCK))
        if codes.dim() != 2 or codes.shape[1] != ld or not codes.is_contiguous():
            raise ValueError(f"codes must be a contiguous tensor of {ld} columns for cols={cols}")
        if (scales.dtype != torch.uint8 or tuple(scales.shape) != (groups, self.rows, 4) or not scales.is_contiguous()):
            raise ValueError(f"scales must be a contiguous uint8 tensor of shape {(groups, self.rows, 4)}")
        C._on_device(codes, "codes")
        if scales.device != codes.device:
            raise ValueError("codes and scales are on different devices")
        self.codes, self.scales = codes, scales
        self.desc = BlocksDesc(codes.data_ptr(), scales.data_ptr(), self.rows, cols, _FORMATS[self.fmt])
        self.ref = ctypes.byref(self.desc)

    @classmethod
    def empty(cls, rows, cols, fmt="e4m3", device="cuda"):
        """Memory for a matrix; quantize_blocks fills it."""
        import torch
        if fmt not in _FORMATS:
            raise ValueError(f"fmt={fmt!r} is neither 'e4m3' nor 'e5m2'")
        ld = _up(cols, BLOCK)
        dtype = torch.float8_e4m3fn if fmt == "e4m3" else torch.float8_e5m2
        return cls(torch.empty((rows, ld), dtype=dtype, device=device),
                   torch.empty((-(-ld // (4 * BLOCK)), rows, 4), dtype=torch.uint8, device=device), cols)


def _matrix(t, name, rows=None, cols=None, current=None):
    """(type, row stride) of a row-major matrix on the current device (`current` where
    the caller has looked it up)."""
    C._on_device(t, name, current)
    kind = _type(t, name)
    shape = t.shape
    if len(shape) != 2 or (shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be a 2-D row-major tensor (unit column stride)")
    if (rows is not None and shape[0] != rows) or (cols is not None and shape[1] != cols):
        raise ValueError(f"{name} has shape {tuple(shape)}; ({rows}, {cols}) is needed")
    ld = t.stride(0)
    if shape[0] <= 1 or shape[1] == 0:           # the stride of a lone row is free
        ld = max(ld, shape[1])
    return kind, ld


def _operand(b, name, current=None):
    """Checks that b is a Blocks on the current device, which it returns."""
    if not isinstance(b, Blocks):
        raise ValueError(f"{name} must be a Blocks, not {type(b).__name__}")
    return C._on_device(b.codes, name, current)


def quantize_blocks(x, rows=None, cols=None, tile=False, stream=None):
    """x (float32 or bfloat16) into the Blocks `rows` (x's shape) and `cols`
    (the transposed shape), either of which may be absent; tile: one scale for
    each 128 x 128 entries (cerar_quantize_blocks)."""
    if rows is None and cols is None:
        raise ValueError("rows or cols is needed")
    current = C._on_device(x, "x")
    kind, ld = _matrix(x, "x", current=current)
    for b, name in ((rows, "rows"), (cols, "cols")):
        if b is not None:
            _operand(b, name, current)
    C._check(lib().cerar_quantize_blocks(x.data_ptr(), kind, x.shape[0], x.shape[1], ld, int(tile),
                                         rows and rows.ref, cols and cols.ref, _queue(stream, current)))


@functools.lru_cache(maxsize=1024)
def matmul_workspace_bytes(M, N, K, linear=False):
    """Bytes of workspace of matmul_blocks, or of linear_blocks, for an M x N
    result and inner length K."""
    b = _SZ()
    C._check(lib().cerar_matmul_workspace_bytes(M, N, K, int(linear), ctypes.byref(b)))
    return b.value


def _workspace(ws, M, N, K, linear, current):
    need = matmul_workspace_bytes(M, N, K, linear)
    if need == 0:
        return None
    if ws is None:
        raise ValueError(f"ws of {need} bytes is needed (matmul_workspace_bytes)")
    C._bytes(ws, "ws", need, current)
    return ws.data_ptr()


def matmul_blocks(a, b, out, ws=None, accumulate=False, fast_sums=False, stream=None):
    """out (a.rows x b.rows, float32 or bfloat16) = a b^T, or out + a b^T
    (float32) with accumulate (cerar_matmul_blocks).  fast_sums: on the 8-bit
    matrix instructions, at twice the rate and with an error of 2e-5 or so of
    the result, for results that are rounded to bfloat16 anyway."""
    current = _operand(b, "b", _operand(a, "a"))
    kind, ld = _matrix(out, "out", a.rows, b.rows, current)
    C._check(lib().cerar_matmul_blocks(a.ref, b.ref, out.data_ptr(), kind, ld, int(accumulate), int(fast_sums),
                                       _workspace(ws, a.rows, b.rows, a.cols, False, current), _queue(stream, current)))
    _written([out])


def linear_blocks(x, w, out, ws=None, fast_sums=False, stream=None):
    """out (rows of x, w.rows) = x w^T with x quantised on the way, as
    quantize_blocks does by rows in e4m3 (cerar_linear_blocks); fast_sums as in
    matmul_blocks."""
    current = _operand(w, "w")
    M = x.shape[0]
    kind, ld = _matrix(x, "x", M, w.cols, current)
    out_kind, ld_out = _matrix(out, "out", M, w.rows, current)
    C._check(lib().cerar_linear_blocks(x.data_ptr(), kind, M, ld, w.ref, out.data_ptr(), out_kind, ld_out, int(fast_sums),
                                       _workspace(ws, M, w.rows, w.cols, True, current), _queue(stream, current)))
    _written([out])
