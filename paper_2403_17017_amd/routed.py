"""Binding of the routed layer and its training step: choices sorted by expert, rows brought to the
experts and back with their gradients, products of 8-bit integers, the norm over many gradients.

The same manner as the calls on sparse matrices (binding.py): argument marshalling only, the work is the
library's.  Outputs may be handed in or are allocated here (on the call's stream); a matrix is a 2-D tensor
whose rows are contiguous.  A call's tensors are all on the current GPU (ValueError).
No call keeps a history: a tensor that requires grad is refused while torch records one (RuntimeError); the gradients are calls
of their own, for the backward of a torch.autograd.Function, say.
"""
from __future__ import annotations

import ctypes as C

from . import binding as B
from .binding import SeerError, _stream_handle

MAX_EXPERTS = 4096
EINVAL, EWORKSPACE, ELIMIT = -1, -4, -6
I8_MAX_K = 131071


class seer_dense(C.Structure):
    _fields_ = [("data", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("ld", C.c_int64), ("type", C.c_int32)]


class seer_routing(C.Structure):
    _fields_ = [("tokens", C.c_int32), ("choices", C.c_int32), ("experts", C.c_int32),
                ("expert_ptr", C.c_void_p), ("slot_choice", C.c_void_p), ("choice_slot", C.c_void_p)]


class seer_grad(C.Structure):
    _fields_ = [("grad", C.c_void_p), ("out", C.c_void_p), ("n", C.c_int64), ("type", C.c_int32)]


_types = None       # torch's dtypes, the number of each as the library has it
_torch = None


def _ready():
    """The library and the native marshalling of its calls, loaded; torch is imported here."""
    global _types, _torch
    if _types is None:
        B.lib()
        import torch
        ids = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2, torch.int8: 3, torch.int32: 4, torch.int64: 5}
        L, m = B.lib(), B._marshal
        m.bind_routed(*(C.cast(f, C.c_void_p).value for f in (
            L.seer_route, L.seer_route_gather, L.seer_route_combine, L.seer_route_grad, L.seer_i8_quantize, L.seer_route_gather_i8,
            L.seer_i8_product, L.seer_grad_norm, L.seer_grad_clip)), torch._C, torch.cuda, torch.is_grad_enabled, *ids)
        m.bind_tokens(*(C.cast(f, C.c_void_p).value for f in (L.seer_route_choose, L.seer_route_choose_grad, L.seer_embed, L.seer_embed_grad)))
        m.bind_mx4(*(C.cast(f, C.c_void_p).value for f in (L.seer_mx4_quantize, L.seer_route_gather_mx4, L.seer_mx4_product)), torch.uint8)
        _types, _torch = ids, torch
    return B._marshal


def _handle(stream) -> int:
    """As _stream_handle; a torch stream is one of the current GPU's."""
    if stream is not None and hasattr(stream, "cuda_stream") and stream.device_index != _torch._C._cuda_getDevice():
        raise ValueError(f"the stream is GPU {stream.device_index}'s and the current one is {_torch._C._cuda_getDevice()}")
    return _stream_handle(stream)


def bind(L):
    """Argument types of the library's functions (called when the library is loaded)."""
    vp, sz, i32, i64 = C.c_void_p, C.c_size_t, C.c_int32, C.c_int64
    dense, routing = C.POINTER(seer_dense), C.POINTER(seer_routing)
    for name, args, res in (
            ("seer_route", [vp, i32, routing, vp, sz, vp], C.c_int),
            ("seer_route_workspace_bytes", [i32, i32, i32], sz),
            ("seer_route_gather", [routing, dense, vp, dense, vp], C.c_int),
            ("seer_route_combine", [routing, dense, vp, dense, vp], C.c_int),
            ("seer_route_grad", [routing, dense, dense, vp, dense, vp, vp], C.c_int),
            ("seer_i8_quantize", [dense, dense, vp, vp], C.c_int),
            ("seer_route_gather_i8", [routing, dense, dense, vp, vp], C.c_int),
            ("seer_i8_product", [dense, vp, dense, vp, vp, i32, dense, vp, sz, vp], C.c_int),
            ("seer_i8_product_workspace_bytes", [i64, i64, i64, i32], sz),
            ("seer_i8_product_kernel", [dense, dense, vp, i32], C.c_int),
            ("seer_grad_norm", [C.POINTER(seer_grad), i32, vp, vp, sz, vp], C.c_int),
            ("seer_grad_clip", [C.POINTER(seer_grad), i32, C.c_float, vp, vp, sz, vp], C.c_int),
            ("seer_grad_workspace_bytes", [], sz)):
        f = getattr(L, name)
        f.argtypes, f.restype = args, res


def _new(shape, dtype, like, stream):
    """Memory for an output or a workspace that `stream` is going to write."""
    if stream is None:
        return _torch.empty(*shape, dtype=dtype, device=like.device)     # (sizes one by one: 0.3 us less)
    if not hasattr(stream, "cuda_stream"):
        raise ValueError("pass every output and workspace when stream is a raw handle: the allocator does not know it")
    with _torch.cuda.stream(stream):
        return _torch.empty(*shape, dtype=dtype, device=like.device)


def _matrix_shape(t, what):
    if t.dim() != 2:
        raise ValueError(f"{what} is to be a matrix with contiguous rows")
    return t.shape


class Routing:
    """The order of tokens' choices by expert (seer_routing): int32 tensors expert_ptr [experts + 1],
    slot_choice [tokens * choices] and choice_slot [tokens, choices] on the GPU."""

    __slots__ = ("experts", "tokens", "choices", "expert_ptr", "slot_choice", "choice_slot")

    def __init__(self, experts: int, expert_ptr, slot_choice, choice_slot):
        _ready()
        self.experts = int(experts)
        self.tokens, self.choices = choice_slot.shape
        self.expert_ptr, self.slot_choice, self.choice_slot = expert_ptr, slot_choice, choice_slot
        for t, n in ((expert_ptr, self.experts + 1), (slot_choice, self.tokens * self.choices), (choice_slot, self.tokens * self.choices)):
            if t.dtype != _torch.int32 or not t.is_cuda or not t.is_contiguous() or t.numel() != n:
                raise ValueError("a routing has contiguous int32 tensors of experts + 1, tokens * choices and as many elements on the GPU")

    @classmethod
    def empty(cls, tokens: int, choices: int, experts: int, device="cuda:0") -> "Routing":
        """Memory for seer_route to fill."""
        _ready()
        n = lambda *shape: _torch.empty(shape, dtype=_torch.int32, device=device)
        return cls(experts, n(experts + 1), n(tokens * choices), n(tokens, choices))

    @classmethod
    def _new(cls, tokens, choices, experts, like, stream, workspace_bytes):
        """(a routing, a workspace for seer_route or None), in one piece of memory."""
        self, count = cls.__new__(cls), tokens * choices
        self.experts, self.tokens, self.choices = experts, tokens, choices
        words, sizes = workspace_bytes // 4, (experts + 1, count, count)
        memory, workspace = _new((words + experts + 1 + 2 * count,), _torch.int32, like, stream), None
        if words:
            workspace, self.expert_ptr, self.slot_choice, slots = memory.split_with_sizes((words, *sizes))
            workspace = workspace.view(_torch.uint8)
        else:
            self.expert_ptr, self.slot_choice, slots = memory.split_with_sizes(sizes)
        self.choice_slot = slots.view(tokens, choices)
        return self, workspace


def route_workspace_bytes(tokens: int, choices: int, experts: int) -> int:
    return int(B.lib().seer_route_workspace_bytes(tokens, choices, experts))


def seer_route(expert, experts: int, routing: Routing = None, workspace=None, stream=None) -> Routing:
    """The choices expert [tokens, choices] (int32 or int64; anything outside [0, experts) is no expert's) sorted by
    expert; asynchronous on the stream."""
    m = _ready()
    if expert.dim() != 2 or not expert.is_cuda or expert.dtype not in (_torch.int32, _torch.int64):
        raise ValueError("expert is to be a contiguous int32 or int64 matrix [tokens, choices] on the GPU")
    tokens, choices = expert.shape
    if not 0 < experts <= MAX_EXPERTS:
        raise SeerError(ELIMIT if experts > 0 else EINVAL, "seer_route")
    if routing is None:
        # (asking costs as much as the call, and up to 2048 choices need none)
        need = route_workspace_bytes(tokens, choices, experts) if workspace is None and tokens * choices > 2048 else 0
        routing, room = Routing._new(tokens, choices, int(experts), expert, stream, need)
        workspace = room if workspace is None else workspace
    elif (routing.tokens, routing.choices, routing.experts) != (tokens, choices, experts):
        raise ValueError("routing has other sizes")
    h = _handle(stream)
    rc = m.route(expert, routing, workspace, h)
    if rc == EWORKSPACE and workspace is None:
        workspace = _new((route_workspace_bytes(tokens, choices, experts),), _torch.uint8, expert, stream)
        rc = m.route(expert, routing, workspace, h)
    if rc:
        raise SeerError(rc, "seer_route")
    return routing


def seer_route_gather(r: Routing, x, out=None, weight=None, stream=None):
    """x [tokens, n] brought into the experts' order, out [tokens * choices, n], rows times weight if given."""
    m = _ready()
    if out is None:
        out = _new((r.tokens * r.choices, _matrix_shape(x, "x")[1]), x.dtype, x, stream)
    rc = m.gather(r, x, out, weight, _handle(stream))
    if rc:
        raise SeerError(rc, "seer_route_gather")
    return out


def seer_route_combine(r: Routing, z, y=None, weight=None, stream=None):
    """The experts' rows z [tokens * choices, n] added up by token, times weight if given: y [tokens, n]."""
    m = _ready()
    if y is None:
        y = _new((r.tokens, _matrix_shape(z, "z")[1]), z.dtype, z, stream)
    rc = m.combine(r, z, y, weight, _handle(stream))
    if rc:
        raise SeerError(rc, "seer_route_combine")
    return y


def seer_route_grad(r: Routing, dy, z, weight=None, dz=None, dweight=None, stream=None, need_dz=True, need_dweight=True):
    """(dz, dweight): the gradients of seer_route_combine in z and weight for that of its output, dy."""
    m = _ready()
    if dz is None and need_dz:
        dz = _new((r.tokens * r.choices, _matrix_shape(dy, "dy")[1]), dy.dtype, dy, stream)
    if dweight is None and need_dweight:
        dweight = _new((r.tokens, r.choices), _torch.float32, dy, stream)
    rc = m.grad(r, dy, z, weight, dz, dweight, _handle(stream))
    if rc:
        raise SeerError(rc, "seer_route_grad")
    return dz, dweight


def _new_i8(rows, cols, like, stream):
    """int8 rows at distances of a multiple of 16, which is what products read fastest."""
    if cols % 16 == 0:
        return _new((rows, cols), _torch.int8, like, stream)
    return _new((rows, (cols + 15) // 16 * 16), _torch.int8, like, stream)[:, :cols]


def _room_for_pieces(q, cols):
    """The columns up to the next multiple of 16 are written where rows are further apart: in the last row, too."""
    rows, ld = q.shape[0], q.stride(0) if q.dim() == 2 else 0
    if rows and ld > cols and q.storage_offset() + (rows - 1) * ld + min(ld, (cols + 15) // 16 * 16) > q.untyped_storage().nbytes():
        raise ValueError("the memory of q ends within the last row's columns up to the next multiple of 16")


def seer_i8_quantize(x, q=None, scale=None, stream=None):
    """(q, scale): the rows of x in 8-bit integers with a scale each."""
    m = _ready()
    rows, cols = _matrix_shape(x, "x")
    if q is None:
        q = _new_i8(rows, cols, x, stream)
    elif cols % 16:
        _room_for_pieces(q, cols)
    if scale is None:
        scale = _new((rows,), _torch.float32, x, stream)
    rc = m.quantize(None, x, q, scale, _handle(stream))
    if rc:
        raise SeerError(rc, "seer_i8_quantize")
    return q, scale


def seer_route_gather_i8(r: Routing, x, q=None, scale=None, stream=None):
    """(q, scale): x [tokens, n] in 8-bit integers, brought into the experts' order."""
    m = _ready()
    rows = r.tokens * r.choices
    cols = _matrix_shape(x, "x")[1]
    if q is None:
        q = _new_i8(rows, cols, x, stream)
    elif cols % 16:
        _room_for_pieces(q, cols)
    if scale is None:
        scale = _new((rows,), _torch.float32, x, stream)
    rc = m.quantize(r, x, q, scale, _handle(stream))
    if rc:
        raise SeerError(rc, "seer_route_gather_i8")
    return q, scale


def i8_product_workspace_bytes(rows: int, channels: int, columns: int, groups: int = 1) -> int:
    return int(B.lib().seer_i8_product_workspace_bytes(rows, channels, columns, groups))


I8_KERNELS = ("none", "any", "few", "tiles", "shared")


def i8_product_kernel(a, b, group_ptr=None) -> str:
    """Which kernel seer_i8_product takes for these operands, one of I8_KERNELS; nothing is launched."""
    if b.dim() not in (2, 3):
        raise ValueError("b is to be [groups, channels, columns]")
    groups = b.shape[0] if b.dim() == 3 else 1
    dense = lambda t, rows: C.byref(seer_dense(t.data_ptr(), rows, t.shape[-1], max(t.stride(-2) if rows > 1 else 0, t.shape[-1]), 3))
    rc = B.lib().seer_i8_product_kernel(dense(a, a.shape[0]), dense(b, groups * b.shape[-2]),
                                        group_ptr.data_ptr() if group_ptr is not None else None, groups)
    if rc < 0:
        raise SeerError(rc, "seer_i8_product_kernel")
    return I8_KERNELS[rc]


def seer_i8_product(a, a_scale, b, b_scale, out=None, group_ptr=None, dtype=None, workspace=None, stream=None):
    """out[i, n] = a_scale[i] * b_scale[g, n] * sum_k a[i, k] * b[g, n, k] for the rows i of group g (group_ptr, int32
    [groups + 1]; None: one group).  a int8 [rows, k], b int8 [groups, channels, k] or, for one group, [channels, k];
    out of type dtype (bfloat16 if neither is given)."""
    m = _ready()
    if a_scale is None or b_scale is None:
        raise ValueError("a_scale and b_scale are wanted")
    shape = b.shape
    if len(shape) not in (2, 3):
        raise ValueError("b is to be [groups, channels, columns]")
    groups, channels, columns = shape if len(shape) == 3 else (1, *shape)
    rows = _matrix_shape(a, "a")[0]
    if b.dtype != _torch.int8:
        raise ValueError("b is to be an int8 tensor")
    if out is None:
        out = _new((rows, channels), dtype or _torch.bfloat16, a, stream)
    elif dtype is not None and out.dtype != dtype:
        raise TypeError(f"out is {out.dtype}, not {dtype}")
    h = _handle(stream)
    rc = m.product(a, a_scale, b, b_scale, group_ptr, out, workspace, h)
    if rc == EWORKSPACE and workspace is None:
        workspace = _new((i8_product_workspace_bytes(rows, channels, columns, groups),), _torch.uint8, a, stream)
        rc = m.product(a, a_scale, b, b_scale, group_ptr, out, workspace, h)
    if rc:
        raise SeerError(rc, "seer_i8_product")
    return out


def grad_workspace_bytes() -> int:
    return int(B.lib().seer_grad_workspace_bytes())


class GradTensors:
    """Many gradient tensors as the library sees them: where each lies and, with `outs`, where its clipped form goes
    (else it is clipped in place).  Keeps the tensors; made once for gradients that stay where they are."""

    def __init__(self, grads, outs=None):
        m = _ready()
        self.grads, self.outs = list(grads), list(outs) if outs is not None else None
        self.count = len(self.grads)
        if self.outs is not None and len(self.outs) != self.count:
            raise ValueError("as many outputs as gradients are wanted")
        self.c = (seer_grad * max(self.count, 1))()
        self.gpu = m.grads(self.grads, self.outs, C.addressof(self.c), self.count)      # that they are on; -1: there are none


def _grad_call(what, tensors, max_norm, norm, workspace, stream):
    m = _ready()
    if not isinstance(tensors, GradTensors):
        tensors = GradTensors(tensors)
    if norm is None:
        if not tensors.count:
            raise ValueError("pass norm= where there are no tensors: nothing says which GPU it is to lie on")
        norm = _new((1,), _torch.float32, tensors.grads[0], stream).view(())
    if workspace is None:
        workspace = _new((grad_workspace_bytes(),), _torch.uint8, norm, stream)
    rc = m.clip(C.addressof(tensors.c), tensors.count, max_norm, norm, workspace, _handle(stream), tensors.gpu)
    if rc:
        raise SeerError(rc, what)
    return norm


def seer_grad_norm(tensors, norm=None, workspace=None, stream=None):
    """The norm over all gradients (a GradTensors, or a list of tensors), as a tensor of one fp32 element."""
    return _grad_call("seer_grad_norm", tensors, None, norm, workspace, stream)


def seer_grad_clip(tensors, max_norm: float, norm=None, workspace=None, stream=None):
    """Clips the gradients by their norm, which is returned: each becomes itself times max_norm / (norm + 1e-6) where that
    is less than 1, in place or in the GradTensors' outputs."""
    return _grad_call("seer_grad_clip", tensors, float(max_norm), norm, workspace, stream)
