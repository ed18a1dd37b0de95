"""Binding of the routed layer and its training step: choices sorted by expert, rows brought to the
experts and back with their gradients, products of 8-bit integers, the norm over many gradients.

The same manner as the calls on sparse matrices (binding.py): argument marshalling only, the work is the
library's.  Outputs may be handed in or are allocated here (on the call's stream); a matrix is a 2-D tensor
whose rows are contiguous.
"""
from __future__ import annotations

import ctypes as C

from . import binding as B
from .binding import SeerError, _stream_handle

MAX_EXPERTS = 4096
I8_MAX_K = 131071


class seer_dense(C.Structure):
    _fields_ = [("data", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("ld", C.c_int64), ("type", C.c_int32)]


class seer_routing(C.Structure):
    _fields_ = [("tokens", C.c_int32), ("choices", C.c_int32), ("experts", C.c_int32),
                ("expert_ptr", C.c_void_p), ("slot_choice", C.c_void_p), ("choice_slot", C.c_void_p)]


class seer_grad(C.Structure):
    _fields_ = [("grad", C.c_void_p), ("out", C.c_void_p), ("n", C.c_int64), ("type", C.c_int32)]


_types = None


def _type_ids():
    global _types
    if _types is None:
        import torch
        _types = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2, torch.int8: 3, torch.int32: 4, torch.int64: 5}
    return _types


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
            ("seer_grad_norm", [C.POINTER(seer_grad), i32, vp, vp, sz, vp], C.c_int),
            ("seer_grad_clip", [C.POINTER(seer_grad), i32, C.c_float, vp, vp, sz, vp], C.c_int),
            ("seer_grad_workspace_bytes", [], sz)):
        f = getattr(L, name)
        f.argtypes, f.restype = args, res


def _new(shape, dtype, like, stream):
    """Memory for an output or a workspace that `stream` is going to write."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    if not hasattr(stream, "cuda_stream"):
        raise ValueError("pass every output and workspace when stream is a raw handle: the allocator does not know it")
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=like.device)


def _dense(t, what):
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1 and t.shape[0] > 0):
        raise ValueError(f"{what} is to be a matrix with contiguous rows")
    if not t.is_cuda:
        raise ValueError(f"{what} is not on a GPU")
    type_id = _type_ids().get(t.dtype)
    if type_id is None:
        raise TypeError(f"{what} is {t.dtype}")
    rows, cols = t.shape
    return seer_dense(t.data_ptr(), rows, cols, t.stride(0) if rows > 1 else max(cols, t.stride(0)), type_id)


def _vector(t, what, dtype, n):
    """The address of a contiguous tensor of n elements (None: null)."""
    if t is None:
        return None
    if t.dtype != dtype or not t.is_contiguous() or not t.is_cuda or t.numel() != n:
        raise ValueError(f"{what} is to be a contiguous {dtype} tensor of {n} elements on the GPU")
    return t.data_ptr()


def _check(rc, what):
    if rc:
        raise SeerError(rc, what)


class Routing:
    """The order of tokens' choices by expert (seer_routing): int32 tensors expert_ptr [experts + 1],
    slot_choice [tokens * choices] and choice_slot [tokens, choices] on the GPU."""

    __slots__ = ("experts", "tokens", "choices", "expert_ptr", "slot_choice", "choice_slot")

    def __init__(self, experts: int, expert_ptr, slot_choice, choice_slot):
        import torch
        self.experts = int(experts)
        self.tokens, self.choices = choice_slot.shape
        self.expert_ptr, self.slot_choice, self.choice_slot = expert_ptr, slot_choice, choice_slot
        _vector(expert_ptr, "expert_ptr", torch.int32, self.experts + 1)
        _vector(slot_choice, "slot_choice", torch.int32, self.tokens * self.choices)
        _vector(choice_slot, "choice_slot", torch.int32, self.tokens * self.choices)

    @classmethod
    def empty(cls, tokens: int, choices: int, experts: int, device="cuda:0") -> "Routing":
        """Memory for seer_route to fill."""
        import torch
        n = lambda *shape: torch.empty(shape, dtype=torch.int32, device=device)
        return cls(experts, n(experts + 1), n(tokens * choices), n(tokens, choices))

    def c_struct(self) -> seer_routing:
        return seer_routing(self.tokens, self.choices, self.experts, self.expert_ptr.data_ptr(), self.slot_choice.data_ptr(),
                            self.choice_slot.data_ptr())


def route_workspace_bytes(tokens: int, choices: int, experts: int) -> int:
    return int(B.lib().seer_route_workspace_bytes(tokens, choices, experts))


def seer_route(expert, experts: int, routing: Routing = None, workspace=None, stream=None) -> Routing:
    """The choices expert [tokens, choices] (int32 or int64; anything outside [0, experts) is no expert's) sorted by
    expert; asynchronous on the stream."""
    import torch
    L = B.lib()
    if expert.dim() != 2 or not expert.is_contiguous() or not expert.is_cuda or expert.dtype not in (torch.int32, torch.int64):
        raise ValueError("expert is to be a contiguous int32 or int64 matrix [tokens, choices] on the GPU")
    tokens, choices = expert.shape
    if routing is None:
        n = max(int(experts), 0)
        routing = Routing(n, _new((n + 1,), torch.int32, expert, stream), _new((tokens * choices,), torch.int32, expert, stream),
                          _new((tokens, choices), torch.int32, expert, stream))
    elif (routing.tokens, routing.choices, routing.experts) != (tokens, choices, experts):
        raise ValueError("routing has other sizes")
    need = L.seer_route_workspace_bytes(tokens, choices, experts)
    if need and workspace is None:
        workspace = _new((need,), torch.uint8, expert, stream)
    _check(L.seer_route(expert.data_ptr(), _type_ids()[expert.dtype], C.byref(routing.c_struct()),
                        workspace.data_ptr() if workspace is not None else None,
                        workspace.numel() if workspace is not None else 0, _stream_handle(stream)), "seer_route")
    return routing


def _weight(weight, r):
    import torch
    return _vector(weight, "weight", torch.float32, r.tokens * r.choices)


def seer_route_gather(r: Routing, x, out=None, weight=None, stream=None):
    """x [tokens, n] brought into the experts' order, out [tokens * choices, n], rows times weight if given."""
    if out is None:
        out = _new((r.tokens * r.choices, x.shape[1]), x.dtype, x, stream)
    _check(B.lib().seer_route_gather(C.byref(r.c_struct()), C.byref(_dense(x, "x")), _weight(weight, r), C.byref(_dense(out, "out")),
                                     _stream_handle(stream)), "seer_route_gather")
    return out


def seer_route_combine(r: Routing, z, y=None, weight=None, stream=None):
    """The experts' rows z [tokens * choices, n] added up by token, times weight if given: y [tokens, n]."""
    if y is None:
        y = _new((r.tokens, z.shape[1]), z.dtype, z, stream)
    _check(B.lib().seer_route_combine(C.byref(r.c_struct()), C.byref(_dense(z, "z")), _weight(weight, r), C.byref(_dense(y, "y")),
                                      _stream_handle(stream)), "seer_route_combine")
    return y


def seer_route_grad(r: Routing, dy, z, weight=None, dz=None, dweight=None, stream=None, need_dz=True, need_dweight=True):
    """(dz, dweight): the gradients of seer_route_combine in z and weight for that of its output, dy."""
    import torch
    if dz is None and need_dz:
        dz = _new((r.tokens * r.choices, dy.shape[1]), dy.dtype, dy, stream)
    if dweight is None and need_dweight:
        dweight = _new((r.tokens, r.choices), torch.float32, dy, stream)
    _check(B.lib().seer_route_grad(C.byref(r.c_struct()), C.byref(_dense(dy, "dy")), C.byref(_dense(z, "z")) if z is not None else None,
                                   _weight(weight, r), C.byref(_dense(dz, "dz")) if dz is not None else None,
                                   _vector(dweight, "dweight", torch.float32, r.tokens * r.choices), _stream_handle(stream)),
           "seer_route_grad")
    return dz, dweight


def _new_i8(rows, cols, like, stream):
    """int8 rows at distances of a multiple of 16, which is what products read fastest."""
    import torch
    return _new((rows, (cols + 15) // 16 * 16), torch.int8, like, stream)[:, :cols]


def seer_i8_quantize(x, q=None, scale=None, stream=None):
    """(q, scale): the rows of x in 8-bit integers with a scale each."""
    import torch
    if q is None:
        q = _new_i8(x.shape[0], x.shape[1], x, stream)
    if scale is None:
        scale = _new((x.shape[0],), torch.float32, x, stream)
    _check(B.lib().seer_i8_quantize(C.byref(_dense(x, "x")), C.byref(_dense(q, "q")),
                                    _vector(scale, "scale", torch.float32, x.shape[0]), _stream_handle(stream)), "seer_i8_quantize")
    return q, scale


def seer_route_gather_i8(r: Routing, x, q=None, scale=None, stream=None):
    """(q, scale): x [tokens, n] in 8-bit integers, brought into the experts' order."""
    import torch
    rows = r.tokens * r.choices
    if q is None:
        q = _new_i8(rows, x.shape[1], x, stream)
    if scale is None:
        scale = _new((rows,), torch.float32, x, stream)
    _check(B.lib().seer_route_gather_i8(C.byref(r.c_struct()), C.byref(_dense(x, "x")), C.byref(_dense(q, "q")),
                                        _vector(scale, "scale", torch.float32, rows), _stream_handle(stream)), "seer_route_gather_i8")
    return q, scale


def i8_product_workspace_bytes(rows: int, channels: int, columns: int, groups: int = 1) -> int:
    return int(B.lib().seer_i8_product_workspace_bytes(rows, channels, columns, groups))


def seer_i8_product(a, a_scale, b, b_scale, out=None, group_ptr=None, dtype=None, workspace=None, stream=None):
    """out[i, n] = a_scale[i] * b_scale[g, n] * sum_k a[i, k] * b[g, n, k] for the rows i of group g (group_ptr, int32
    [groups + 1]; None: one group).  a int8 [rows, k], b int8 [groups, channels, k] or, for one group, [channels, k];
    out of type dtype (bfloat16 if neither is given)."""
    import torch
    L = B.lib()
    if b.dim() == 2:
        b = b.unsqueeze(0)
    if b.dim() != 3:
        raise ValueError("b is to be [groups, channels, columns]")
    groups, channels, columns = b.shape
    if groups > 1 and channels > 1 and b.stride(0) != channels * b.stride(1):
        raise ValueError("the matrices of b are to lie one behind the other")
    if out is None:
        out = _new((a.shape[0], channels), dtype or torch.bfloat16, a, stream)
    elif dtype is not None and out.dtype != dtype:
        raise TypeError(f"out is {out.dtype}, not {dtype}")
    need = L.seer_i8_product_workspace_bytes(a.shape[0], channels, columns, groups)
    if need and workspace is None:
        workspace = _new((need,), torch.uint8, a, stream)
    if not b.is_cuda or b.dtype != torch.int8 or (columns > 1 and b.stride(2) != 1):
        raise ValueError("b is to be an int8 tensor on the GPU with contiguous rows")
    ld = b.stride(1) if channels > 1 else b.stride(0) if groups > 1 else columns
    _check(L.seer_i8_product(C.byref(_dense(a, "a")), _vector(a_scale, "a_scale", torch.float32, a.shape[0]),
                             C.byref(seer_dense(b.data_ptr(), groups * channels, columns, ld, 3)),
                             _vector(b_scale, "b_scale", torch.float32, groups * channels),
                             _vector(group_ptr, "group_ptr", torch.int32, groups + 1), groups, C.byref(_dense(out, "out")),
                             workspace.data_ptr() if workspace is not None else None,
                             workspace.numel() if workspace is not None else 0, _stream_handle(stream)), "seer_i8_product")
    return out


def grad_workspace_bytes() -> int:
    return int(B.lib().seer_grad_workspace_bytes())


class GradTensors:
    """Many gradient tensors as the library sees them: where each lies and, with `outs`, where its clipped form goes
    (else it is clipped in place).  Keeps the tensors; made once for gradients that stay where they are."""

    def __init__(self, grads, outs=None):
        ids = _type_ids()
        self.grads, self.outs = list(grads), list(outs) if outs is not None else None
        to = self.outs if self.outs is not None else self.grads
        if len(to) != len(self.grads):
            raise ValueError("as many outputs as gradients are wanted")
        self.count = len(self.grads)
        self.c = (seer_grad * max(self.count, 1))()
        for i, (g, o) in enumerate(zip(self.grads, to)):
            if not g.is_cuda or not o.is_cuda or not g.is_contiguous() or not o.is_contiguous():
                raise ValueError("gradients and outputs are to be contiguous and on the GPU")
            if g.dtype != o.dtype or g.numel() != o.numel():
                raise ValueError("an output is to have its gradient's type and size")
            if ids.get(g.dtype, 9) > 2:
                raise TypeError(f"a gradient is {g.dtype}")
            self.c[i] = seer_grad(g.data_ptr(), o.data_ptr(), g.numel(), ids[g.dtype])


def _grad_call(tensors, norm, workspace, stream):
    import torch
    if not isinstance(tensors, GradTensors):
        tensors = GradTensors(tensors)
    if norm is None:
        if not tensors.count:
            raise ValueError("pass norm= where there are no tensors: nothing says which GPU it is to lie on")
        norm = _new((), torch.float32, tensors.grads[0], stream)
    if workspace is None:
        workspace = _new((grad_workspace_bytes(),), torch.uint8, norm, stream)
    return tensors, norm, workspace


def seer_grad_norm(tensors, norm=None, workspace=None, stream=None):
    """The norm over all gradients (a GradTensors, or a list of tensors), as a tensor of one fp32 element."""
    import torch
    tensors, norm, workspace = _grad_call(tensors, norm, workspace, stream)
    _check(B.lib().seer_grad_norm(tensors.c, tensors.count, _vector(norm, "norm", torch.float32, 1), workspace.data_ptr(),
                                  workspace.numel(), _stream_handle(stream)), "seer_grad_norm")
    return norm


def seer_grad_clip(tensors, max_norm: float, norm=None, workspace=None, stream=None):
    """Clips the gradients by their norm, which is returned: each becomes itself times max_norm / (norm + 1e-6) where that
    is less than 1, in place or in the GradTensors' outputs."""
    import torch
    tensors, norm, workspace = _grad_call(tensors, norm, workspace, stream)
    _check(B.lib().seer_grad_clip(tensors.c, tensors.count, float(max_norm), _vector(norm, "norm", torch.float32, 1),
                                  workspace.data_ptr(), workspace.numel(), _stream_handle(stream)), "seer_grad_clip")
    return norm
