"""Binding of rows in 4-bit floating point with a power of two as the scale of every 32 values: quantisation and products over ragged
groups of rows.  The same manner, and the same refusals, as the routed layer's other calls (routed.py).

Codes are uint8 tensors, [rows, 16 * blocks], two values to a byte, the first in the lower half, and scales uint8 tensors [rows, blocks]
of exponents plus 127, with a block for every 32 columns begun; the values behind the last column are zeros."""
from __future__ import annotations

import ctypes as C

from . import binding as B
from . import routed as R
from .binding import SeerError

EWORKSPACE = -4


class seer_mx4(C.Structure):
    _fields_ = [("data", C.c_void_p), ("scale", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("ld", C.c_int64), ("scale_ld", C.c_int64)]


def bind(L):
    """Argument types of the library's functions (called when the library is loaded)."""
    vp, sz, i32, i64 = C.c_void_p, C.c_size_t, C.c_int32, C.c_int64
    dense, mx4, routing = C.POINTER(R.seer_dense), C.POINTER(seer_mx4), C.POINTER(R.seer_routing)
    for name, args, res in (("seer_mx4_quantize", [dense, mx4, vp], C.c_int), ("seer_route_gather_mx4", [routing, dense, mx4, vp], C.c_int),
                            ("seer_mx4_product", [mx4, mx4, vp, i32, dense, vp, sz, vp], C.c_int),
                            ("seer_mx4_product_kernel", [mx4, mx4, vp, i32], C.c_int),
                            ("seer_mx4_product_plan", [mx4, mx4, vp, i32, C.POINTER(i32), C.POINTER(i32)], C.c_int),
                            ("seer_mx4_product_workspace_bytes", [i64, i64, i64, i32], sz)):
        f = getattr(L, name)
        f.argtypes, f.restype = args, res


def _quantize(what, r, rows, x, q, scale, stream):
    m = R._ready()
    if q is None or scale is None:
        blocks = (R._matrix_shape(x, "x")[1] + 31) // 32
        if q is None:
            q = R._new((rows, 16 * blocks), R._torch.uint8, x, stream)
        if scale is None:
            scale = R._new((rows, blocks), R._torch.uint8, x, stream)
    rc = m.mx4_quantize(r, x, q, scale, R._handle(stream))
    if rc:
        raise SeerError(rc, what)
    return q, scale


def seer_mx4_quantize(x, q=None, scale=None, stream=None):
    """(q, scale): the rows of x in 4 bits."""
    return _quantize("seer_mx4_quantize", None, x.shape[0], x, q, scale, stream)


def seer_route_gather_mx4(r: R.Routing, x, q=None, scale=None, stream=None):
    """(q, scale): x [tokens, n] in 4 bits, brought into the experts' order."""
    return _quantize("seer_route_gather_mx4", r, r.tokens * r.choices, x, q, scale, stream)


def mx4_product_workspace_bytes(rows: int, channels: int, columns: int, groups: int = 1) -> int:
    return int(B.lib().seer_mx4_product_workspace_bytes(rows, channels, columns, groups))


MX4_KERNELS = ("none", "any", "few", "tiles", "shared")


def mx4_product_plan(a, b, group_ptr=None):
    """(kernel, tokens, shares) that seer_mx4_product takes for these codes: one of MX4_KERNELS, the rows of a tile (0 without tiles), and
    between how many workgroups a tile's columns are shared out; nothing is launched."""
    if b.dim() not in (2, 3):
        raise ValueError("b is to be [groups, channels, bytes]")
    groups, blocks = b.shape[0] if b.dim() == 3 else 1, a.shape[-1] // 16
    rows_of = lambda t, rows: C.byref(seer_mx4(t.data_ptr(), t.data_ptr(), rows, 32 * blocks, t.stride(-2) if rows > 1 else 16 * blocks, blocks))
    tokens, shares = C.c_int32(), C.c_int32()
    rc = B.lib().seer_mx4_product_plan(rows_of(a, a.shape[0]), rows_of(b, groups * b.shape[-2]), group_ptr.data_ptr() if group_ptr is not None else None, groups,
                                       C.byref(tokens), C.byref(shares))
    if rc < 0:
        raise SeerError(rc, "seer_mx4_product_plan")
    return MX4_KERNELS[rc], tokens.value, shares.value


def mx4_product_kernel(a, b, group_ptr=None) -> str:
    """Which kernel seer_mx4_product takes for these codes, one of MX4_KERNELS; nothing is launched."""
    return mx4_product_plan(a, b, group_ptr)[0]


def seer_mx4_product(a, a_scale, b, b_scale, out=None, group_ptr=None, dtype=None, workspace=None, stream=None):
    """out[i, n] = sum_k a[i, k] * b[g, n, k] for the rows i of group g (group_ptr, int32 [groups + 1]; None: one group), of rows in
    4 bits: a and a_scale [rows, ..], b and b_scale [groups, channels, ..] or, for one group, [channels, ..]; out of type dtype
    (bfloat16 if neither is given)."""
    m = R._ready()
    shape = b.shape
    if len(shape) not in (2, 3):
        raise ValueError("b is to be [groups, channels, bytes]")
    groups, channels = (shape[0], shape[1]) if len(shape) == 3 else (1, shape[0])
    rows = a.shape[0]
    if out is None:
        out = R._new((rows, channels), dtype or R._torch.bfloat16, a, stream)
    elif dtype is not None and out.dtype != dtype:
        raise TypeError(f"out is {out.dtype}, not {dtype}")
    h = R._handle(stream)
    rc = m.mx4_product(a, a_scale, b, b_scale, group_ptr, out, workspace, h)
    if rc == EWORKSPACE and workspace is None:
        workspace = R._new((mx4_product_workspace_bytes(rows, channels, 2 * shape[-1], groups),), R._torch.uint8, a, stream)
        rc = m.mx4_product(a, a_scale, b, b_scale, group_ptr, out, workspace, h)
    if rc:
        raise SeerError(rc, "seer_mx4_product")
    return out
