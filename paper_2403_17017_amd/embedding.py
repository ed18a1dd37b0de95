"""Binding of the embedding of tokens: rows of a table, and the gradient in the table.
The same manner, and the same refusals, as the routed layer's calls (routed.py)."""
from __future__ import annotations

import ctypes as C

from . import binding as B
from . import routed as R
from .binding import SeerError


def bind(L):
    """Argument types of the library's functions (called when the library is loaded)."""
    vp, sz, i32, i64, f32, dense = C.c_void_p, C.c_size_t, C.c_int32, C.c_int64, C.c_float, C.POINTER(R.seer_dense)
    for name, args, res in (("seer_embed", [vp, i32, dense, f32, dense, vp], C.c_int),
                            ("seer_embed_grad", [vp, i32, dense, f32, i32, dense, vp, sz, vp], C.c_int),
                            ("seer_embed_grad_workspace_bytes", [i64, i64, i64], sz)):
        f = getattr(L, name)
        f.argtypes, f.restype = args, res


def _numbers(token):
    if token is None or token.dtype not in (R._torch.int32, R._torch.int64):
        raise ValueError("token is to be a contiguous int32 or int64 tensor on the GPU")
    return token.numel()


def seer_embed(token, table, scale: float = 1.0, out=None, stream=None):
    """scale * table[token], a row for each of token's elements, [numbers, columns]; zeros for tokens that are no row's."""
    m = R._ready()
    n = _numbers(token)
    if out is None:
        out = R._new((n, R._matrix_shape(table, "table")[1]), table.dtype, table, stream)
    rc = m.embed(token, table, scale, out, R._handle(stream))
    if rc:
        raise SeerError(rc, "seer_embed")
    return out


def embed_grad_workspace_bytes(tokens: int, rows: int, columns: int) -> int:
    return int(B.lib().seer_embed_grad_workspace_bytes(tokens, rows, columns))


def seer_embed_grad(token, dy, rows: int = None, scale: float = 1.0, dtable=None, dtype=None, accumulate: bool = False, workspace=None, stream=None):
    """The gradient of seer_embed in a table of `rows` rows, for that of its output, dy [numbers, columns], of dy's type or fp32 (dtype);
    accumulate adds it to what dtable holds."""
    m = R._ready()
    n = _numbers(token)
    if dtable is None:
        if rows is None or accumulate:
            raise ValueError("rows are wanted, or a dtable" if rows is None else "a dtable to add to is wanted")
        dtable = R._new((rows, R._matrix_shape(dy, "dy")[1]), dtype or dy.dtype, dy, stream)
    elif (rows is not None and rows != dtable.shape[0]) or (dtype is not None and dtype != dtable.dtype):
        raise ValueError("dtable has other rows or another type")
    if workspace is None:
        need = embed_grad_workspace_bytes(n, dtable.shape[0], R._matrix_shape(dy, "dy")[1])
        workspace = R._new((need,), R._torch.uint8, dy, stream) if need else None
    rc = m.embed_grad(token, dy, scale, accumulate, dtable, workspace, R._handle(stream))
    if rc:
        raise SeerError(rc, "seer_embed_grad")
    return dtable
