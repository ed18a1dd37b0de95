"""Calls of the routed layer whose workspace lies over what they read or write are refused (on the host, before any launch)."""
import ctypes as C

import pytest

import paper_2403_17017_amd as S
from paper_2403_17017_amd import routed as R

EINVAL, EWORKSPACE = -1, -4
MB = 1 << 20
FAR = 1 << 40


def test_sort():
    tokens, choices, experts = 20000, 4, 64
    need = S.route_workspace_bytes(tokens, choices, experts)
    assert need > 0
    e, ptr, order, slots = FAR, FAR + 16 * MB, FAR + 32 * MB, FAR + 48 * MB
    r = C.byref(R.seer_routing(tokens, choices, experts, ptr, order, slots))
    f = S.lib().seer_route
    count = 4 * tokens * choices
    for where in (e, e + 2 * count - 16, ptr - need + 16, ptr + 256, order + count - 16, slots - need + 16, slots):
        assert f(e, 5, r, where, need, None) == EINVAL, hex(where - FAR)
    assert f(e, 5, r, FAR + 64 * MB, need - 1, None) == EWORKSPACE


def test_products():
    rows, channels, columns = 300, 512, 8192
    need = S.i8_product_workspace_bytes(rows, channels, columns)
    assert need > 0
    a, b, out, sa, sb, ptr = (FAR + i * 64 * MB for i in range(1, 7))
    d = lambda at, n, k, kind: C.byref(R.seer_dense(at, n, k, k, kind))

    def call(ws, group_ptr=None, size=need):
        return S.lib().seer_i8_product(d(a, rows, columns, 3), sa, d(b, channels, columns, 3), sb, group_ptr, 1, d(out, rows, channels, 1), ws, size, None)
    assert S.lib().seer_i8_product_kernel(d(a, rows, columns, 3), d(b, channels, columns, 3), None, 1) == 4
    for where in (a, a + rows * columns - 16, b - need + 16, b, out, out + 2 * rows * channels - 16, sa, sa - need + 16, sb, sb + 4 * channels - 16):
        assert call(where) == EINVAL, hex(where - FAR)
    assert call(ptr - 16, ptr) == EINVAL
    assert call(FAR, size=need - 1) == EWORKSPACE


@pytest.mark.parametrize("clip", [True, False])
def test_gradients(clip):
    need = S.grad_workspace_bytes()
    g, o, norm = FAR + 16 * MB, FAR + 32 * MB, FAR + 48 * MB
    t = (R.seer_grad * 2)(R.seer_grad(g, o, 1000, 0), R.seer_grad(g + MB, g + MB, 1000, 1))

    def call(ws, size=need, at=norm):
        return S.lib().seer_grad_clip(t, 2, 1.0, at, ws, size, None) if clip else S.lib().seer_grad_norm(t, 2, at, ws, size, None)
    for where in (g, g - need + 16, g + 4000 - 16, g + MB, norm - need + 16, norm):
        assert call(where) == EINVAL, hex(where - FAR)
    if clip:
        assert call(o) == EINVAL and call(o + 4000 - 16) == EINVAL
    assert call(FAR + 64 * MB, size=need - 1) == EWORKSPACE and call(g - need + 16, size=need - 16) == EWORKSPACE
