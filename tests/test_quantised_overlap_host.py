"""seer_route_gather_i8 refuses a q whose columns of zeros, up to the next multiple of 16, lie over the slots (on the host)."""
import ctypes as C

import paper_2403_17017_amd as S
from paper_2403_17017_amd import routed as R

FAR = 1 << 40


def test_zeros_behind_the_last_row():
    tokens, choices, cols, ld = 4, 2, 20, 48
    rows = tokens * choices
    q = FAR
    x = C.byref(R.seer_dense(2 * FAR, tokens, cols, cols, 0))
    end = q + (rows - 1) * ld + 32                       # what is written of q
    for slots in (end - 4, end - 12, q + (rows - 1) * ld + 16, q):
        r = C.byref(R.seer_routing(tokens, choices, 3, 3 * FAR, 4 * FAR, slots))
        assert S.lib().seer_route_gather_i8(r, x, C.byref(R.seer_dense(q, rows, cols, ld, 3)), 5 * FAR, None) == -1, hex(slots - q)
