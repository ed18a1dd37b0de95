"""Which kernel an 8-bit product takes: the host-side query, by sizes and alignment alone."""
import csv
import ctypes as C
import os

import numpy as np
import pytest
import torch

import paper_2403_17017_amd as S
from paper_2403_17017_amd import routed as R

A, B_, P = 1 << 20, 1 << 30, 1 << 10      # addresses that nothing reads


def kernel(rows, channels, columns, groups=1, ld=None, at=0, ptr=None):
    ld = columns if ld is None else ld
    a, b = R.seer_dense(A + at, rows, columns, ld, 3), R.seer_dense(B_ + at, groups * channels, columns, ld, 3)
    rc = S.lib().seer_i8_product_kernel(C.byref(a), C.byref(b), P if groups > 1 else ptr, groups)
    return S.I8_KERNELS[rc] if rc >= 0 else rc


def test_kinds():
    assert kernel(1, 8192, 8192) == "few" and kernel(1, 8192, 8192, at=1) == "few" and kernel(256, 2048, 4096, groups=64) == "few"
    assert kernel(3000, 5000, 4096) == "tiles" and kernel(30000, 4096, 4096, groups=32) == "tiles" and kernel(3000, 5000, 4111, ld=4112) == "tiles"
    assert kernel(300, 512, 8192) == "shared" and S.i8_product_workspace_bytes(300, 512, 8192) > 0
    assert kernel(3000, 5000, 4096, at=4) == "any" and kernel(3000, 5000, 4111) == "any" and kernel(3000, 700, 100) == "any"
    assert kernel(3000, 5000, 4096, ld=1 << 23) == "any"       # too far apart for 32-bit offsets into a tile
    assert kernel(5, 6, 0) == "any"
    assert kernel(0, 5, 64) == kernel(5, 0, 64) == "none"


def test_refusals():
    assert kernel(4, 8, 131072) == -6 and kernel(4, 8, 64, ld=63) == -1 and kernel(4, 8, 64, groups=0) == -1
    a, b = R.seer_dense(A, 4, 64, 64, 3), R.seer_dense(B_, 9, 64, 64, 3)
    f = S.lib().seer_i8_product_kernel
    assert f(C.byref(a), C.byref(b), P, 2) == -1               # nine rows are not two matrices
    assert f(C.byref(a), C.byref(b), None, 3) == -1 and f(None, C.byref(b), None, 1) == -1 and f(C.byref(a), None, None, 1) == -1
    with pytest.raises(ValueError):
        S.i8_product_kernel(torch.zeros(4, 64, dtype=torch.int8), torch.zeros(64, dtype=torch.int8))
    assert S.i8_product_kernel(torch.zeros(4, 64, dtype=torch.int8), torch.zeros(2, 8, 64, dtype=torch.int8), torch.zeros(3, dtype=torch.int32)) == "few"


def test_rows_off_multiples_of_16_bytes_are_priced_by_their_own_kernels():
    """Sizes at which the tiles for aligned rows would share the columns out, which nothing else does."""
    for size in ((97, 16, 3089), (100, 512, 8190), (47, 656, 8946)):
        assert kernel(*size) == "few", size            # on 1 to 6 workgroups of the tiles for any address, 40 to 140 us; few rows 23 to 62
    assert kernel(500, 130, 4111) == "any"             # few rows 113 us, tiles 57
    assert kernel(85 * 17, 186, 2278, groups=17, at=1) == "any"
    # rows too far apart for the tiles: the same choice, without a workspace
    assert kernel(97, 16, 3104, ld=1 << 23) == "few" and S.i8_product_workspace_bytes(97, 16, 3104) > 0



def test_most_tiles():
    """2^30 tiles of 128 rows by 128 channels are too many for 32-bit numbers of tiles."""
    assert kernel(1 << 22, 1 << 22, 1) == -6 and kernel((1 << 22) - 1024, (1 << 22) - 1024, 1) in S.I8_KERNELS
    assert kernel(1 << 20, 1 << 19, 1, groups=4096) == -1 and kernel(4, 8, 1, groups=4097) == -6


def test_many_short_rows_off_multiples_of_16_bytes():
    """Thousands of workgroups of few columns each cost few rows more than their bytes."""
    for size, groups in (((6435, 2168, 123), 39), ((21850, 2984, 111), 46), ((2968, 13736, 86), 7)):
        assert kernel(*size, groups=groups, at=1) == "any", size       # 33, 107 and 66 us; few rows 89, 261 and 143


def measured(where):
    import bench
    with open(os.path.join(bench.ROOT, "profiles", "i8_kernel_times.csv")) as f:
        rows = list(csv.DictReader(line for line in f if not line.startswith("#")))
    for r in (r for r in rows if r["rows_at"] == where):
        times = {k: float(r[k]) for k in ("any", "few", "tiles_64", "tiles_128", "tiles_256", "shared", "chosen") if r[k]}
        yield kernel(int(r["rows"]), int(r["channels"]), int(r["columns"]), groups=int(r["groups"]), at=where == "odd"), r["kernel"], times


def test_choice_on_measured_draws_at_odd_addresses():
    lost = [times[k] / min(times.values()) for k, _, times in measured("odd") if k in times]
    assert len(lost) > 350
    assert np.exp(np.mean(np.log(lost))) < 1.02 and max(lost) < 1.7


def test_choice_on_measured_draws():
    """The times of the kernel that was chosen when they were taken; it is of the same kind now."""
    lost = []
    for now, then, times in measured("aligned"):
        assert now == then
        lost.append(times.pop("chosen") / min(times.values()))
    assert len(lost) == 256 and np.exp(np.mean(np.log(lost))) < 1.04 and max(lost) < 1.7
