"""seer_grad_clip refuses lists in which something that is written is anything else's, too (on the host, before any launch)."""
import ctypes as C
import random

import pytest

import paper_2403_17017_amd as S
from paper_2403_17017_amd import routed as R

EINVAL, EWORKSPACE = -1, -4
BASE, NORM = 1 << 30, 1 << 20


def clip(tensors, norm=True):
    """The status of a call that lacks only its workspace; tensors: (grad, out, n, type)."""
    t = (R.seer_grad * max(len(tensors), 1))(*(R.seer_grad(*x) for x in tensors))
    if norm:
        return S.lib().seer_grad_clip(t, len(tensors), 1.0, NORM, None, 0, None)
    return S.lib().seer_grad_norm(t, len(tensors), NORM, None, 0, None)


def test_lists_that_are_refused():
    a, b, c, d = (BASE + i * 4096 for i in range(4))
    assert clip([(a, a, 100, 0), (b, b, 100, 0), (c, d, 100, 0)]) == EWORKSPACE           # these are fine
    assert clip([(a, a, 100, 0), (a, a, 100, 0)]) == EINVAL                               # a tensor listed twice, in place
    assert clip([(a, a, 100, 0), (b, b, 10, 0), (a + 396, a + 396, 9, 0)]) == EINVAL      # ... or a part of it
    assert clip([(a, c, 100, 0), (b, c + 200, 100, 0)]) == EINVAL                         # results on top of one another
    assert clip([(a, c, 100, 0), (b, d, 100, 0), (c + 396, d + 2048, 4, 0)]) == EINVAL    # a result on another's gradient
    assert clip([(c, d, 100, 1), (a, c + 198, 8, 2)]) == EINVAL
    assert clip([(a, a, 100, 0), (b, a, 100, 0)]) == EINVAL                               # a result on a gradient clipped in place
    assert clip([(a, c, 100, 0), (b, c + 400, 100, 0)]) == EWORKSPACE                     # one right behind the other
    assert clip([(a, c, 100, 0), (a, d, 100, 0)]) == EWORKSPACE                           # read twice, written apart
    assert clip([(a, a, 100, 0), (a, a, 0, 0), (None, None, 0, 1)]) == EWORKSPACE         # nothing of an empty one is written
    assert clip([(a, a, 100, 0), (a, a, 100, 0)], norm=False) == EWORKSPACE               # the norm alone only reads


@pytest.mark.parametrize("seed", range(200))
def test_against_every_pair(seed):
    """Lists of every length to either side of the array that is held without an allocation, in any order."""
    rng = random.Random(seed)
    tensors, at = [], BASE
    for _ in range(rng.choice((1, 2, 3, 10, 63, 64, 65, 127, 128, 129, 300))):
        kind, n = rng.randrange(3), rng.choice((0, 1, rng.randrange(1, 200)))
        room = 4 * n + 4 * rng.randrange(3)
        grad, at = at, at + room
        out, at = (grad, at) if rng.random() < 0.5 else (at, at + room)
        tensors.append([grad, out, n, kind])
    if rng.random() < 0.6:                                             # and something moved to where something else may be
        for _ in range(rng.randrange(1, 3)):
            i, j = rng.randrange(len(tensors)), rng.randrange(len(tensors))
            where = rng.randrange(2)
            to = tensors[j][rng.randrange(2)] + 4 * rng.randrange(-3, 60)
            if where == 1 or tensors[i][0] != tensors[i][1]:
                tensors[i][where] = to
            else:
                tensors[i][0] = tensors[i][1] = to
    rng.shuffle(tensors)
    size = lambda t: t[2] * (4 if t[3] == 0 else 2)
    reads = [(i, t[0], t[0] + size(t)) for i, t in enumerate(tensors) if t[2]]
    writes = [(i, t[1], t[1] + size(t)) for i, t in enumerate(tensors) if t[2]]
    bad = any(a < d and c < b for i, a, b in writes for j, c, d in writes if i < j)
    bad = bad or any(a < d and c < b and not (i == j and a == c) for i, a, b in writes for j, c, d in reads)
    assert clip(tensors) == (EINVAL if bad else EWORKSPACE)
