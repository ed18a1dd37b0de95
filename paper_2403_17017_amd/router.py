"""Binding of the router's choice: every token's experts and their weights from the logits, and the weights' gradient.
The same manner, and the same refusals, as the routed layer's other calls (routed.py), which take what is chosen here."""
from __future__ import annotations

import ctypes as C

from . import routed as R
from .binding import SeerError

MAX_CHOICES, MAX_EXPERT_GROUPS = 64, 64
_SCORES = {"softmax": 0, "sigmoid": 1}


class seer_choice(C.Structure):
    _fields_ = [("choices", C.c_int32), ("score", C.c_int32), ("groups", C.c_int32), ("best_groups", C.c_int32),
                ("group_best", C.c_int32), ("renormalise", C.c_int32), ("factor", C.c_float)]


def bind(L):
    """Argument types of the library's functions (called when the library is loaded)."""
    vp, dense, how = C.c_void_p, C.POINTER(R.seer_dense), C.POINTER(seer_choice)
    for name, args in (("seer_route_choose", [dense, vp, how, vp, vp, vp]), ("seer_route_choose_grad", [dense, how, vp, vp, dense, vp])):
        f = getattr(L, name)
        f.argtypes, f.restype = args, C.c_int


class Choice:
    """How experts are chosen (seer_choice): `choices` of each token by `score`, "softmax" or "sigmoid"; from the best_groups of
    `groups` groups of experts that have the best expert (group_best 1) or the largest sum of two (2); their scores divided by
    their sum (renormalise) and multiplied by `factor`."""

    __slots__ = ("c", "choices")

    def __init__(self, choices: int, score: str = "softmax", groups: int = 1, best_groups: int = None, group_best: int = 1, renormalise: bool = True,
                 factor: float = 1.0):
        if score not in _SCORES:
            raise ValueError(f"score is one of {', '.join(_SCORES)}")
        self.c = seer_choice(choices, _SCORES[score], groups, groups if best_groups is None else best_groups, group_best, bool(renormalise), factor)
        self.choices = self.c.choices

    def __repr__(self):
        return "Choice(" + ", ".join(f"{n}={getattr(self.c, n)}" for n, _ in seer_choice._fields_) + ")"


def seer_route_choose(logits, how: Choice, bias=None, expert=None, weight=None, stream=None):
    """(expert int32, weight fp32), both [tokens, choices]: the experts chosen by logits [tokens, experts] and, if given, the
    fp32 bias [experts]; -1 with weight 0 where too few are to be had."""
    m = R._ready()
    if expert is None:
        expert = R._new((R._matrix_shape(logits, "logits")[0], max(how.choices, 0)), R._torch.int32, logits, stream)
    if weight is None:
        weight = R._new((R._matrix_shape(logits, "logits")[0], max(how.choices, 0)), R._torch.float32, logits, stream)
    rc = m.choose(logits, bias, C.addressof(how.c), expert, weight, R._handle(stream))
    if rc:
        raise SeerError(rc, "seer_route_choose")
    return expert, weight


def seer_route_choose_grad(logits, how: Choice, expert, dweight, dlogits=None, stream=None):
    """The gradient of seer_route_choose's weights in the logits, for that of the weights, dweight."""
    m = R._ready()
    if expert is None or dweight is None:
        raise ValueError("expert and dweight are wanted")
    if dlogits is None:
        dlogits = R._new(R._matrix_shape(logits, "logits"), logits.dtype, logits, stream)
    rc = m.choose_grad(logits, C.addressof(how.c), expert, dweight, dlogits, R._handle(stream))
    if rc:
        raise SeerError(rc, "seer_route_choose_grad")
    return dlogits
