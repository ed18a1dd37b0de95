"""Helpers shared by the tests of the routed layer (not a test module)."""
import numpy as np
import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
#: Half a unit in the last place, relative: what one rounding to the type is off by at most.
ROUND = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
#: Half of the smallest subnormal: the same below the normal range.
TINY = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}
U32 = 2.0 ** -24


def host(t):
    """A tensor's values as a float64 (or integer) numpy array."""
    t = t.detach().cpu()
    return t.double().numpy() if t.is_floating_point() else t.numpy()


def rounded(values, kind):
    """float64 values rounded to the type, on the GPU."""
    return torch.from_numpy(np.ascontiguousarray(values)).to("cuda:0").to(TYPES[kind])


def spread(t, ld, fill=float("nan")):
    """The same matrix with `ld` elements from row to row and `fill` between."""
    wide = torch.full((t.shape[0], ld), fill, dtype=t.dtype, device=t.device)
    wide[:, : t.shape[1]] = t
    return wide[:, : t.shape[1]]


def shifted(t, by):
    """The same matrix `by` elements past where an allocation begins."""
    room = torch.empty(t.numel() + by, dtype=t.dtype, device=t.device)
    moved = room[by:].view(t.shape)
    moved.copy_(t)
    return moved


def choices(rng, tokens, choices_, experts, skew=0.0, padding=0.0):
    """[tokens, choices] experts, some far more popular than others; -1 throughout for padding tokens."""
    p = (1.0 / np.arange(1, experts + 1) ** skew)
    p /= p.sum()
    e = rng.choice(experts, size=(tokens, choices_), p=p)
    if padding:
        e[rng.random(tokens) < padding] = -1
    return e


def assert_within(got, want, allowed, what):
    assert got.shape == want.shape, (what, got.shape, want.shape)
    err = np.abs(got - want)
    bad = ~(err <= allowed)
    if bad.any():
        at = np.unravel_index(int(np.argmax(np.where(bad, np.nan_to_num(err - allowed, nan=np.inf), -np.inf))), bad.shape)
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} off; at {at} got {got[at]!r} want {want[at]!r} allowed {np.broadcast_to(allowed, bad.shape)[at]!r}")
