"""The routed layer's operators by their definitions, in numpy and 64 bits: what the HIP kernels are checked
against.  Inputs are host arrays; 16-bit inputs come as the float64 values they stand for."""
import numpy as np


def route(expert, experts):
    """(expert_ptr, slot_choice, choice_slot) of expert [tokens, choices]: a stable sort by expert, choices
    outside [0, experts) last and marked as -1 - slot."""
    flat = np.asarray(expert).reshape(-1).astype(np.int64)
    key = np.where((flat >= 0) & (flat < experts), flat, experts)
    slot_choice = np.array(sorted(range(flat.size), key=lambda c: (key[c], c)), np.int64)
    expert_ptr = np.array([np.count_nonzero(key < e) for e in range(experts + 1)], np.int64)
    choice_slot = np.empty(flat.size, np.int64)
    for p, c in enumerate(slot_choice):
        choice_slot[c] = p if key[c] < experts else -1 - p
    return expert_ptr, slot_choice, choice_slot.reshape(np.asarray(expert).shape)


def gather(choice_slot, x, weight=None):
    T, C = choice_slot.shape
    out = np.zeros((T * C, x.shape[1]))
    for t in range(T):
        for k in range(C):
            if choice_slot[t, k] >= 0:
                out[choice_slot[t, k]] = x[t] * (1.0 if weight is None else weight[t, k])
    return out


def combine(choice_slot, z, weight=None):
    """(y, sum of the magnitudes added up): the second bounds what fp32 sums may be off by."""
    T, C = choice_slot.shape
    y, size = np.zeros((T, z.shape[1])), np.zeros((T, z.shape[1]))
    for t in range(T):
        for k in range(C):
            if choice_slot[t, k] >= 0:
                v = z[choice_slot[t, k]] * (1.0 if weight is None else weight[t, k])
                y[t] += v
                size[t] += np.abs(v)
    return y, size


def combine_grad(choice_slot, dy, z, weight=None):
    """(dz, dweight, sum of the magnitudes in dweight)."""
    T, C = choice_slot.shape
    dz, dw, size = np.zeros((T * C, dy.shape[1])), np.zeros((T, C)), np.zeros((T, C))
    for t in range(T):
        for k in range(C):
            p = choice_slot[t, k]
            if p >= 0:
                dz[p] = dy[t] * (1.0 if weight is None else weight[t, k])
                dw[t, k] = np.sum(dy[t] * z[p])
                size[t, k] = np.sum(np.abs(dy[t] * z[p]))
    return dz, dw, size


def quantize(x):
    """(q, scale) of fp32 rows: both divisions in fp32, as the definition says."""
    x = np.asarray(x, np.float32)
    scale = (np.abs(x).max(axis=1, initial=np.float32(0)) / np.float32(127)).astype(np.float32)
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where(scale[:, None] > 0, np.rint((x / scale[:, None]).astype(np.float32)), 0)
    return np.clip(q, -127, 127).astype(np.int8), scale


def i8_product(a, a_scale, b, b_scale, group_ptr=None):
    """float64 [rows, channels]; a int8 [rows, k], b int8 [groups, channels, k]."""
    rows, groups = a.shape[0], b.shape[0]
    ptr = [0, rows] if group_ptr is None else np.clip(np.asarray(group_ptr, np.int64), 0, rows)
    out = np.zeros((rows, b.shape[1]))
    for g in range(groups):
        i = slice(int(ptr[g]), int(ptr[g + 1]))
        out[i] = (a[i].astype(np.int64) @ b[g].astype(np.int64).T) * a_scale[i].astype(np.float64)[:, None] * b_scale[g].astype(np.float64)
    return out


def grad_norm(grads):
    return float(np.sqrt(sum(float(np.sum(np.asarray(g, np.float64) ** 2)) for g in grads)))


def clip_factor(norm, max_norm):
    return min(1.0, max_norm / (norm + 1e-6))
