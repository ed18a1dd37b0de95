"""The router's choice and the embedding of tokens by their definitions, in numpy and 64 bits: what the HIP kernels are
checked against.  Inputs are host arrays; 16-bit inputs come as the float64 values they stand for."""
import numpy as np


def scores(logits, score):
    """(s, log s) of every logit; a row of minus infinities has scores of 0."""
    x = np.asarray(logits, np.float64)
    with np.errstate(all="ignore"):
        if score == "sigmoid":
            log_s = -np.logaddexp(0.0, -x)
            return np.exp(log_s), log_s
        top = x.max(axis=1, keepdims=True)
        log_s = x - np.where(np.isneginf(top), 0.0, top)
        log_s = log_s - np.log(np.exp(log_s).sum(axis=1, keepdims=True))
        log_s = np.where(np.isneginf(top), -np.inf, log_s)
        return np.exp(log_s), log_s


def _ranked(keys):
    """The numbers of a dictionary's keys: the largest value first, a NaN above all, ties to the lower number."""
    return sorted(keys, key=lambda n: (not np.isnan(keys[n]), 0.0 if np.isnan(keys[n]) else -keys[n], n))


def choose(logits, choices, score="softmax", bias=None, groups=1, best_groups=None, group_best=1, renormalise=True, factor=1.0):
    """(expert [tokens, choices], weight): a plain reading of the definition, token by token."""
    x = np.asarray(logits, np.float64)
    T, E = x.shape
    best_groups = groups if best_groups is None else best_groups
    s, log_s = scores(x, score)
    # the order is by the 64-bit scores: 1 / (1 + exp(-x)) is 1 from where exp(-x) is lost beside 1
    with np.errstate(all="ignore"):
        s64 = 1 / (1 + np.exp(-x)) if score == "sigmoid" else s
    expert, weight = np.full((T, choices), -1, np.int64), np.zeros((T, choices))
    for t in range(T):
        b = np.zeros(E) if bias is None else np.asarray(bias, np.float64)
        there = [e for e in range(E) if not np.isneginf(x[t, e]) and not np.isneginf(b[e])]
        key = {e: (x[t, e] if bias is None else s64[t, e] + b[e]) for e in there}
        if best_groups < groups:
            n, worth = E // groups, {}
            for g in range(groups):
                mine = [key[e] if bias is not None or group_best == 1 else s64[t, e] for e in there if e // n == g]
                mine.sort(key=lambda v: (not np.isnan(v), -v if not np.isnan(v) else 0))
                if mine:
                    worth[g] = mine[0] if group_best == 1 else sum(mine[:2])
            best = _ranked(worth)[:best_groups]
            there = [e for e in there if e // n in best]
        mine = _ranked({e: key[e] for e in there})[:choices]
        expert[t, :len(mine)] = mine
        if not mine:
            continue
        with np.errstate(all="ignore"):
            if renormalise:
                share = np.exp(log_s[t, mine] - log_s[t, mine].max()) if not np.isnan(log_s[t, mine]).any() else np.full(len(mine), np.nan)
                share = share / share.sum()
            else:
                share = s[t, mine]
        weight[t, :len(mine)] = factor * share
    return expert, weight


def choose_grad(logits, expert, dweight, score="softmax", renormalise=True, factor=1.0):
    """(dlogits, the sum of the magnitudes of what is added up in each)."""
    x = np.asarray(logits, np.float64)
    T, E = x.shape
    s, log_s = scores(x, score)
    d, size = np.zeros((T, E)), np.zeros((T, E))
    for t in range(T):
        mine = [(k, e) for k, e in enumerate(expert[t]) if 0 <= e < E and not np.isneginf(x[t, e])]
        if not mine:
            continue
        es = [e for _, e in mine]
        dw = np.array([dweight[t, k] for k, _ in mine])
        with np.errstate(all="ignore"):
            if renormalise:
                w = np.exp(log_s[t, es] - log_s[t, es].max())
                w = w / w.sum()
                g, m = w * (dw - np.sum(w * dw)), w * (np.abs(dw) + np.sum(w * np.abs(dw)))
            else:
                w = s[t, es]
                g, m = w * dw, w * np.abs(dw)
            if score == "sigmoid":
                other = np.exp(-np.logaddexp(0.0, x[t, es]))
                g, m = g * other, m * other
            elif not renormalise:
                d[t] -= np.where(np.isneginf(x[t]), 0.0, s[t] * g.sum())
                size[t] += np.where(np.isneginf(x[t]), 0.0, s[t] * m.sum())
        for i, e in enumerate(es):
            d[t, e] += g[i]
            size[t, e] += m[i]
    return factor * d, abs(factor) * size


def embed(token, table, scale=1.0):
    rows = table.shape[0]
    return np.stack([scale * table[v] if 0 <= v < rows else np.zeros(table.shape[1]) for v in np.asarray(token).reshape(-1)]) if np.size(token) else np.zeros((0, table.shape[1]))


def embed_grad(token, dy, rows, scale=1.0):
    """(dtable, the sum of the magnitudes of what is added up, how many rows each adds up [rows, 1])."""
    d, size, n = np.zeros((rows, dy.shape[1])), np.zeros((rows, dy.shape[1])), np.zeros((rows, 1))
    for t, v in enumerate(np.asarray(token).reshape(-1)):
        if 0 <= v < rows:
            d[v] += dy[t]
            size[v] += np.abs(dy[t])
            n[v] += 1
    return scale * d, abs(scale) * size, n
