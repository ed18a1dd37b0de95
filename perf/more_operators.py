"""A routed layer's router, its experts' products in 4 bits and its tokens' embedding, as measurable cases.

Kinds of case (`op`):

  choose      every token's experts and their weights, from the router's scores (seer_route_choose)
  train       the same with the gradient that the weights hand back to the logits
              (seer_route_choose, seer_route_choose_grad)
  mx4         4-bit floating point in blocks of 32 with a shared power of two: the tokens are quantised
              (seer_mx4_quantize, or seer_route_gather_mx4 on the way to the experts) and multiplied
              (seer_mx4_product), with one weight matrix or with each expert's own
  embed       rows of a table by token, scaled (seer_embed)
  embed_grad  the gradient of that in the table, summed over each token's places (seer_embed_grad)

Logits of minus infinity belong to experts that are not to be chosen; a token whose logits are nothing else is
padding and chooses none (-1).  Tokens of -1 are padding, too: no row of the table is theirs.
"""
import math

import torch

own = False

_DEVICE = "cuda:0"
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_BLOCK = 32                                  # values that share a scale


def listed():
    return [
        # one token of a running answer: scores, groups and choice in one small launch
        {"name": "choose_one_token", "op": "choose", "tokens": 1, "experts": 256, "choices": 8, "score": "sigmoid", "bias": True,
         "groups": 8, "best_groups": 4, "group_best": 2, "renormalise": True, "factor": 2.5, "type": "f32", "padding": 0.0, "masked": 0.0},
        # prompts of a whole batch, packed to an odd number of tokens, padding among them, a few experts out of service
        {"name": "choose_batch", "op": "choose", "tokens": 16411, "experts": 160, "choices": 6, "score": "softmax", "bias": False,
         "groups": 8, "best_groups": 3, "group_best": 1, "renormalise": False, "factor": 1.0, "type": "bf16", "padding": 0.03, "masked": 0.02},
        # a small model's micro batch, there and back in 32 bits
        {"name": "choose_train_micro", "op": "train", "tokens": 1031, "experts": 8, "choices": 2, "score": "softmax", "bias": False,
         "groups": 1, "best_groups": 1, "group_best": 1, "renormalise": True, "factor": 1.0, "type": "f32", "padding": 0.0, "masked": 0.0},
        # a training step with many experts, balanced by a bias, there and back
        {"name": "choose_train_batch", "op": "train", "tokens": 65536, "experts": 256, "choices": 8, "score": "sigmoid", "bias": True,
         "groups": 8, "best_groups": 4, "group_best": 2, "renormalise": True, "factor": 2.5, "type": "f32", "padding": 0.01, "masked": 0.0},
        # one token through one 4-bit weight matrix: the time it takes to read the weights
        {"name": "mx4_one_token", "op": "mx4", "tokens": 1, "choices": 1, "experts": 1, "columns": 8192, "channels": 8192,
         "type": "bf16", "padding": 0.0, "skew": 0.0},
        # a prompt through one 4-bit weight matrix, every size odd, the last block of a row not whole
        {"name": "mx4_prompt_odd", "op": "mx4", "tokens": 3001, "choices": 1, "experts": 1, "columns": 4111, "channels": 5001,
         "type": "f16", "padding": 0.0, "skew": 0.0},
        # 32 running answers through the 4-bit matrices of the experts that they chose: a few rows each
        {"name": "mx4_experts_decode", "op": "mx4", "tokens": 32, "choices": 8, "experts": 64, "columns": 4096, "channels": 2048,
         "type": "bf16", "padding": 0.0, "skew": 1.0},
        # prompts of a batch through the experts' 4-bit matrices: the largest product
        {"name": "mx4_experts_batch", "op": "mx4", "tokens": 8192, "choices": 4, "experts": 32, "columns": 4096, "channels": 4096,
         "type": "bf16", "padding": 0.01, "skew": 0.5},
        # 48 running answers look up the token that each has just chosen
        {"name": "embed_decode", "op": "embed", "tokens": 48, "rows": 131072, "columns": 4096, "type": "bf16", "scale": 64.0, "padding": 0.0, "skew": 1.0},
        # prompts of a whole batch, packed to an odd number of tokens
        {"name": "embed_batch", "op": "embed", "tokens": 32771, "rows": 131072, "columns": 4096, "type": "bf16", "scale": 64.0, "padding": 0.02, "skew": 1.0},
        # a small model's micro batch in 32 bits, an odd number of tokens and columns
        {"name": "embed_grad_micro", "op": "embed_grad", "tokens": 1031, "rows": 8009, "columns": 1023, "type": "f32", "grad": "f32",
         "scale": 1.0, "padding": 0.0, "skew": 1.0},
        # a training step: the gradient of a large table, most of whose rows no token of the step touches
        {"name": "embed_grad_batch", "op": "embed_grad", "tokens": 32768, "rows": 131072, "columns": 4096, "type": "bf16", "grad": "bf16",
         "scale": 64.0, "padding": 0.01, "skew": 1.0},
    ]


def _size(rng, low, high, step=1):
    """A size whose logarithm is uniform."""
    n = int(math.exp(rng.uniform(math.log(low), math.log(high + 0.999))))
    return max(low, min(high, n // step * step if step > 1 and n >= step else n))


def draw(rng):
    op = rng.choice(("choose", "train", "mx4", "mx4", "embed", "embed_grad"))
    kind = rng.choice(("bf16", "f16", "f32"))
    if op in ("choose", "train"):
        groups = rng.choice((1, 1, 2, 4, 8))
        experts = groups * _size(rng, 2, 512 // groups)
        best = groups if groups == 1 else rng.randint(1, groups)
        return {"op": op, "tokens": _size(rng, 1, min(65536, 65536 * 256 // experts)), "experts": experts,
                "choices": rng.randint(1, min(10, best * (experts // groups))), "score": rng.choice(("softmax", "sigmoid")),
                "bias": rng.random() < 0.5, "groups": groups, "best_groups": best, "group_best": rng.choice((1, 2)),
                "renormalise": rng.random() < 0.6, "factor": rng.choice((1.0, 1.0, 2.5)), "type": kind,
                "padding": rng.choice((0.0, 0.0, 0.02, 0.2)), "masked": rng.choice((0.0, 0.0, 0.05))}
    if op in ("embed", "embed_grad"):
        columns = _size(rng, 64, 8192, rng.choice((1, 8, 64, 64)))
        case = {"op": op, "tokens": 1, "rows": _size(rng, 2, min(262144, (1 << 30) // (columns * 4))), "columns": columns, "type": kind,
                "scale": rng.choice((1.0, 32.0, columns ** 0.5)), "padding": rng.choice((0.0, 0.0, 0.02, 0.2)), "skew": rng.choice((0.0, 0.5, 1.0, 1.3))}
        if op == "embed_grad":
            case["grad"] = rng.choice((kind, "f32"))
        case["tokens"] = _size(rng, 1, min(32768, (256 << 20) // (columns * _BYTES[kind])))
        return case
    one = rng.random() < 0.5
    experts = 1 if one else _size(rng, 2, 64)
    case = {"op": op, "tokens": 1, "choices": min(experts, rng.randint(1, 8)), "experts": experts,
            "columns": _size(rng, 256, 8192, rng.choice((1, 32, 64, 64))), "channels": _size(rng, 128, 8192, rng.choice((1, 8, 64, 64))),
            "type": rng.choice(("bf16", "f16")), "padding": 0.0 if one else rng.choice((0.0, 0.0, 0.02, 0.2)), "skew": rng.choice((0.0, 0.5, 1.0))}
    while case["experts"] * case["columns"] * case["channels"] > 32 * 4096 * 4096:
        case["experts"] = max(1, case["experts"] // 2)
        case["choices"] = min(case["choices"], case["experts"])
    if case["experts"] == 1:
        case["padding"] = 0.0
    case["tokens"] = _size(rng, 1, max(1, min(8192, 8192 * 4 * 4096 * 4096 // (case["choices"] * case["columns"] * case["channels"]))))
    return case


# ---------------------------------------------------------------- inputs

def _choices(case, g):
    """int64 [tokens, choices]: distinct experts of each token, some of them chosen far more often than others, and -1
    throughout for padding tokens."""
    T, C, E = case["tokens"], case["choices"], case["experts"]
    liking = -case["skew"] * torch.log(torch.arange(1, E + 1, device=_DEVICE, dtype=torch.float32))
    liking = liking[torch.randperm(E, generator=g, device=_DEVICE)]
    u = torch.rand(T, E, generator=g, device=_DEVICE).clamp_(1e-9, 1 - 1e-7)
    expert = torch.topk(liking - torch.log(-torch.log(u)), C, dim=1).indices
    if case["padding"]:
        pad = torch.rand(T, 1, generator=g, device=_DEVICE) < case["padding"]
        expert = torch.where(pad, torch.full_like(expert, -1), expert)
    return expert.contiguous()


def _order(expert, E):
    """The choices sorted by expert, by elementary operations: (expert_ptr, slot_choice, choice_slot)."""
    flat = expert.reshape(-1)
    key = torch.where((flat >= 0) & (flat < E), flat, torch.full_like(flat, E))
    slot_choice = torch.argsort(key, stable=True)
    expert_ptr = torch.searchsorted(key[slot_choice], torch.arange(E + 1, device=flat.device))
    choice_slot = torch.empty_like(slot_choice)
    choice_slot[slot_choice] = torch.arange(flat.numel(), device=flat.device)
    choice_slot = torch.where(key == E, -1 - choice_slot, choice_slot)
    return expert_ptr.int(), slot_choice.int(), choice_slot.int().reshape(expert.shape)


def _tokens(case, g):
    """int64 [tokens]: ids by a power law over the table, the most frequent ones anywhere in it, and -1 for padding."""
    T, V = case["tokens"], case["rows"]
    share = torch.arange(1, V + 1, device=_DEVICE, dtype=torch.float64) ** -case["skew"]
    upto = torch.cumsum(share, 0)
    rank = torch.searchsorted(upto, torch.rand(T, generator=g, device=_DEVICE, dtype=torch.float64) * upto[-1]).clamp_(max=V - 1)
    token = torch.randperm(V, generator=g, device=_DEVICE)[rank]
    pad = torch.rand(T, generator=g, device=_DEVICE) < case["padding"]
    return torch.where(pad, torch.full_like(token, -1), token)


def prepare(case, seed):
    g = torch.Generator(device=_DEVICE).manual_seed(int(seed))
    dtype = _TYPES[case["type"]]
    op = case["op"]

    def normal(*shape, scale=1.0, dtype=dtype):
        return torch.randn(*shape, generator=g, device=_DEVICE, dtype=dtype) * scale

    state = {"case": dict(case)}
    if op in ("choose", "train"):
        T, E = case["tokens"], case["experts"]
        liking = normal(1, E, scale=0.7, dtype=torch.float32)
        x = normal(T, E, scale=1.5, dtype=torch.float32) + liking
        out = torch.rand(E, generator=g, device=_DEVICE) < case["masked"]
        out[: 2 * case["choices"]] = False
        pad = torch.rand(T, generator=g, device=_DEVICE) < case["padding"]
        x.masked_fill_(out[None, :] | pad[:, None], -math.inf)
        state["logits"] = x.to(dtype)
        # what a balancing rule leaves that takes steps of 0.001 against the experts' load
        state["bias"] = torch.round(-30 * liking[0] + normal(E, scale=5, dtype=torch.float32)) * 0.001 if case["bias"] else None
        if op == "train":
            state["dweight"] = normal(T, case["choices"], scale=0.01, dtype=torch.float32)
        if own:
            import paper_2403_17017_amd as S
            state["how"] = S.Choice(**{k: case[k] for k in ("choices", "score", "groups", "best_groups", "group_best", "renormalise", "factor")})
        return state
    if op in ("embed", "embed_grad"):
        state["token"] = _tokens(case, g)
        if op == "embed":
            state["table"] = normal(case["rows"], case["columns"], scale=0.02)
        else:
            state["dy"] = normal(case["tokens"], case["columns"], scale=0.01)
        return state
    T, E, D, N = case["tokens"], case["experts"], case["columns"], case["channels"]
    state["expert"] = _choices(case, g)
    state["x"] = normal(T, D)
    state["x"][:, :: 97] *= 8                # a few columns are far larger than the others
    state["order"] = _order(state["expert"], E) if E > 1 else None
    state["most"] = int((state["order"][0][1:] - state["order"][0][:-1]).max()) if E > 1 else T    # rows of the busiest expert
    blocks = -(-D // _BLOCK)
    state["w"] = torch.empty(E, N, blocks * _BLOCK // 2, dtype=torch.uint8, device=_DEVICE)
    state["w_scale"] = torch.empty(E, N, blocks, dtype=torch.uint8, device=_DEVICE)
    for e in range(E):                       # weights in 4 bits: two to a byte, the first in the lower half
        value, exponent = _plain_quantised(normal(N, D, scale=D ** -0.5, dtype=torch.float32))
        m = value.abs()
        code = torch.where(m < 2, 2 * m, torch.where(m < 4, m + 2, m / 2 + 4)).to(torch.uint8) + 8 * (value < 0).to(torch.uint8)
        state["w"][e] = code[:, 0::2] + 16 * code[:, 1::2]
        state["w_scale"][e] = (exponent + 127).to(torch.uint8)
    return state


# ---------------------------------------------------------------- one pass

def run(state):
    op = state["case"]["op"]
    if own:
        return _RUN_OWN[op](state)
    return _RUN_PLAIN[op](state)


def _own_choose(state):
    import paper_2403_17017_amd as S
    return list(S.seer_route_choose(state["logits"], state["how"], bias=state["bias"]))


def _own_train(state):
    import paper_2403_17017_amd as S
    expert, weight = S.seer_route_choose(state["logits"], state["how"], bias=state["bias"])
    return [expert, weight, S.seer_route_choose_grad(state["logits"], state["how"], expert, state["dweight"])]


def _own_mx4(state):
    import paper_2403_17017_amd as S
    dtype = state["x"].dtype
    if state["order"] is None:
        q, scale = S.seer_mx4_quantize(state["x"])
        return S.seer_mx4_product(q, scale, state["w"], state["w_scale"], dtype=dtype)
    r = S.Routing(state["case"]["experts"], *state["order"])
    q, scale = S.seer_route_gather_mx4(r, state["x"])
    return S.seer_mx4_product(q, scale, state["w"], state["w_scale"], group_ptr=r.expert_ptr, dtype=dtype)


def _own_embed(state):
    import paper_2403_17017_amd as S
    return S.seer_embed(state["token"], state["table"], scale=state["case"]["scale"])


def _own_embed_grad(state):
    import paper_2403_17017_amd as S
    case = state["case"]
    return S.seer_embed_grad(state["token"], state["dy"], case["rows"], scale=case["scale"], dtype=_TYPES[case["grad"]])


def _plain_scores(case, logits):
    """The scores in 64 bits: next to a border 32 would choose otherwise."""
    x = logits.double()
    if case["score"] == "sigmoid":
        return torch.sigmoid(x)
    most = x.amax(1, keepdim=True)
    e = torch.exp(x - torch.where(torch.isinf(most), torch.zeros_like(most), most))
    return e / e.sum(1, keepdim=True)


def _plain_chosen(case, logits, bias):
    """(experts int64 [tokens, choices], -1 for none; the scores): best first, ties to the lower number."""
    x, G, lowest = logits.double(), case["groups"], -math.inf
    score = _plain_scores(case, logits)
    shut = x == lowest
    key = torch.where(shut, torch.full_like(x, lowest), score + bias.double() if bias is not None else x)
    if case["best_groups"] < G:
        T, E = x.shape
        by_score = key if bias is not None else torch.where(shut, key, score)
        if case["group_best"] == 1:
            group = key.view(T, G, -1).amax(2)
        else:
            two = torch.sort(by_score.view(T, G, -1), dim=2, descending=True).values[:, :, :2]
            group = torch.where(two[:, :, 0] == lowest, two[:, :, 0], torch.where(two == lowest, torch.zeros_like(two), two).sum(2))
        best = torch.sort(group, dim=1, descending=True, stable=True).indices[:, : case["best_groups"]]
        open_ = torch.zeros(T, G, dtype=torch.bool, device=x.device).scatter_(1, best, True)
        key = torch.where(open_.repeat_interleave(E // G, 1), key, torch.full_like(key, lowest))
    top = torch.sort(key, dim=1, descending=True, stable=True)
    expert = top.indices[:, : case["choices"]]
    return torch.where(top.values[:, : case["choices"]] == lowest, torch.full_like(expert, -1), expert), score


def _plain_weights(case, expert, score):
    s = torch.where(expert >= 0, score.gather(1, expert.clamp(min=0)), torch.zeros((), dtype=score.dtype, device=score.device))
    if case["renormalise"]:
        total = s.sum(1, keepdim=True)
        s = s / torch.where(total > 0, total, torch.ones_like(total))
    return s


def _plain_choose(state):
    case = state["case"]
    expert, score = _plain_chosen(case, state["logits"], state["bias"])
    return [expert.int(), (case["factor"] * _plain_weights(case, expert, score)).float()]


def _plain_train(state):
    case, logits = state["case"], state["logits"]
    expert, score = _plain_chosen(case, logits, state["bias"])
    w = _plain_weights(case, expert, score)
    dw, chosen, at = state["dweight"], expert >= 0, expert.clamp(min=0)
    weight = (case["factor"] * w).float()
    w, score = w.float(), score.float()
    dw = torch.where(chosen, dw, torch.zeros_like(dw)) * case["factor"]
    if case["renormalise"]:
        inner = w * (dw - (w * dw).sum(1, keepdim=True))
    else:
        inner = w * dw
    if case["score"] == "sigmoid":
        inner = inner * torch.sigmoid(-logits.float()).gather(1, at)
    dlogits = torch.zeros_like(score).scatter_add_(1, at, torch.where(chosen, inner, torch.zeros_like(inner)))
    if case["score"] == "softmax" and not case["renormalise"]:
        dlogits = dlogits - torch.nan_to_num(score) * inner.sum(1, keepdim=True)
    return [expert.int(), weight, dlogits.to(logits.dtype)]


def _plain_quantised(x):
    """(values in blocks of 32 as 4 bits hold them, the exponents of their scales): scale = 2^(floor(log2 max|x|) - 2), value
    = x / scale to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to the even code.  The last block is filled up with zeros."""
    rows, cols = x.shape
    blocks = -(-cols // _BLOCK)
    x = torch.nn.functional.pad(x.float(), (0, blocks * _BLOCK - cols)).view(rows, blocks, _BLOCK)
    most = x.abs().amax(2)
    exponent = torch.where(most > 0, torch.frexp(most).exponent - 3, torch.full((), -127, dtype=torch.int32, device=x.device)).clamp(-127, 127)
    x = torch.ldexp(x, -exponent[:, :, None])
    m = x.abs()
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0))
    value = (torch.round(m / step) * step).clamp(max=6.0)
    return torch.where(x < 0, -value, value).view(rows, -1), exponent


def _plain_values(code, scale):
    """What 4-bit codes, two to a byte, and their blocks' scales stand for, in 32 bits."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=code.device)
    value = torch.stack((table[(code & 15).int()], table[(code >> 4).int()]), -1).view(*scale.shape, _BLOCK)
    return torch.ldexp(value, (scale.int() - 127)[..., None]).view(*code.shape[:-1], -1)


def _plain_mx4(state):
    x, w = state["x"], _plain_values(state["w"], state["w_scale"])
    value, exponent = _plain_quantised(x)
    value = torch.ldexp(value.view(*exponent.shape, _BLOCK), exponent[:, :, None]).view(value.shape)
    if state["order"] is None:
        return (value @ w[0].t()).to(x.dtype)
    ptr, slot_choice, choice_slot = (t.long() for t in state["order"])
    E, most, S = w.shape[0], state["most"], slot_choice.numel()
    # every expert's rows in a block of its own, as many as the busiest one has
    place = ptr[:-1, None] + torch.arange(most, device=x.device)[None, :]
    mine = place < ptr[1:, None]
    token = slot_choice[place.clamp(max=S - 1)] // choice_slot.shape[1]
    out = torch.zeros(S + 1, w.shape[1], dtype=x.dtype, device=x.device)
    for e in range(E):
        y = (value[token[e]] @ w[e].t()).to(x.dtype)
        out[torch.where(mine[e], place[e], torch.full_like(place[e], S))] = y      # what is no row of the expert goes to a row of its own
    return out[:S]


def _plain_embed(state):
    token, table = state["token"], state["table"]
    known = (token >= 0) & (token < table.shape[0])
    rows = table[token.clamp(0, table.shape[0] - 1)].float() * state["case"]["scale"]
    return torch.where(known[:, None], rows, torch.zeros_like(rows)).to(table.dtype)


def _plain_embed_grad(state):
    token, dy, case = state["token"], state["dy"], state["case"]
    at = torch.where((token >= 0) & (token < case["rows"]), token, torch.full_like(token, case["rows"]))
    total = torch.zeros(case["rows"] + 1, dy.shape[1], device=dy.device).index_add_(0, at, dy.float())
    return (total[:-1] * case["scale"]).to(_TYPES[case["grad"]])


_RUN_OWN = {"choose": _own_choose, "train": _own_train, "mx4": _own_mx4, "embed": _own_embed, "embed_grad": _own_embed_grad}
_RUN_PLAIN = {"choose": _plain_choose, "train": _plain_train, "mx4": _plain_mx4, "embed": _plain_embed, "embed_grad": _plain_embed_grad}


# ---------------------------------------------------------------- the definition in 64 bits

def _exact_choice(case, state):
    import numpy as np
    x = state["logits"].double().cpu().numpy()
    T, E, C, G = x.shape[0], case["experts"], case["choices"], case["groups"]
    there = ~np.isneginf(x)
    with np.errstate(all="ignore"):
        if case["score"] == "softmax":
            log_s = x - np.where(there.any(1), x.max(1), 0)[:, None]
            log_s -= np.log(np.exp(log_s).sum(1, keepdims=True))
        else:
            log_s = -np.logaddexp(0.0, -x)
        s = np.where(there, np.exp(log_s), 0.0)
    key = s + state["bias"].double().cpu().numpy() if case["bias"] else x.copy()
    key[~there] = -np.inf
    if case["best_groups"] < G:
        points = key if case["bias"] or case["group_best"] == 1 else np.where(there, s, -np.inf)
        ranked = -np.sort(-points.reshape(T, G, E // G), axis=2)
        group = ranked[:, :, 0].copy()
        if case["group_best"] == 2 and E // G > 1:
            group += np.where(np.isneginf(ranked[:, :, 1]), 0.0, ranked[:, :, 1])
        shut = np.ones((T, G), bool)
        for _ in range(case["best_groups"]):
            first = np.argmax(np.where(shut, group, -np.inf), axis=1)
            shut[np.arange(T), first] = False
        key[np.repeat(shut, E // G, axis=1)] = -np.inf
    expert = np.empty((T, C), np.int64)
    for k in range(C):
        expert[:, k] = np.argmax(key, axis=1)
        expert[np.isneginf(key[np.arange(T), expert[:, k]]), k] = -1
        at = expert[:, k] >= 0
        key[np.flatnonzero(at), expert[at, k]] = -np.inf
    logs = np.where(expert >= 0, np.take_along_axis(np.where(there, log_s, -np.inf), np.maximum(expert, 0), 1), -np.inf)
    if case["renormalise"]:
        some = np.where(expert[:, 0] >= 0, logs.max(1), 0.0)
        share = np.exp(logs - some[:, None])
        share /= np.maximum(share.sum(1, keepdims=True), 1e-300)
    else:
        share = np.exp(logs)
    return x, s, expert, share


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op in ("choose", "train"):
        import numpy as np
        x, s, expert, share = _exact_choice(case, state)
        weight = torch.from_numpy(case["factor"] * share)
        if op == "choose":
            return [None, weight]
        dw = np.where(expert >= 0, state["dweight"].double().cpu().numpy(), 0.0)
        # d weight_k / d score, score by score, then d score / d logit
        dlogits = np.zeros_like(x)
        for k in range(case["choices"]):
            at = np.flatnonzero(expert[:, k] >= 0)
            e = expert[at, k]
            dlog = dw[at, k] - (dw[at] * share[at]).sum(1) if case["renormalise"] else dw[at, k]
            dlog = case["factor"] * dlog * share[at, k]                # the gradient in the logarithm of the chosen score
            dlogits[at, e] += dlog * (1 / (1 + np.exp(x[at, e])) if case["score"] == "sigmoid" else 1.0)
            if case["score"] == "softmax":
                dlogits[at] -= dlog[:, None] * s[at]
        return [None, weight, torch.from_numpy(dlogits)]
    if op == "embed":
        token = state["token"]
        out = torch.zeros(case["tokens"], case["columns"], dtype=torch.float64, device=_DEVICE)
        known = torch.nonzero(token >= 0)[:, 0]
        out[known] = state["table"][token[known]].double() * case["scale"]
        return out
    if op == "embed_grad":
        out = torch.zeros(case["rows"], case["columns"], dtype=torch.float64, device=_DEVICE)
        known = torch.nonzero(state["token"] >= 0)[:, 0]
        return out.index_add_(0, state["token"][known], state["dy"][known].double()).mul_(case["scale"])
    # 4 bits: by the distance to each of the values that there are, the even code first
    x = state["x"].double()
    T, D = x.shape
    grid = torch.tensor([0.0, 1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0], dtype=torch.float64, device=_DEVICE)
    blocks = -(-D // _BLOCK)
    rows = torch.zeros(T, blocks * _BLOCK, dtype=torch.float64, device=_DEVICE)
    for b in range(blocks):
        part = x[:, b * _BLOCK: (b + 1) * _BLOCK]
        most = part.abs().amax(1)
        scale = 2.0 ** (torch.floor(torch.log2(most.clamp(min=2.0 ** -125))) - 2).clamp(min=-127)
        scale = torch.where(most >= 8 * scale, scale * 2, torch.where(most < 4 * scale, scale / 2, scale))[:, None]
        near = (part.abs()[:, :, None] / scale[:, :, None] - grid).abs().argmin(2)
        rows[:, b * _BLOCK: b * _BLOCK + part.shape[1]] = torch.sign(part) * grid[near] * scale
    C, E, N = case["choices"], case["experts"], case["channels"]
    lists = [[] for _ in range(E)]
    for c, e in enumerate(state["expert"].reshape(-1).tolist()):
        if e >= 0:
            lists[e].append(c // C)
    out = torch.zeros(T * C, N, dtype=torch.float64, device=_DEVICE)
    sign_grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=_DEVICE)
    sign_grid = torch.cat((sign_grid, -sign_grid))
    at = 0
    for e, mine in enumerate(lists):
        if mine:
            w = torch.empty(N, blocks * _BLOCK, dtype=torch.float64, device=_DEVICE)
            w[:, 0::2] = sign_grid[(state["w"][e] % 16).long()]
            w[:, 1::2] = sign_grid[(state["w"][e] // 16).long()]
            w *= (2.0 ** (state["w_scale"][e].double() - 127)).repeat_interleave(_BLOCK, 1)
            out[at: at + len(mine)] = rows[torch.tensor(mine, device=_DEVICE)] @ w.t()
            at += len(mine)
    return out


def work(case):
    op, b = case["op"], _BYTES[case["type"]]
    T = case["tokens"]
    if op in ("choose", "train"):
        E, C = case["experts"], case["choices"]
        there = T * E * b + 8 * T * C + (4 * E if case["bias"] else 0)
        # back: the logits again (of a softmax that is renormalised, and of sigmoids, the chosen ones), the choices and their gradients
        again = T * E * b if case["score"] == "softmax" and not case["renormalise"] else T * min(E, C) * b
        return {"bytes": there + (again + 8 * T * C + T * E * b if op == "train" else 0), "flops": (8 if op == "train" else 5) * T * E}
    if op == "embed":
        return {"bytes": 8 * T + 2 * T * case["columns"] * b, "flops": T * case["columns"]}
    if op == "embed_grad":
        return {"bytes": 8 * T + T * case["columns"] * b + case["rows"] * case["columns"] * _BYTES[case["grad"]], "flops": T * case["columns"]}
    S, E, D, N = T * case["choices"], case["experts"], case["columns"], case["channels"]
    blocks, used = -(-D // _BLOCK), min(E, S)
    return {"bytes": T * D * b + used * N * blocks * 17 + S * N * b + 4 * S, "flops": 2 * S * N * D}
