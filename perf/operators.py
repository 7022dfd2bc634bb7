"""The operators in front of the experts that this library is measured on: routing rules, and the matrix product with an epilogue.

Every case is one call.  ``op`` says of which operator:

``route``   scores of T tokens over E experts -> chosen experts and their weights (``moe_ep.route``)
    ``tokens, experts, top_k``; ``groups, top_groups, top2`` (groups of experts, how many of them are kept, whether a group counts by
    the sum of its two best instead of its best); ``sigmoid`` (else softmax), ``bias`` (for balance, in the choice only), ``renorm``,
    ``scale``; ``bf16`` (type of the scores), ``padded`` (a share of the tokens is padding), ``absent`` (a share of the experts is masked
    with minus infinity), ``pitch`` (scores between the beginnings of two tokens' rows)
``linear``  act(x W^T + bias) + residual (``moe_ep.linear``)
    ``rows, outs, ins``; ``w32`` (weights in fp32, else bf16), ``out32`` (results, and residual, in fp32, else bf16), ``bias``,
    ``residual``, ``act``, ``pitch`` (elements between the beginnings of two rows of x)
"""
from __future__ import annotations

import math

import torch

own = False

_ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")


def _route(tokens, experts, top_k, *, groups=1, top_groups=1, top2=False, sigmoid=False, bias=False, renorm=True, scale=1.0,
           bf16=False, padded=False, absent=False, pitch=0):
    return dict(op="route", tokens=tokens, experts=experts, top_k=top_k, groups=groups, top_groups=top_groups, top2=top2, sigmoid=sigmoid,
                bias=bias, renorm=renorm, scale=scale, bf16=bf16, padded=padded, absent=absent, pitch=pitch or experts)


def _linear(rows, outs, ins, *, w32=False, out32=False, bias=False, residual=False, act="none", pitch=0):
    return dict(op="linear", rows=rows, outs=outs, ins=ins, w32=w32, out32=out32, bias=bias, residual=residual, act=act, pitch=pitch or ins)


def listed():
    named = {
        # one sequence being decoded: 160 experts in eight groups, three of them kept, weights as they are times a constant
        "route_decode_1": _route(1, 160, 6, groups=8, top_groups=3, renorm=False, scale=16.0),
        # a decode step of a padded batch, scores from a projection that rounds to bf16
        "route_padded_256": _route(256, 128, 8, bf16=True, padded=True),
        # a ragged prefill on an odd number of experts, some of them taken out of service, scores inside wider rows
        "route_ragged_1531": _route(1531, 61, 5, sigmoid=True, bias=True, absent=True, pitch=67),
        # prefill with sigmoid scores, a bias for balance and groups that count by their two best
        "route_groups_8192": _route(8192, 256, 8, groups=8, top_groups=4, top2=True, sigmoid=True, bias=True, scale=2.5),
        # a large batch of long prompts, softmax with a bias
        "route_prefill_65536": _route(65536, 256, 8, bias=True),
        # the gate's scores of one token, its weights in fp32
        "gate_decode_1": _linear(1, 160, 5120, w32=True, out32=True),
        # and of a prefill micro-batch
        "gate_prefill_4096": _linear(4096, 128, 4096, w32=True, out32=True),
        # a few sequences decoded together: a down projection onto the residual stream
        "linear_decode_33": _linear(33, 2048, 1408, bias=True, residual=True),
        # a ragged prefill with no size that is a multiple of anything
        "linear_odd_1531": _linear(1531, 1409, 2049, bias=True, act="gelu"),
        # a micro-batch whose results and residual stay in fp32
        "linear_f32_1024": _linear(1024, 4096, 1536, out32=True, residual=True),
        # a dense layer's first projection over a prefill
        "linear_silu_4096": _linear(4096, 5632, 2048, bias=True, act="silu"),
        # the output projection of a large prefill, added to the residual stream
        "linear_residual_16384": _linear(16384, 5120, 5120, residual=True),
    }
    return [dict(case, name=name) for name, case in named.items()]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """One more call of the same ranges."""
    if rng.random() < 0.5:
        groups = rng.choice((1, 1, 1, 2, 4, 8, 16))
        experts = groups * max(1 if groups > 1 else 8, _log(rng, 16, 512) // groups)
        top_groups = rng.randint(1, groups)
        top_k = rng.randint(1, min(16, experts // groups * top_groups))
        return _route(_log(rng, 1, 65536 * 256 // max(256, experts)), experts, top_k, groups=groups, top_groups=top_groups,
                      top2=rng.random() < 0.5, sigmoid=rng.random() < 0.5, bias=rng.random() < 0.5, renorm=rng.random() < 0.7,
                      scale=rng.choice((1.0, 2.5, 16.0)), bf16=rng.random() < 0.3, padded=rng.random() < 0.3, absent=rng.random() < 0.2,
                      pitch=experts + rng.choice((0, 0, 0, 1, 8)))
    w32 = rng.random() < 0.3   # a gate: as many outputs as there are experts
    outs = _log(rng, 8, 512) if w32 else _log(rng, 64, 5632)
    ins = _log(rng, 64, 5120)
    if rng.random() < 0.75:    # most sizes are multiples of 64
        ins = (ins + 63) // 64 * 64
        outs = outs if w32 else (outs + 63) // 64 * 64
    return _linear(_log(rng, 1, 16384), outs, ins, w32=w32, out32=w32 or rng.random() < 0.2, bias=rng.random() < 0.5,
                   residual=not w32 and rng.random() < 0.5, act="none" if w32 else rng.choice(_ACTS), pitch=ins + rng.choice((0, 0, 0, 8, 3)))


# ---- inputs

def _route_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    T, E, pitch = case["tokens"], case["experts"], case["pitch"]
    # scores of a trained gate: a spread of about one over the experts, and some experts liked by all tokens
    rows = torch.empty((T, pitch), dtype=torch.float32, device="cuda").normal_(generator=gen)
    rows += 0.5 * torch.empty(pitch, dtype=torch.float32, device="cuda").normal_(generator=gen)
    bias = 0.05 * torch.empty(E, dtype=torch.float32, device="cuda").normal_(generator=gen) if case["bias"] else None
    mask = None
    if case["padded"]:
        mask = (torch.empty(T, dtype=torch.float32, device="cuda").uniform_(generator=gen) < 0.7).to(torch.uint8)
    if case["absent"]:
        rows[:, torch.empty(pitch, dtype=torch.float32, device="cuda").uniform_(generator=gen) < 0.1] = -math.inf
    rows = rows.to(torch.bfloat16) if case["bf16"] else rows
    return rows[:, :E], bias, mask


def _linear_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    R, N, K = case["rows"], case["outs"], case["ins"]

    def normal(shape, std, wide):
        return torch.empty(shape, dtype=torch.float32 if wide else torch.bfloat16, device="cuda").normal_(0.0, std, generator=gen)

    # activations behind a normalisation, weights at the usual initialisation scale
    x = normal((R, case["pitch"]), 1.0, False)[:, :K]
    weight = normal((N, K), 0.02, case["w32"])
    bias = normal((N,), 0.1, True) if case["bias"] else None
    residual = normal((R, N), 1.0, case["out32"]) if case["residual"] else None
    return x, weight, bias, residual


def prepare(case, seed):
    if case["op"] == "route":
        scores, bias, mask = _route_inputs(case, seed)
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        state = dict(case=case, args=(scores, bias, mask), idx=torch.empty((T, k), dtype=torch.int32, device="cuda"),
                     w=torch.empty((T, k), dtype=torch.float32, device="cuda"))
        if own:
            import paper_2512_21487_amd as moe_ep
            state["call"] = moe_ep.route
            state["rule"] = moe_ep.Routing(
                n_experts=E, top_k=k, n_groups=case["groups"], top_groups=case["top_groups"],
                score=moe_ep.SCORE_SIGMOID if case["sigmoid"] else moe_ep.SCORE_SOFTMAX,
                group_score=moe_ep.GROUP_TOP2 if case["top2"] else moe_ep.GROUP_MAX, renormalise=int(case["renorm"]), scale=case["scale"],
                score_type=moe_ep.BF16 if case["bf16"] else moe_ep.F32, score_stride=case["pitch"])
        return state
    x, weight, bias, residual = _linear_inputs(case, seed)
    out_type = torch.float32 if case["out32"] else torch.bfloat16
    state = dict(case=case, args=(x, weight, bias, residual), out=torch.empty((case["rows"], case["outs"]), dtype=out_type, device="cuda"))
    if own:
        import paper_2512_21487_amd as moe_ep
        state["call"] = moe_ep.linear
        state["rule"] = moe_ep.LinearConfig(
            in_features=case["ins"], out_features=case["outs"], weight_type=moe_ep.F32 if case["w32"] else moe_ep.BF16,
            out_type=moe_ep.F32 if case["out32"] else moe_ep.BF16, activation=_ACTS.index(case["act"]), x_stride=case["pitch"])
    return state


# ---- the plain forms

def _route_plain(case, scores, bias, mask):
    """In 64 bits throughout: which experts are chosen may not hang on the rounding of a sum."""
    T, E, k, G = case["tokens"], case["experts"], case["top_k"], case["groups"]
    there = scores > torch.finfo(scores.dtype).min
    if bias is not None:
        there = there & (bias > -math.inf)
    if mask is not None:
        there = there & (mask != 0)[:, None]
    s = torch.where(there, scores.double().clamp(max=torch.finfo(torch.float32).max), -math.inf)
    if case["sigmoid"]:
        p = 1.0 / (1.0 + torch.exp(-s))
    else:
        top = s.amax(dim=1, keepdim=True)
        p = torch.exp(s - torch.where(top > -math.inf, top, 0.0))
        total = p.sum(dim=1, keepdim=True)
        p = p / torch.where(total > 0.0, total, 1.0)
    value = p if bias is None else p + bias.double()
    value = torch.where(there, value, -math.inf)
    key = s if bias is None else value
    if G > 1:
        best = (value if case["top2"] or bias is not None else s).view(T, G, E // G).sort(dim=2, descending=True).values
        group = best[:, :, 0]
        if case["top2"] and E // G > 1:
            group = group + torch.where(best[:, :, 1] > -math.inf, best[:, :, 1], 0.0)
        place = torch.sort(group, dim=1, descending=True, stable=True).indices
        kept = torch.zeros((T, G), dtype=torch.bool, device=s.device).scatter_(1, place[:, :case["top_groups"]], True)
        key = torch.where(kept[:, :, None].expand(T, G, E // G).reshape(T, E), key, -math.inf)
    best, idx = torch.sort(key, dim=1, descending=True, stable=True)
    best, idx = best[:, :k], idx[:, :k]
    full = best > -math.inf
    w = torch.where(full, p.gather(1, idx), 0.0)
    if case["renorm"]:
        total = w.sum(dim=1, keepdim=True)
        w = w / torch.where(total > 0.0, total, 1.0)
    return torch.where(full, idx, -1).to(torch.int32), (w * case["scale"]).float()


def _act(name, z):
    if name == "relu":
        return z.clamp(min=0.0)
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _linear_plain(case, x, weight, bias, residual):
    y = x.float() @ weight.float().t()
    if bias is not None:
        y = y + bias
    y = _act(case["act"], y)
    if residual is not None:
        y = y + residual.float()
    return y if case["out32"] else y.to(torch.bfloat16)


def run(state):
    case = state["case"]
    if case["op"] == "route":
        scores, bias, mask = state["args"]
        if own:
            state["call"](state["rule"], scores, bias, mask, idx=state["idx"], w=state["w"])
            return {"idx": state["idx"], "w": state["w"]}
        idx, w = _route_plain(case, scores, bias, mask)
        return {"idx": idx, "w": w}
    if own:
        x, weight, bias, residual = state["args"]
        state["call"](state["rule"], x, weight, bias, residual, out=state["out"])
        return {"out": state["out"]}
    return {"out": _linear_plain(case, *state["args"])}


def work(case):
    if case["op"] == "route":
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        read = T * E * (2 if case["bf16"] else 4) + (4 * E if case["bias"] else 0) + (T if case["padded"] else 0)
        # an exponential, a division and a comparison for every score
        return {"bytes": float(read + 8 * T * k), "flops": 3.0 * T * E}
    R, N, K = case["rows"], case["outs"], case["ins"]
    size = 4 if case["out32"] else 2
    read = 2 * R * K + (4 if case["w32"] else 2) * N * K + (4 * N if case["bias"] else 0) + (size * R * N if case["residual"] else 0)
    return {"bytes": float(read + size * R * N), "flops": 2.0 * R * N * K}


# ---- from the definitions, in 64 bits

def _exact_weights(case, scores, bias, mask):
    """The weights alone, a token's chosen experts found by counting how many are before each."""
    T, E, k, G = case["tokens"], case["experts"], case["top_k"], case["groups"]
    out = torch.zeros((T, k), dtype=torch.float64, device=scores.device)
    step = max(1, (1 << 25) // (E * E))
    number = torch.arange(E, device=scores.device)
    for t0 in range(0, T, step):
        s = scores[t0:t0 + step].double()
        n = s.shape[0]
        gone = torch.isnan(s) | (s <= torch.finfo(scores.dtype).min)
        if bias is not None:
            gone |= torch.isnan(bias) | torch.isneginf(bias)
        if mask is not None:
            gone |= (mask[t0:t0 + step] == 0)[:, None]
        s = s.masked_fill(gone, -math.inf)
        p = torch.sigmoid(s) if case["sigmoid"] else torch.nan_to_num(torch.softmax(s, dim=1))
        c = (p + bias.double() if bias is not None else p).masked_fill(gone, -math.inf)
        order = c if bias is not None else s
        if G > 1:
            size = E // G
            members = c.view(n, G, size)
            if case["top2"]:
                two = members.topk(min(2, size), dim=2).values
                value = two.masked_fill(torch.isneginf(two), 0.0).sum(dim=2).masked_fill(torch.isneginf(two[:, :, 0]), -math.inf)
            else:
                value = members.amax(dim=2) if bias is not None else s.view(n, G, size).amax(dim=2)
            g = torch.arange(G, device=s.device)
            ahead = (value[:, None, :] > value[:, :, None]) | ((value[:, None, :] == value[:, :, None]) & (g[None, :] < g[:, None]))
            lost = ahead.sum(dim=2) >= case["top_groups"]
            order = order.masked_fill(lost[:, :, None].expand(n, G, size).reshape(n, E), -math.inf)
        ahead = (order[:, None, :] > order[:, :, None]) | ((order[:, None, :] == order[:, :, None]) & (number[None, :] < number[:, None]))
        place = ahead.sum(dim=2)
        chosen = (place < k) & ~torch.isneginf(order)
        token, expert = torch.nonzero(chosen, as_tuple=True)
        out[t0 + token, place[token, expert]] = p[token, expert]
    if case["renorm"]:
        out = torch.nan_to_num(out / out.sum(dim=1, keepdim=True))
    return out * case["scale"]


def exact(case, seed):
    if case["op"] == "route":
        return {"idx": None, "w": _exact_weights(case, *_route_inputs(case, seed))}
    x, weight, bias, residual = (None if v is None else v.double() for v in _linear_inputs(case, seed))
    z = torch.matmul(x, weight.t())
    z = z if bias is None else z + bias
    y = {"none": lambda v: v, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu,
         "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}[case["act"]](z)
    return {"out": y if residual is None else y + residual}
