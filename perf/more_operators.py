"""The operators around a block that this library is measured on: norms with gate and residual, and the projection with adapters.

Every case is one call.  ``op`` says of which operator:

``norm``      h = residual_scale residual + block_scale f(gate) N_after(block);  sum = h,  out = N_before(h)  (``moe_ep.norm``)
    ``rows, cols``; ``after``, ``before`` (none, rms, layer); ``weights`` (of the norm behind the block: no ``after`` and weights is a scale per
    feature), ``biases``, ``offset`` (added to the weights); ``gate`` (none, row: one number a row, element) and ``form`` (as_is, sigmoid, silu);
    ``residual``, ``block_scale``, ``residual_scale``; ``block32, stream32, out32, weight32, gate32`` (fp32, else bf16); ``sums`` (the sum is
    written); ``pitch`` (elements between the beginnings of two rows of the block)
``adapters``  act(x W^T + bias + s_a (x A_a^T) B_a^T) + residual, a = the row's adapter  (``moe_ep.linear_adapters``)
    ``rows, outs, ins, rank, adapters``; ``requests`` (runs of rows with one adapter; as many as rows: decoding), ``bare`` (share of the requests
    without an adapter), ``out32, bias, residual, act, pitch``
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_NORMS = ("none", "rms", "layer")
_FORMS = ("as_is", "sigmoid", "silu")
_ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")
_EPS = 1e-6


def _norm(rows, cols, *, after="none", before="rms", weights=None, biases=False, offset=0.0, gate="none", form="as_is", residual=True, block_scale=1.0,
          residual_scale=1.0, block32=False, stream32=False, out32=False, weight32=False, gate32=False, sums=True, pitch=0):
    return dict(op="norm", rows=rows, cols=cols, after=after, before=before, weights=after != "none" if weights is None else weights, biases=biases,
                offset=offset, gate=gate, form=form, residual=residual, block_scale=block_scale, residual_scale=residual_scale, block32=block32,
                stream32=stream32, out32=out32, weight32=weight32, gate32=gate32, sums=sums, pitch=pitch or cols)


def _adapters(rows, outs, ins, rank, adapters, *, requests=0, bare=0.0, out32=False, bias=False, residual=False, act="none", pitch=0):
    return dict(op="adapters", rows=rows, outs=outs, ins=ins, rank=rank, adapters=adapters, requests=requests or rows, bare=bare, out32=out32,
                bias=bias, residual=residual, act=act, pitch=pitch or ins)


def listed():
    named = {
        # one sequence being decoded: the block's result onto the residual stream, and the norm in front of the next block
        "norm_decode_1": _norm(1, 5120),
        # a few sequences, norms on both sides of the block, weights stored around zero
        "norm_sandwich_33": _norm(33, 2048, after="rms", offset=1.0),
        # shared experts by a gate of their own, one score a token, onto the stream; no norm follows in this call
        "norm_gated_256": _norm(256, 4096, before="none", gate="row", form="sigmoid", gate32=True),
        # a ragged prefill with a mean taken out, biases, a stream in fp32 and no size that is a multiple of anything
        "norm_layer_1531": _norm(1531, 1409, after="layer", before="layer", biases=True, stream32=True, weight32=True, block_scale=0.22, pitch=1411),
        # a micro-batch whose block is gated element by element behind its norm
        "norm_gate_rows_4096": _norm(4096, 4096, after="rms", gate="element", form="silu", residual_scale=0.5, weight32=True),
        # a large prefill: residual and norm in front of the next block
        "norm_prefill_16384": _norm(16384, 5120, weight32=True),
        # one sequence being decoded by one of eight adapters
        "adapters_decode_1": _adapters(1, 5120, 5120, 16, 8),
        # a few sequences, most of them with an adapter of their own: a down projection onto the residual stream
        "adapters_decode_33": _adapters(33, 2048, 1408, 16, 64, bare=0.1, bias=True, residual=True),
        # a full decode step: popular adapters serve many of its rows, in no order
        "adapters_decode_256": _adapters(256, 4096, 4096, 64, 32),
        # a ragged prefill of some prompts, no size that is a multiple of anything but the rank
        "adapters_odd_1531": _adapters(1531, 1409, 2049, 24, 5, requests=7, bias=True, act="gelu"),
        # prompts and chunks of prompts, a quarter of them without an adapter: a dense layer's first projection
        "adapters_prefill_4096": _adapters(4096, 5632, 2048, 32, 16, requests=24, bare=0.25, bias=True, act="silu"),
        # the output projection of a large prefill, added to the residual stream
        "adapters_prefill_16384": _adapters(16384, 5120, 5120, 64, 16, requests=16, residual=True),
    }
    return [dict(case, name=name) for name, case in named.items()]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """One more call of the same ranges."""
    if rng.random() < 0.5:
        cols = _log(rng, 64, 8192)
        if rng.random() < 0.75:    # most sizes are multiples of 64
            cols = (cols + 63) // 64 * 64
        after, before = rng.choice(("none", "none", "rms", "layer")), rng.choice(("none", "rms", "rms", "layer"))
        return _norm(_log(rng, 1, min(16384, 16384 * 5120 // (2 * cols))), cols, after=after, before=before, weights=after != "none" or rng.random() < 0.3,
                     biases=rng.random() < 0.3, offset=rng.choice((0.0, 0.0, 1.0)), gate=rng.choice(("none", "none", "row", "element")),
                     form=rng.choice(_FORMS), residual=rng.random() < 0.8, block_scale=rng.choice((1.0, 1.0, 0.22)),
                     residual_scale=rng.choice((1.0, 1.0, 0.5)), block32=rng.random() < 0.2, stream32=rng.random() < 0.3, out32=rng.random() < 0.1,
                     weight32=rng.random() < 0.5, gate32=rng.random() < 0.5, sums=before == "none" or rng.random() < 0.8,
                     pitch=cols + rng.choice((0, 0, 0, 8, 3)))
    rows, outs, ins = _log(rng, 1, 16384), _log(rng, 64, 5120), _log(rng, 64, 5120)
    if rng.random() < 0.75:
        ins, outs = (ins + 63) // 64 * 64, (outs + 63) // 64 * 64
    rank = rng.choice((8, 16, 16, 24, 32, 48, 64, 128))
    if rows > 512 or rng.random() < 0.2:
        rank, requests = min(rank, 64), min(rows, _log(rng, 1, 48))
    else:
        requests = rows
    return _adapters(rows, outs, ins, rank, _log(rng, 1, 64 if rows <= 512 else 32), requests=requests, bare=rng.choice((0.0, 0.1, 0.25)),
                     out32=rng.random() < 0.2, bias=rng.random() < 0.5, residual=rng.random() < 0.5, act=rng.choice(_ACTS),
                     pitch=ins + rng.choice((0, 0, 0, 8, 3)))


# ---- inputs

def _type(wide):
    return torch.float32 if wide else torch.bfloat16


def _norm_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    R, M = case["rows"], case["cols"]

    def normal(shape, std, wide):
        return torch.empty(shape, dtype=_type(wide), device="cuda").normal_(0.0, std, generator=gen)

    # a block's results, and a stream that has grown over many layers, some of its features far beyond the others
    block = normal((R, case["pitch"]), 1.0, case["block32"])[:, :M]
    residual = None
    if case["residual"]:
        residual = normal((R, M), 4.0, case["stream32"])
        residual[:, torch.empty(M, device="cuda").uniform_(generator=gen) < 0.01] *= 16.0
    gate = None
    if case["gate"] != "none":
        gate = normal((R,) if case["gate"] == "row" else (R, M), 1.5, case["gate32"])

    def weights(there):
        return (normal((M,), 0.3, True) + (1.0 - case["offset"])).to(_type(case["weight32"])) if there else None

    def biases(there):
        return normal((M,), 0.1, case["weight32"]) if there and case["biases"] else None

    after, before = case["weights"], case["before"] != "none"
    return block, residual, gate, weights(after), biases(after), weights(before), biases(before)


def _popularity(n):
    """Shares of the requests that n adapters have: few of them have most."""
    p = 1.0 / np.arange(1, n + 1)
    return p / p.sum()


def _index(case, seed):
    """The adapter of every row: requests one behind another, each with an adapter or without one."""
    rng = np.random.default_rng(seed)
    R, n = case["rows"], case["requests"]
    adapter = rng.permutation(case["adapters"])[rng.choice(case["adapters"], size=n, p=_popularity(case["adapters"]))]
    adapter[rng.random(n) < case["bare"]] = -1
    lengths = np.ones(n, dtype=np.int64)
    if n < R:
        share = rng.lognormal(0.0, 1.0, size=n)
        lengths += np.floor((R - n) * share / share.sum()).astype(np.int64)
        lengths[-1] += R - lengths.sum()
    return np.repeat(adapter, lengths).astype(np.int32)


def _adapter_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    R, N, K, r, n = case["rows"], case["outs"], case["ins"], case["rank"], case["adapters"]

    def normal(shape, std, wide=False):
        return torch.empty(shape, dtype=_type(wide), device="cuda").normal_(0.0, std, generator=gen)

    x = normal((R, case["pitch"]), 1.0)[:, :K]
    weight = normal((N, K), 0.02)
    index = torch.from_numpy(_index(case, seed)).cuda()
    down, up = normal((n, r, K), 0.02), normal((n, N, r), 0.02)
    scale = torch.empty(n, dtype=torch.float32, device="cuda").uniform_(0.5, 4.0, generator=gen)
    bias = normal((N,), 0.1, True) if case["bias"] else None
    residual = normal((R, N), 1.0, case["out32"]) if case["residual"] else None
    return x, weight, index, down, up, scale, bias, residual


def prepare(case, seed):
    if case["op"] == "norm":
        args = _norm_inputs(case, seed)
        shape = (case["rows"], case["cols"])
        state = dict(case=case, args=args, sum=torch.empty(shape, dtype=_type(case["stream32"]), device="cuda") if case["sums"] else None,
                     out=torch.empty(shape, dtype=_type(case["out32"]), device="cuda") if case["before"] != "none" else None)
        if own:
            import paper_2512_21487_amd as moe_ep
            state["call"] = moe_ep.norm
            state["rule"] = moe_ep.NormConfig(
                features=case["cols"], norm_after=_NORMS.index(case["after"]), norm_before=_NORMS.index(case["before"]),
                block_type=int(case["block32"]), stream_type=int(case["stream32"]), out_type=int(case["out32"]), weight_type=int(case["weight32"]),
                gate_type=int(case["gate32"]), gate_form=_FORMS.index(case["form"]), gate_per_row=int(case["gate"] == "row"), eps=_EPS,
                block_scale=case["block_scale"], residual_scale=case["residual_scale"], weight_offset=case["offset"], block_stride=case["pitch"])
        return state
    args = _adapter_inputs(case, seed)
    state = dict(case=case, args=args, out=torch.empty((case["rows"], case["outs"]), dtype=_type(case["out32"]), device="cuda"))
    if own:
        import paper_2512_21487_amd as moe_ep
        state["call"] = moe_ep.linear_adapters
        state["rule"] = moe_ep.LinearConfig(in_features=case["ins"], out_features=case["outs"], weight_type=moe_ep.BF16,
                                            out_type=moe_ep.F32 if case["out32"] else moe_ep.BF16, activation=_ACTS.index(case["act"]),
                                            x_stride=case["pitch"])
        state["adapters"] = moe_ep.AdapterConfig(n_adapters=case["adapters"], rank=case["rank"])
        state["workspace"] = torch.empty(moe_ep.linear_adapters_workspace_bytes(state["rule"], state["adapters"], case["rows"]),
                                         dtype=torch.uint8, device="cuda")
    return state


# ---- the plain forms

def _plain_norm(kind, x, weight, bias, offset):
    if kind == "layer":
        x = x - x.mean(dim=1, keepdim=True)
    if kind != "none":
        x = x * torch.rsqrt((x * x).mean(dim=1, keepdim=True) + _EPS)
    if weight is not None:
        x = x * (weight.float() + offset)
    return x if bias is None else x + bias.float()


def _norm_plain(case, block, residual, gate, after_w, after_b, before_w, before_b):
    z = _plain_norm(case["after"], block.float(), after_w, after_b, case["offset"])
    if gate is not None:
        g = gate.float()
        g = g if case["form"] == "as_is" else 1.0 / (1.0 + torch.exp(-g)) if case["form"] == "sigmoid" else g / (1.0 + torch.exp(-g))
        z = z * (g[:, None] if case["gate"] == "row" else g)
    h = case["block_scale"] * z
    if residual is not None:
        h = h + case["residual_scale"] * residual.float()
    got = {"sum": h.to(_type(case["stream32"]))} if case["sums"] else {}
    if case["before"] != "none":
        got["out"] = _plain_norm(case["before"], h, before_w, before_b, case["offset"]).to(_type(case["out32"]))
    return got


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


def _adapters_plain(case, x, weight, index, down, up, scale, bias, residual):
    """All adapters' small products at once, those of a row's own kept."""
    R, N, K, r, n = case["rows"], case["outs"], case["ins"], case["rank"], case["adapters"]
    x = x.float()
    mine = (index[:, None] == torch.arange(n, device=index.device)[None, :]).float() * scale[None, :]
    low = (x @ down.float().view(n * r, K).t()).view(R, n, r) * mine[:, :, None]
    y = x @ weight.float().t() + low.view(R, n * r) @ up.float().permute(0, 2, 1).reshape(n * r, N)
    if bias is not None:
        y = y + bias
    y = _act(case["act"], y)
    if residual is not None:
        y = y + residual.float()
    return y.to(_type(case["out32"]))


def run(state):
    case = state["case"]
    if case["op"] == "norm":
        if not own:
            return _norm_plain(case, *state["args"])
        block, residual, gate, after_w, after_b, before_w, before_b = state["args"]
        state["call"](state["rule"], block, residual, gate, after_w, after_b, before_w, before_b, sum=state["sum"], out=state["out"])
        return {name: state[name] for name in ("sum", "out") if state[name] is not None}
    if not own:
        return {"out": _adapters_plain(case, *state["args"])}
    x, weight, index, down, up, scale, bias, residual = state["args"]
    state["call"](state["rule"], state["adapters"], x, weight, index, down, up, scale, bias, residual, out=state["out"], workspace=state["workspace"])
    return {"out": state["out"]}


def work(case):
    if case["op"] == "norm":
        R, M = case["rows"], case["cols"]

        def size(name):
            return 4.0 if case[name] else 2.0

        element = size("block32") + (size("stream32") if case["residual"] else 0.0) + (size("stream32") if case["sums"] else 0.0)
        element += (size("out32") if case["before"] != "none" else 0.0) + (size("gate32") if case["gate"] == "element" else 0.0)
        vectors = (int(case["weights"]) + int(case["before"] != "none")) * (2 if case["biases"] else 1)
        norms = (case["after"] != "none") + (case["before"] != "none")
        return {"bytes": R * M * element + vectors * M * size("weight32") + (R * size("gate32") if case["gate"] == "row" else 0.0),
                "flops": R * M * (6.0 * norms + 4.0)}
    R, N, K, r = case["rows"], case["outs"], case["ins"], case["rank"]
    share = 1.0 - case["bare"]
    used = float((1.0 - (1.0 - share * _popularity(case["adapters"])) ** case["requests"]).sum())   # adapters that some request has
    size = 4 if case["out32"] else 2
    read = 2 * R * K + 2 * N * K + 4 * R + used * (2 * r * (K + N) + 4) + (4 * N if case["bias"] else 0) + (size * R * N if case["residual"] else 0)
    return {"bytes": float(read + size * R * N), "flops": 2.0 * R * N * K + 2.0 * R * share * r * (K + N)}


# ---- from the definitions, in 64 bits

def _exact_norm(kind, v, weight, bias, offset):
    if kind != "none":
        second, first = torch.var_mean(v, dim=1, keepdim=True, correction=0)
        centred = v - first if kind == "layer" else v
        power = second if kind == "layer" else second + first ** 2
        v = centred / torch.sqrt(power + _EPS)
    gain = offset + weight.double() if weight is not None else torch.ones((), dtype=torch.float64, device=v.device)
    return torch.addcmul(torch.zeros_like(v) if bias is None else bias.double().expand_as(v), v, gain.expand_as(v))


def exact(case, seed):
    if case["op"] == "norm":
        block, residual, gate, after_w, after_b, before_w, before_b = _norm_inputs(case, seed)
        h = case["block_scale"] * _exact_norm(case["after"], block.double(), after_w, after_b, case["offset"])
        if gate is not None:
            g = gate.double().view(case["rows"], -1)
            h = h * {"as_is": lambda t: t, "sigmoid": torch.sigmoid, "silu": torch.nn.functional.silu}[case["form"]](g)
        if residual is not None:
            h = torch.add(h, residual.double(), alpha=case["residual_scale"])
        got = {"sum": h} if case["sums"] else {}
        if case["before"] != "none":
            got["out"] = _exact_norm(case["before"], h, before_w, before_b, case["offset"])
        return got
    x, weight, index, down, up, scale, bias, residual = _adapter_inputs(case, seed)
    x = x.double()
    z = torch.matmul(x, weight.double().t())
    of_row = _index(case, seed)
    for a in np.unique(of_row[of_row >= 0]).tolist():
        rows = torch.from_numpy(np.flatnonzero(of_row == a)).cuda()
        z[rows] += scale[a].double() * torch.matmul(torch.matmul(x[rows], down[a].double().t()), up[a].double().t())
    z = z if bias is None else z + bias.double()
    y = {"none": lambda v: v, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu,
         "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}[case["act"]](z)
    return {"out": y if residual is None else y + residual.double()}
