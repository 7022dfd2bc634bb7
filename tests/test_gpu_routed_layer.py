"""The layer by a routing rule (moe_ep_set_routing), and gate projection, routing and experts together."""
import numpy as np
import pytest

from helpers import dense_ffn, f64, rel_err_rows, split_expert
from test_gpu_route import by_rule, weight_bound
from workloads import bf16_bits_to_f32, f32_to_bf16_bits, make_inputs, tiny_workload

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def layer(wl, inp, idx, w):
    """The routed and shared experts of the local share in float64, for given experts and weights."""
    x = f64(inp["tokens"])
    out = np.zeros_like(x)
    for e in range(wl.n_local):
        y = dense_ffn(x, *split_expert(inp["routed_w"], e, wl.hidden, wl.inter))
        out += np.where(idx == wl.local_begin + e, w, 0.0).sum(axis=1)[:, None] * y
    for i in range(wl.n_shared):
        out += dense_ffn(x, *split_expert(inp["shared_w"], i, wl.hidden, wl.shared_inter))
    return out


RULES = {
    "sigmoid_groups": dict(k=6, groups=4, top_groups=2, top2=True, sigmoid=True, renorm=True, scale=2.5),
    "softmax_as_it_is": dict(k=4, groups=8, top_groups=3, renorm=False, scale=16.0),
    "softmax_plain": dict(k=8, renorm=True, scale=1.0),
}


def rule_of(pkg, E, how):
    return pkg.Routing(n_experts=E, top_k=how["k"], n_groups=how.get("groups", 0), top_groups=how.get("top_groups", 0), score=int(how.get("sigmoid", False)),
                       group_score=int(how.get("top2", False)), renormalise=int(how["renorm"]), scale=how["scale"], score_type=pkg.F32)


def case(T, how, shared=1, local=(3, 23)):
    wl = tiny_workload(name="rule", n_tokens=T, hidden=128, inter=192, n_experts=32, local_begin=local[0], n_local=local[1], top_k=how["k"], n_shared=shared,
                       shared_inter=128 if shared else 0)
    inp = make_inputs(wl, seed=91)
    lg = inp["gate_logits"]
    lg[T // 3] = -np.inf                     # padding
    lg[T // 2, 5:] = -np.inf                 # fewer experts than slots
    return wl, inp


@pytest.mark.parametrize("T", [1, 4, 5, 33, 64, 65, 400, 1500])
@pytest.mark.parametrize("name", sorted(RULES))
@pytest.mark.parametrize("with_bias", [False, True])
def test_layer_by_a_rule(T, name, with_bias):
    import gpu_util as g
    import paper_2512_21487_amd as pkg
    how = RULES[name]
    wl, inp = case(T, how)
    E = wl.n_experts
    bias = (0.1 * np.random.default_rng(4).standard_normal(E)).astype(np.float32) if with_bias else None
    on_gpu = torch.from_numpy(bias).cuda() if with_bias else None
    idx, w = by_rule(inp["gate_logits"].astype(np.float64), bias, None, **how)
    want = layer(wl, inp, idx, w)
    for pinned, r, order in ((False, 1, 0), (False, 3, 1), (True, 1, 0), (True, 2, 1)):
        ctx = g.make_ctx(wl, pinned=pinned)
        ctx.set_routing(rule_of(pkg, E, how), on_gpu)
        d = g.DeviceInputs(wl, inp, pinned=pinned)
        got = bf16_bits_to_f32(g.run_forward(ctx, wl, d, r=r, order=order))
        assert rel_err_rows(got, want) <= 2e-2           # the bound of every full-path comparison
        routing = ctx.get_routing(0)
        n = routing["idx"].shape[0]
        assert np.array_equal(routing["idx"], idx[:n])
        bound = weight_bound(inp["gate_logits"][np.isfinite(inp["gate_logits"])], how["k"])
        assert np.all(np.abs(routing["w"] - w[:n]) <= bound * w[:n] + 1e-37)
        assert np.array_equal(routing["pos"] >= 0, (idx[:n] >= wl.local_begin) & (idx[:n] < wl.local_begin + wl.n_local))
        if not pinned:
            dep = bf16_bits_to_f32(g.run_forward_dep(ctx, wl, d, r_1=2, r_2=2))
            assert rel_err_rows(dep, want) <= 2e-2
        ctx.destroy()


def test_without_shared_experts_a_padded_token_is_zero_and_no_rule_is_as_before():
    import gpu_util as g
    import paper_2512_21487_amd as pkg
    how = RULES["softmax_plain"]
    wl, inp = case(120, how, shared=0)
    ctx = g.make_ctx(wl)
    d = g.DeviceInputs(wl, inp)
    ctx.set_routing(rule_of(pkg, wl.n_experts, how))
    got = g.run_forward(ctx, wl, d)
    assert not got[40].any() and got[0].any()
    inp["gate_logits"] = make_inputs(wl, seed=91)["gate_logits"]
    d = g.DeviceInputs(wl, inp)
    by = g.run_forward(ctx, wl, d)
    ctx.set_routing(None)
    plain = g.run_forward(ctx, wl, d)
    fresh = g.make_ctx(wl)
    assert np.array_equal(plain, g.run_forward(fresh, wl, d))
    # the same rule by another kernel: the weights' last bits may differ
    assert rel_err_rows(bf16_bits_to_f32(by), bf16_bits_to_f32(plain).astype(np.float64)) <= 2.0 ** -7
    ctx.destroy()
    fresh.destroy()


def test_refusals():
    import gpu_util as g
    import paper_2512_21487_amd as pkg
    how = RULES["softmax_plain"]
    wl, inp = case(16, how)
    ctx = g.make_ctx(wl)
    good = rule_of(pkg, wl.n_experts, how)
    for name, value, word in (("n_experts", 16, "n_experts"), ("top_k", 9, "max_top_k"), ("score_type", pkg.BF16, "fp32"), ("score_stride", 40, "fp32"),
                              ("device", 1, "device"), ("scale", 0.0, "scale")):
        bad = rule_of(pkg, wl.n_experts, how)
        setattr(bad, name, value)
        with pytest.raises(pkg.MoeEpError, match=word):
            ctx.set_routing(bad)
    with pytest.raises(pkg.MoeEpError, match="rule"):
        ctx.set_routing(None, torch.zeros(wl.n_experts, device="cuda"))
    with pytest.raises(ValueError):
        ctx.set_routing(good, torch.zeros(wl.n_experts - 1, device="cuda"))
    with pytest.raises(pkg.MoeEpError, match="bias"):
        ctx.set_routing(good, np.zeros(wl.n_experts, np.float32).ctypes.data)
    ctx.set_routing(good)
    d = g.DeviceInputs(wl, inp)
    with pytest.raises(pkg.MoeEpError, match="rule"):
        ctx.forward(d.tokens, d.logits, d.routed, d.shared, 4, out=d.out)
    with pytest.raises(pkg.MoeEpError, match="rule"):
        ctx.forward_dep(d.tokens, d.logits, d.routed, d.shared, 4, out=d.out)
    ctx.destroy()


@pytest.mark.parametrize("T", [1, 37, 300])
def test_gate_projection_routing_and_experts_as_one_graph(T):
    """Scores from the tokens with fp32 gate weights, experts by a rule, the layer, and a projection of its output onto the residual stream; eager and replayed."""
    import gpu_util as g
    import paper_2512_21487_amd as pkg
    how = RULES["sigmoid_groups"]
    wl, inp = case(T, how)
    M, E = wl.hidden, wl.n_experts
    rng = np.random.default_rng(8)
    gate_w = (0.1 * rng.standard_normal((E, M))).astype(np.float32)
    bias = (0.05 * rng.standard_normal(E)).astype(np.float32)
    proj = f32_to_bf16_bits((rng.standard_normal((M, M)) / np.sqrt(M)).astype(np.float32))
    d = g.DeviceInputs(wl, inp)
    dev = lambda a: torch.from_numpy(a).cuda()
    gw, b, pw = dev(gate_w), dev(bias), dev(proj.view(np.int16))
    scores = torch.zeros((T, E), device="cuda")
    idx, w = torch.zeros((T, how["k"]), dtype=torch.int32, device="cuda"), torch.zeros((T, how["k"]), device="cuda")
    final = torch.zeros((T, M), device="cuda", dtype=torch.int16)
    rule = rule_of(pkg, E, how)
    gate = pkg.LinearConfig(in_features=M, out_features=E, weight_type=pkg.F32, out_type=pkg.F32)
    outp = pkg.LinearConfig(in_features=M, out_features=M)
    ctx = g.make_ctx(wl)
    ctx.set_routing(rule, b)

    def run():
        pkg.linear(gate, d.tokens, gw, out=scores)
        pkg.route(rule, scores, b, idx=idx, w=w)
        ctx.forward(d.tokens, scores, d.routed, d.shared, how["k"], out=d.out)
        pkg.linear(outp, d.out, pw, residual=d.tokens, out=final)

    run()
    torch.cuda.synchronize()
    s = scores.cpu().numpy()
    x = f64(inp["tokens"])
    size = np.abs(x) @ np.abs(gate_w.astype(np.float64)).T
    assert np.all(np.abs(s - x @ gate_w.astype(np.float64).T) <= (M + 8) * 2.0 ** -24 * size)
    ref_idx, ref_w = by_rule(s.astype(np.float64), bias, None, **how)
    assert np.array_equal(idx.cpu().numpy(), ref_idx)
    routing = ctx.get_routing(0)
    assert np.array_equal(routing["idx"], ref_idx) and np.array_equal(routing["w"], w.cpu().numpy())
    out = bf16_bits_to_f32(d.out.cpu().numpy().view(np.uint16)).astype(np.float64)
    assert rel_err_rows(out, layer(wl, inp, ref_idx, ref_w)) <= 2e-2
    want = out @ f64(proj).T + x
    got = bf16_bits_to_f32(final.cpu().numpy().view(np.uint16))
    assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + (M + 8) * 2.0 ** -23 * (np.abs(out) @ np.abs(f64(proj)).T + np.abs(x)))
    keep = [t.clone() for t in (scores, idx, w, d.out, final)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        for t in (scores, idx, w, d.out, final):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for t, k in zip((scores, idx, w, d.out, final), keep):
            assert torch.equal(t, k)
        run()                                # eager work between the replays
        torch.cuda.synchronize()
    ctx.destroy()
