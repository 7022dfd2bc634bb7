"""Norms, projections with adapters, gate, routing and experts one behind another, as a decoder's step uses them."""
import numpy as np
import pytest

from test_gpu_routed_layer import layer
from workloads import make_inputs, tiny_workload

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HIDDEN, INNER, RANK, ADAPTERS, TOP_K = 256, 192, 16, 5, 4


class Block:
    """stream -> norm -> projection with adapters -> projection with adapters onto the stream -> norm -> gate -> route -> experts -> norm, gate and residual."""

    def __init__(self, T, seed=1):
        import paper_2512_21487_amd as pkg
        self.T = T
        self.wl = tiny_workload(name="block", n_tokens=T, hidden=HIDDEN, inter=192, n_experts=32, local_begin=0, n_local=32, top_k=TOP_K, n_shared=1, shared_inter=128)
        self.inp = make_inputs(self.wl, seed=seed)
        gen = torch.Generator(device="cuda").manual_seed(seed + T)
        n = lambda *shape, std=1.0, dtype=torch.bfloat16: torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=gen).to(dtype)
        e = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype, device="cuda")
        self.stream, self.index = n(T, HIDDEN, dtype=torch.float32), torch.randint(-1, ADAPTERS, (T,), generator=gen, device="cuda", dtype=torch.int32)
        self.g = [1.0 + n(HIDDEN, std=0.1, dtype=torch.float32) for _ in range(3)]
        self.w = [n(INNER, HIDDEN, std=0.06), n(HIDDEN, INNER, std=0.07)]
        self.down = [n(ADAPTERS, RANK, HIDDEN, std=0.06), n(ADAPTERS, RANK, INNER, std=0.07)]
        self.up = [n(ADAPTERS, INNER, RANK, std=0.1), n(ADAPTERS, HIDDEN, RANK, std=0.1)]
        self.scale = torch.empty(ADAPTERS, device="cuda").uniform_(0.5, 2.0, generator=gen)
        self.w_gate, self.w_close = n(32, HIDDEN, std=0.06, dtype=torch.float32), n(1, HIDDEN, std=0.06)
        self.x, self.mid, self.attn, self.h, self.y = e(T, HIDDEN), e(T, INNER), e(T, HIDDEN), e(T, HIDDEN), e(T, HIDDEN)
        self.h32, self.out = e(T, HIDDEN, dtype=torch.float32), e(T, HIDDEN, dtype=torch.float32)
        self.scores, self.close = e(T, 32, dtype=torch.float32), e(T, 1, dtype=torch.float32)
        self.idx, self.wt = e(T, TOP_K, dtype=torch.int32), e(T, TOP_K, dtype=torch.float32)
        put = lambda a: torch.from_numpy(a.view(np.int16)).cuda()
        self.routed, self.shared = put(self.inp["routed_w"]), put(self.inp["shared_w"])
        self.ctx = pkg.MoeEp(hidden=HIDDEN, inter=192, n_experts=32, local_begin=0, n_local=32, n_shared=1, shared_inter=128, max_tokens=T, max_top_k=TOP_K, max_chunks=1)
        self.adapters = pkg.AdapterConfig(n_adapters=ADAPTERS, rank=RANK)
        self.rule = pkg.Routing(n_experts=32, top_k=TOP_K, renormalise=1, score=pkg.SCORE_SIGMOID, score_type=pkg.F32)
        self.ctx.set_routing(self.rule)
        self.cfg = [pkg.LinearConfig(in_features=HIDDEN, out_features=INNER, activation=pkg.ACT_SILU), pkg.LinearConfig(in_features=INNER, out_features=HIDDEN)]
        # one workspace for both: they follow one another
        self.workspace = torch.empty(max(pkg.linear_adapters_workspace_bytes(c, self.adapters, T) for c in self.cfg), dtype=torch.uint8, device="cuda")
        self.norm1 = pkg.NormConfig(features=HIDDEN, norm_before=pkg.NORM_RMS, block_type=pkg.F32, weight_type=pkg.F32)
        self.norm2 = pkg.NormConfig(features=HIDDEN, norm_after=pkg.NORM_RMS, norm_before=pkg.NORM_RMS, stream_type=pkg.F32, weight_type=pkg.F32)
        self.norm3 = pkg.NormConfig(features=HIDDEN, stream_type=pkg.F32, gate_type=pkg.F32, gate_form=pkg.GATE_SIGMOID, gate_per_row=1, residual_scale=0.5)
        self.gate = pkg.LinearConfig(in_features=HIDDEN, out_features=32, weight_type=pkg.F32, out_type=pkg.F32)
        self.closing = pkg.LinearConfig(in_features=HIDDEN, out_features=1, out_type=pkg.F32)

    def run(self):
        import paper_2512_21487_amd as pkg
        pkg.norm(self.norm1, self.stream, before_weight=self.g[0], out=self.x)
        pkg.linear_adapters(self.cfg[0], self.adapters, self.x, self.w[0], self.index, self.down[0], self.up[0], self.scale, out=self.mid, workspace=self.workspace)
        pkg.linear_adapters(self.cfg[1], self.adapters, self.mid, self.w[1], self.index, self.down[1], self.up[1], self.scale, out=self.attn, workspace=self.workspace)
        pkg.norm(self.norm2, self.attn, self.stream, after_weight=self.g[1], before_weight=self.g[2], sum=self.h32, out=self.h)
        pkg.linear(self.gate, self.h, self.w_gate, out=self.scores)
        pkg.route(self.rule, self.scores, idx=self.idx, w=self.wt)
        pkg.linear(self.closing, self.h, self.w_close, out=self.close)
        self.ctx.forward(self.h, self.scores, self.routed, self.shared, TOP_K, 1, 0, n_tokens=self.T, out=self.y)
        pkg.norm(self.norm3, self.y, self.h32, self.close, sum=self.out)

    def check(self):
        """Every step from what the one in front of it wrote, in float64."""
        torch.cuda.synchronize()
        near = lambda got, want, tol: bool(((got.double() - want).abs() <= tol * want.abs().clamp(min=float(want.square().mean().sqrt()))).all())
        rms = lambda v, g: v / torch.sqrt(v.square().mean(dim=1, keepdim=True) + 1e-6) * g.double()
        half = 2.0 ** -8                                   # a rounding to bf16, and fp32 steps that are far below it
        s = self.stream.double()
        assert near(self.x, rms(s, self.g[0]), 1.01 * half)

        def projected(x, i):
            z = x.double() @ self.w[i].double().t()
            for a in range(ADAPTERS):
                rows = self.index == a
                z[rows] += float(self.scale[a]) * (x[rows].double() @ self.down[i][a].double().t()) @ self.up[i][a].double().t()
            return z

        z = projected(self.x, 0)
        assert near(self.mid, z * torch.sigmoid(z), 1.01 * half) and near(self.attn, projected(self.mid, 1), 1.01 * half)
        h = s + rms(self.attn.double(), self.g[1])
        assert near(self.h32, h, 1e-5) and near(self.h, rms(h, self.g[2]), 1.01 * half)
        assert near(self.scores, self.h.double() @ self.w_gate.double().t(), 1e-5)
        assert near(self.close, self.h.double() @ self.w_close.double().t(), 1e-5)
        idx, w = self.idx.cpu().numpy(), self.wt.cpu().numpy().astype(np.float64)
        want = layer(self.wl, dict(self.inp, tokens=self.h.view(torch.int16).cpu().numpy().view(np.uint16)), idx, w)
        assert near(self.y, torch.from_numpy(want).cuda(), 2e-2)   # the bound of every full-path comparison
        assert near(self.out, 0.5 * self.h32.double() + torch.sigmoid(self.close.double()) * self.y.double(), 1e-5)


@pytest.mark.parametrize("T", [1, 4, 33, 200, 700, 900])
def test_a_block(T):
    b = Block(T)
    b.run()
    b.check()


@pytest.mark.parametrize("T", [1, 33, 900])
def test_a_block_in_a_graph(T):
    b = Block(T)
    b.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.run()
    other = Block(T, seed=7)
    for source in (None, other, None):
        if source is not None:
            b.stream.copy_(source.stream), b.index.copy_(source.index)
        b.out.zero_(), b.attn.zero_(), b.mid.zero_()
        graph.replay()
        b.check()
        got = b.out.clone()
        b.run()
        torch.cuda.synchronize()
        assert torch.equal(got, b.out)
