"""moe_ep_linear against the product in float64."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")


def act(name, z):
    if name == "relu":
        return z.clamp(min=0.0)
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return 0.5 * z * torch.erfc(-z * math.sqrt(0.5))
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


class Case:
    def __init__(self, R, N, K, *, w32=False, out32=False, bias=False, residual=False, name="none", pads=(0, 0, 0, 0), shifts=(0, 0, 0, 0), seed=0):
        """pads: elements between rows of x, weight, residual, out; shifts: elements before their first."""
        import paper_2512_21487_amd as pkg
        gen = torch.Generator(device="cuda").manual_seed(seed + R + 7 * N + 13 * K)
        ot = torch.float32 if out32 else torch.bfloat16

        def rows(n, cols, pad, shift, dtype, std, fill=None):
            flat = torch.empty(shift + n * (cols + pad), dtype=dtype, device="cuda")
            flat.normal_(0.0, std, generator=gen) if fill is None else flat.fill_(fill)
            return flat, flat[shift:].view(n, cols + pad)[:, :cols]

        # what lies beside the operands is no number: nothing of it may reach a result
        def operand(n, cols, pad, shift, dtype, std):
            flat, view = rows(n, cols, pad, shift, dtype, std, float("nan"))
            view.copy_(torch.empty((n, cols), dtype=dtype, device="cuda").normal_(0.0, std, generator=gen))
            return view

        self.x = operand(R, K, pads[0], shifts[0], torch.bfloat16, 1.0)
        self.w = operand(N, K, pads[1], shifts[1], torch.float32 if w32 else torch.bfloat16, 0.5 / math.sqrt(K) * 2)
        self.b = torch.empty(N, device="cuda").normal_(generator=gen) if bias else None
        self.r = operand(R, N, pads[2], shifts[2], ot, 1.0) if residual else None
        self.flat, self.out = rows(R, N, pads[3], shifts[3], ot, 0.0, 3.0)
        self.name, self.out32, self.R, self.N, self.K = name, out32, R, N, K
        self.cfg = pkg.LinearConfig(in_features=K, out_features=N, weight_type=int(w32), out_type=int(out32), activation=ACTS.index(name),
                                    x_stride=K + pads[0], weight_stride=K + pads[1], residual_stride=N + pads[2], out_stride=N + pads[3])

    def run(self, stream=None):
        import paper_2512_21487_amd as pkg
        pkg.linear(self.cfg, self.x, self.w, self.b, self.r, out=self.out, n_rows=self.R, stream=stream)

    def want(self):
        x, w = self.x.double(), self.w.double()
        z = x @ w.t()
        size = x.abs() @ w.abs().t()
        if self.b is not None:
            z, size = z + self.b.double(), size + self.b.double().abs()
        y = act(self.name, z)
        # K fp32 sums, each off by half a step of what has been added up; an activation's slope is below 1.13, its own fp32 steps add a
        # few of the result's size (gelu's erf: of z's) and of exp's argument; then the residual's sum and the rounding of the result
        bound = 1.13 * (self.K + 8) * 2.0 ** -24 * size + 16 * 2.0 ** -24 * z.abs() * (1 + z.abs())
        if self.r is not None:
            y = y + self.r.double()
        return y, bound + (2.0 ** -23 if self.out32 else 2.0 ** -8) * (y.abs() + bound) + 1e-37

    def check(self):
        torch.cuda.synchronize()
        y, bound = self.want()
        got = self.out.double()
        off = (got - y).abs()
        assert bool(torch.isfinite(got).all())
        worst = float((off / bound).max())
        assert worst <= 1.0, f"{worst} times the bound"
        # nothing but the results was written
        whole = torch.full_like(self.flat, 3.0)
        start = self.out.storage_offset()
        whole[start:].view(self.R, -1)[:, :self.N] = self.out
        assert torch.equal(whole, self.flat)


@pytest.mark.parametrize("R", [1, 2, 15, 16, 17, 33, 64, 65, 200])
@pytest.mark.parametrize("N,K", [(1, 1), (3, 7), (16, 64), (17, 63), (61, 129), (160, 512), (128, 1000), (257, 2049)])
@pytest.mark.parametrize("w32", [False, True])
def test_sizes(R, N, K, w32):
    c = Case(R, N, K, w32=w32, out32=w32, bias=R % 2 == 0)
    c.run()
    c.check()


@pytest.mark.parametrize("R,N,K", [(127, 128, 64), (128, 384, 192), (129, 640, 128), (256, 256, 512), (257, 1000, 264), (700, 513, 1408), (1025, 1544, 328),
                                   (2048, 2048, 1088), (4100, 1288, 72), (5000, 520, 8)])
@pytest.mark.parametrize("name,out32,residual", [("none", False, True), ("silu", True, False), ("gelu", False, False)])
def test_large_products(R, N, K, name, out32, residual):
    c = Case(R, N, K, out32=out32, bias=True, residual=residual, name=name)
    c.run()
    c.check()


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("R,N,K", [(5, 96, 200), (300, 512, 256)])
@pytest.mark.parametrize("w32", [False, True])
@pytest.mark.parametrize("out32", [False, True])
@pytest.mark.parametrize("bias,residual", [(False, False), (True, False), (False, True), (True, True)])
def test_epilogues(name, R, N, K, w32, out32, bias, residual):
    c = Case(R, N, K, w32=w32, out32=out32, bias=bias, residual=residual, name=name)
    c.run()
    c.check()


@pytest.mark.parametrize("pads", [(0, 0, 0, 0), (8, 8, 8, 8), (1, 0, 0, 0), (0, 3, 0, 0), (0, 0, 5, 0), (0, 0, 0, 1), (4, 12, 20, 36)])
@pytest.mark.parametrize("shifts", [(0, 0, 0, 0), (8, 8, 8, 8), (1, 1, 1, 1), (4, 2, 4, 2)])
@pytest.mark.parametrize("R,N,K", [(7, 130, 192), (520, 520, 200), (520, 520, 203)])
@pytest.mark.parametrize("w32,out32", [(False, False), (True, True), (False, True)])
def test_strides_and_alignments(pads, shifts, R, N, K, w32, out32):
    c = Case(R, N, K, w32=w32, out32=out32, bias=True, residual=True, name="silu", pads=pads, shifts=shifts)
    c.run()
    c.check()


@pytest.mark.parametrize("R,N,K,out32", [(9, 200, 128, False), (300, 512, 256, False), (300, 512, 256, True), (33, 61, 70, True)])
def test_residual_in_place(R, N, K, out32):
    c = Case(R, N, K, out32=out32, residual=True, bias=True)
    apart = Case(R, N, K, out32=out32, residual=True, bias=True)
    apart.run()
    c.out.copy_(c.r)
    c.r = c.out
    c.run()
    torch.cuda.synchronize()
    assert torch.equal(c.out, apart.out)


def test_fp32_weights_count_to_the_last_bit():
    """Weights that differ in their last bits only, and a result that is their difference."""
    import paper_2512_21487_amd as pkg
    K = 64
    base = torch.full((16, K), 1.0, device="cuda")
    w = base.clone()
    w[:, 1::2] = -(1.0 + 2.0 ** -23)
    x = torch.ones((4, K), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros((4, 16), device="cuda")
    pkg.linear(pkg.LinearConfig(in_features=K, out_features=16, weight_type=pkg.F32, out_type=pkg.F32), x, w, out=out)
    torch.cuda.synchronize()
    assert bool((out == -(K // 2) * 2.0 ** -23).all())


@pytest.mark.parametrize("R", [3, 300])
def test_numbers_that_are_none(R):
    """Infinities and NaN of x stay in their rows, of the residual in their places; a relu keeps a NaN."""
    c = Case(R, 260, 128, residual=True, name="relu")
    c.x[1, 5], c.x[2, 7] = float("nan"), float("inf")
    c.r[0, 3], c.r[0, 4] = float("inf"), float("nan")
    c.run()
    torch.cuda.synchronize()
    o = c.out
    assert bool(torch.isnan(o[1]).all())
    assert not bool(torch.isfinite(o[2][(c.w[:, 7] > 0)]).any())
    assert bool(torch.isinf(o[0, 3])) and bool(torch.isnan(o[0, 4]))
    rest = torch.cat([o[0, :3], o[0, 5:]] + [v for v in o[3:]])
    assert bool(torch.isfinite(rest).all())


def test_far_rows():
    """Rows further apart than 32 bits of bytes reach from the first to the last."""
    import paper_2512_21487_amd as pkg
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of GPU memory")
    R, N, K, stride = 1100, 300, 128, 1 << 22
    for w32 in (False, True):
        x = torch.empty(R * stride, dtype=torch.bfloat16, device="cuda").view(R, stride)[:, :K]
        x.normal_()
        w = torch.empty((N, K), dtype=torch.float32 if w32 else torch.bfloat16, device="cuda").normal_(0.0, 0.1)
        out = torch.empty(R * stride, dtype=torch.float32, device="cuda").view(R, stride)[:, :N]
        cfg = pkg.LinearConfig(in_features=K, out_features=N, weight_type=int(w32), out_type=pkg.F32, x_stride=stride, out_stride=stride)
        pkg.linear(cfg, x, w, out=out)
        torch.cuda.synchronize()
        want = x.double() @ w.double().t()
        bound = (K + 8) * 2.0 ** -24 * (x.double().abs() @ w.double().abs().t())
        assert bool(((out.double() - want).abs() <= bound).all())
        del x, out
        torch.cuda.empty_cache()


@pytest.mark.parametrize("R,N,K,w32", [(1, 160, 2048, True), (33, 200, 1408, False), (700, 1032, 520, False), (400, 128, 1024, True)])
def test_streams_graphs_and_repeats(R, N, K, w32):
    c = [Case(R, N, K, w32=w32, out32=True, bias=True, residual=True, name="silu", seed=i) for i in range(2)]
    for v in c:
        v.run()
    torch.cuda.synchronize()
    want = [v.out.clone() for v in c]
    side = [torch.cuda.Stream() for _ in range(2)]
    for v in c:
        v.out.fill_(0.0)
    torch.cuda.synchronize()
    for _ in range(5):                               # two streams at once
        for st, v in zip(side, c):
            v.run(st.cuda_stream)
    torch.cuda.synchronize()
    for v, y in zip(c, want):
        assert torch.equal(v.out, y)
    held = c[0].x.clone()
    both = [held, c[1].x.clone()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c[0].run()
    for _ in range(3):
        c[0].out.fill_(0.0)
        c[1].run()                                   # eager work between the replays
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c[0].out, want[0]) and torch.equal(c[1].out, want[1])


def test_buffers_that_are_too_small_or_elsewhere():
    import paper_2512_21487_amd as pkg
    cfg = pkg.LinearConfig(in_features=64, out_features=32)
    x, w = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((32, 64), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros((4, 32), dtype=torch.bfloat16, device="cuda")
    for bad in (dict(x=x[:, :60]), dict(weight=w[:31]), dict(out=out[:3]), dict(x=x.t()), dict(bias=torch.zeros(31, device="cuda")),
                dict(residual=torch.zeros((4, 32), device="cuda"))):
        with pytest.raises(ValueError):
            pkg.linear(cfg, **dict(dict(x=x, weight=w, out=out, n_rows=4), **bad))
    host = np.zeros((4, 64), np.uint16)
    with pytest.raises(pkg.MoeEpError, match="x "):
        pkg.linear(cfg, host.ctypes.data, w, out=out, n_rows=4)
    before = torch.cuda.current_device()
    with pytest.raises(pkg.MoeEpError) as ei:
        pkg.linear(pkg.LinearConfig(in_features=64, out_features=32, device=63), x, w, out=out)
    assert ei.value.code == -3 and torch.cuda.current_device() == before
    pkg.linear(cfg, x, w, out=out)
    torch.cuda.synchronize()


@pytest.mark.parametrize("R,N,K", [(1531, 1409, 2049), (3000, 839, 182), (4200, 4100, 65), (1300, 1300, 71), (4097, 4097, 129), (400, 65, 4100)])
@pytest.mark.parametrize("name,out32,residual", [("none", False, True), ("gelu_tanh", True, False)])
def test_large_products_that_are_not_on_16_bytes(R, N, K, name, out32, residual):
    c = Case(R, N, K, out32=out32, bias=True, residual=residual, name=name, pads=(3, 0, 1, 5), shifts=(1, 2, 0, 0))
    c.run()
    c.check()


@pytest.mark.parametrize("R,N,K", [(4096, 128, 4096), (2100, 60, 3000), (700, 512, 2304), (16384, 160, 640), (64, 128, 5120)])
def test_gates_of_many_tokens(R, N, K):
    c = Case(R, N, K, w32=True, out32=True, bias=True)
    c.run()
    c.check()


def test_columns_of_one_buffer():
    import paper_2512_21487_amd as pkg
    R, N, K = 300, 96, 128
    buf = torch.zeros((R, 384), dtype=torch.bfloat16, device="cuda")
    buf[:, :K].normal_()
    w = torch.empty((N, K), dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.1)
    apart = torch.zeros((R, N), dtype=torch.bfloat16, device="cuda")
    pkg.linear(pkg.LinearConfig(in_features=K, out_features=N, x_stride=384), buf[:, :K], w, out=apart)
    pkg.linear(pkg.LinearConfig(in_features=K, out_features=N, x_stride=384, out_stride=384), buf[:, :K], w, out=buf[:, 200:200 + N])
    torch.cuda.synchronize()
    assert torch.equal(buf[:, 200:200 + N], apart) and not bool(buf[:, K:200].any()) and not bool(buf[:, 200 + N:].any())


def test_more_rows_than_a_grid_has_rows_of_threads():
    """2^32 threads are a grid dimension's; a workgroup of 256 has 64 rows of one column."""
    import paper_2512_21487_amd as pkg
    R = 2 ** 30
    x = torch.randint(-8, 8, (R, 1), device="cuda", dtype=torch.int8).to(torch.bfloat16)
    out = torch.full((R + 1, 1), 77.0, dtype=torch.bfloat16, device="cuda")
    pkg.linear(pkg.LinearConfig(in_features=1, out_features=1), x, torch.tensor([[0.5]], device="cuda", dtype=torch.bfloat16), out=out, n_rows=R)
    torch.cuda.synchronize()
    assert torch.equal(out[:R], x * 0.5) and float(out[R]) == 77.0
