"""moe_ep_linear_adapters against its formula in float64."""
import math

import numpy as np
import pytest

from linear_shapes import KERNELS, SHAPES, kernel_of
from test_gpu_linear import ACTS, Case, act

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

PATTERNS = ("one", "own", "random", "runs", "none", "some")


def index_of(pattern, R, n, seed=0):
    rng = np.random.default_rng(seed + R)
    if pattern == "one":
        return np.full(R, n - 1)
    if pattern == "own":
        return np.arange(R) % n
    if pattern == "random":
        return rng.integers(0, n, R)
    if pattern == "none":                                # no adapter, by every number that means none
        return rng.choice([-1, n, -2 ** 31, 2 ** 31 - 1, -n], R)
    if pattern == "runs":
        starts = np.sort(rng.integers(0, R + 1, 5))
        return rng.integers(-1, n, 6)[np.searchsorted(starts, np.arange(R), side="right")]
    return np.where(rng.random(R) < 0.3, rng.integers(0, n, R), rng.choice([-1, n, -2 ** 31, 2 ** 31 - 1], R))


class Adapted(Case):
    def __init__(self, R, N, K, rank, n, pattern="random", *, scaled=True, seed=0, **kw):
        import paper_2512_21487_amd as pkg
        super().__init__(R, N, K, seed=seed, **kw)
        gen = torch.Generator(device="cuda").manual_seed(seed + 3 * R + 5 * N + 11 * K + rank)

        def normal(*shape, std):
            return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, std, generator=gen)

        index = index_of(pattern, R, n, seed)
        self.rank, self.n = rank, n
        self.down, self.up = normal(n, rank, K, std=1.0 / math.sqrt(K)), normal(n, N, rank, std=1.0 / math.sqrt(rank))
        self.scale = torch.empty(n, device="cuda").uniform_(0.5, 2.0, generator=gen) if scaled else None
        # an adapter that no row has may be anything
        unused = np.setdiff1d(np.arange(n), index)
        if len(unused):
            self.down[unused] = float("nan")
            self.up[unused] = float("nan")
            if scaled:
                self.scale[unused] = float("nan")
        self.index = torch.from_numpy(index.astype(np.int32)).cuda()
        self.adapters = pkg.AdapterConfig(n_adapters=n, rank=rank)
        self.need = pkg.linear_adapters_workspace_bytes(self.cfg, self.adapters, R)
        self.workspace = torch.full((self.need + 256,), 0xFF, dtype=torch.uint8, device="cuda")   # bf16 and fp32 NaN, lists of -1

    def run(self, stream=None):
        import paper_2512_21487_amd as pkg
        pkg.linear_adapters(self.cfg, self.adapters, self.x, self.w, self.index, self.down, self.up, self.scale, self.b, self.r, out=self.out,
                            workspace=self.workspace[:self.need], n_rows=self.R, stream=stream)

    def want(self):
        u = 2.0 ** -24
        x, w = self.x.double(), self.w.double()
        z, size, off = x @ w.t(), x.abs() @ w.abs().t(), torch.zeros((self.R, self.N), dtype=torch.float64, device="cuda")
        # x A^T as bf16 numbers, 8 bits each: of a number in 1..2 less than 2^-7 is left of the first, half a step of that, 2^-16 at most, of two, 2^-24 of three
        cut = 2.0 ** -24 if self.out32 else 2.0 ** -16
        for a in np.unique(self.index.cpu().numpy()).tolist():
            if not 0 <= a < self.n:
                continue
            rows = (self.index == a).nonzero()[:, 0]
            A, B, s = self.down[a].double(), self.up[a].double(), 1.0 if self.scale is None else float(self.scale[a])
            low = x[rows] @ A.t() * s
            # x A^T: K fp32 sums and the scale; then what the parts leave of it
            dlow = ((self.K + 8) * u * (x[rows].abs() @ A.abs().t()) * s) + (cut + u) * low.abs()
            z[rows] += low @ B.t()
            size[rows] += (low.abs() + dlow) @ B.abs().t()
            off[rows] += dlow @ B.abs().t()
        if self.b is not None:
            z, size = z + self.b.double(), size + self.b.double().abs()
        y = act(self.name, z)
        # as of the product alone, with a reduction that is longer by an adapter's parts
        bound = 1.13 * ((self.K + 3 * self.rank + 8) * u * size + off) + 16 * u * z.abs() * (1 + z.abs())
        if self.r is not None:
            y = y + self.r.double()
        return y, bound + (2.0 ** -23 if self.out32 else 2.0 ** -8) * (y.abs() + bound) + 1e-37

    def check(self):
        super().check()
        assert bool((self.workspace[self.need:] == 0xFF).all())


@pytest.mark.parametrize("R", [1, 2, 15, 16, 17, 33, 64, 65, 200, 513])
@pytest.mark.parametrize("N,K", [(1, 1), (3, 7), (16, 64), (17, 63), (61, 129), (160, 512), (257, 2049)])
@pytest.mark.parametrize("rank,n", [(8, 1), (16, 7), (24, 3), (128, 5)])
def test_sizes(R, N, K, rank, n):
    c = Adapted(R, N, K, rank, n, PATTERNS[(R + N + rank) % len(PATTERNS)], out32=R % 2 == 0, bias=R % 3 == 0, scaled=K % 2 == 1)
    c.run()
    c.check()


@pytest.mark.parametrize("name,R,N,K", [(name, *s[:3]) for name in KERNELS for s in SHAPES[name] if not s[3]])
@pytest.mark.parametrize("pattern", PATTERNS)
def test_every_kernel(name, R, N, K, pattern):
    """Each kernel of the product with adapters: one for all rows, one a row, in any order, in runs that end inside tiles, none at all."""
    if torch.cuda.get_device_properties(0).multi_processor_count == 256:
        assert kernel_of(R, N, K) == name
    i = PATTERNS.index(pattern)
    for rank, n, out32, residual in ((16, 9, False, True), (48, 40, True, False)):
        c = Adapted(R, N, K, rank, n, pattern, out32=out32, bias=i % 2 == 0, residual=residual, name=ACTS[i % len(ACTS)], seed=i)
        c.run()
        c.check()


@pytest.mark.parametrize("name,R,N,K", [("staged 64x64", 1531, 1409, 136), ("staged 128x64", 3873, 2061, 72)])
@pytest.mark.parametrize("pattern", ["runs", "some"])
def test_operands_whose_first_row_alone_is_off_16_bytes(name, R, N, K, pattern):
    """They are not copied, and go through registers."""
    c = Adapted(R, N, K, 24, 9, pattern, bias=True, residual=True, name="silu", shifts=(1, 1, 0, 0))
    if torch.cuda.get_device_properties(0).multi_processor_count == 256:
        assert kernel_of(R, N, K, x=c.x.data_ptr(), w=c.w.data_ptr()) == name
    c.run()
    c.check()


@pytest.mark.parametrize("R,N,K", [(600, 1100, 129), (800, 1100, 129), (1531, 1409, 203), (4100, 700, 65), (2000, 2500, 71)])
@pytest.mark.parametrize("pads", [(0, 0, 0, 0), (3, 0, 0, 0), (0, 5, 0, 0), (7, 7, 3, 1)])
@pytest.mark.parametrize("even", [False, True])
def test_rows_that_are_copied(R, N, K, pads, even):
    """Rows that are not on 16 bytes come into tiles from copies: x, W or both, with and without elements behind the last one."""
    K = (K + 7) // 8 * 8 if even else K
    for shifts in ((0, 0, 0, 0), (1, 3, 0, 0)):
        c = Adapted(R, N, K, 16, 5, "runs", bias=True, residual=True, out32=even, pads=pads, shifts=shifts)
        c.run()
        c.check()


# up to 768 rows are grouped, beside the product on each of its kernels
GROUPED = {"rows 1x1": (5, 96, 200), "rows 4x2": (66, 16, 65), "split 16x16": (207, 151, 96), "split 32x16": (66, 707, 65), "split 64x16": (66, 1034, 65), "split 64x32": (65, 2051, 65),
           "split 64x32 by 4": (66, 8294, 65), "staged 128x64": (130, 32886, 65), "staged 64x64": (65, 12304, 65), "tiles 128x128": (67, 32395, 576),
           "tiles 192x256": (66, 2100, 72), "tiles 256x192": (193, 33747, 72), "tiles 256x256": (512, 24719, 128), "tiles 64x64": (300, 2046, 256)}


@pytest.mark.parametrize("name", sorted(GROUPED))
@pytest.mark.parametrize("pattern", ["random", "some", "own"])
def test_grouped_beside_every_kernel(name, pattern):
    R, N, K = GROUPED[name]
    if torch.cuda.get_device_properties(0).multi_processor_count == 256:
        assert kernel_of(R, N, K) == name
    for n, out32 in ((7, False), (300, True)):
        c = Adapted(R, N, K, 24, n, pattern, out32=out32, bias=True, residual=out32, name="gelu_tanh")
        c.run()
        c.check()


@pytest.mark.parametrize("R", [1, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 400, 449, 511, 512, 513, 600, 640, 703, 704, 767, 768, 769])
@pytest.mark.parametrize("n", [1, 2, 20, 1000])
def test_groups_of_every_number_of_rows(R, n):
    """Groups that are full, one row short or over, of rows in any order, on kernels of four, eight and sixteen wavefronts."""
    for N, K, pattern in ((48, 64, "random"), (2050, 72, "some"), (1100, 65, "runs"), (640, 192, "own")):
        c = Adapted(R, N, K, 8, n, pattern, residual=True)
        c.run()
        c.check()


@pytest.mark.parametrize("R,N,K", [(800, 448, 128), (1016, 256, 192), (5692, 128, 192), (2000, 299, 130), (600, 300, 72), (770, 260, 65)])
@pytest.mark.parametrize("pattern", ["runs", "some"])
def test_short_reductions_of_few_columns(R, N, K, pattern):
    c = Adapted(R, N, K, 16, 6, pattern, bias=True, residual=True, name="gelu")
    c.run()
    c.check()


@pytest.mark.parametrize("R,N,K,rank,n", [(111, 448, 2240, 128, 58), (64, 1536, 320, 64, 64), (40, 100, 520, 128, 40), (200, 190, 130, 128, 150)])
def test_many_groups_beside_a_small_product(R, N, K, rank, n):
    for pattern in ("own", "some"):
        c = Adapted(R, N, K, rank, n, pattern, residual=True)
        c.run()
        c.check()


@pytest.mark.parametrize("rank", [8, 16, 24, 32, 40, 56, 64, 72, 96, 120, 128])
@pytest.mark.parametrize("out32", [False, True])
@pytest.mark.parametrize("R,N,K", [(3, 40, 130), (70, 520, 320), (300, 640, 192), (700, 513, 136), (800, 513, 136)])
def test_ranks(rank, out32, R, N, K):
    c = Adapted(R, N, K, rank, 6, "runs" if rank % 16 else "random", out32=out32, residual=True)
    c.run()
    c.check()


@pytest.mark.parametrize("R", [769, 1100, 2048, 5000, 8200, 16384, 16500])
@pytest.mark.parametrize("rank", [8, 16, 24, 64, 72, 128])
@pytest.mark.parametrize("K", [63, 200])
def test_every_tile_of_x_a(R, rank, K):
    """x A^T of many rows, by each of its tiles: ranks that fill them or not, a reduction with and without a whole step, adapters that change inside tiles."""
    for pattern in ("runs", "some"):
        c = Adapted(R, 40, K, rank, 9, pattern, out32=rank == 24, bias=True)
        c.run()
        c.check()


@pytest.mark.parametrize("R", [256, 300, 768, 1100])
@pytest.mark.parametrize("N,K", [(2048, 512), (1544, 328)])
def test_an_adapter_for_every_row(R, N, K):
    c = Adapted(R, N, K, 8, R, "own")
    c.run()
    c.check()


@pytest.mark.parametrize("pads", [(8, 8, 8, 8), (1, 0, 0, 0), (0, 3, 0, 0), (0, 0, 5, 1), (4, 12, 20, 36)])
@pytest.mark.parametrize("shifts", [(0, 0, 0, 0), (1, 1, 1, 1), (4, 2, 4, 2)])
@pytest.mark.parametrize("R,N,K", [(7, 130, 192), (520, 520, 200), (520, 520, 203), (780, 520, 203)])
@pytest.mark.parametrize("out32", [False, True])
def test_strides_and_alignments(pads, shifts, R, N, K, out32):
    c = Adapted(R, N, K, 16, 4, "some", out32=out32, bias=True, residual=True, name="silu", pads=pads, shifts=shifts)
    c.run()
    c.check()


@pytest.mark.parametrize("R,N,K", [(9, 200, 128), (300, 512, 256), (2100, 1288, 136)])
def test_residual_in_place_and_the_same_bits_again(R, N, K):
    apart, c = (Adapted(R, N, K, 32, 5, "runs", residual=True, bias=True) for _ in range(2))
    apart.run()
    apart.check()
    c.out.copy_(c.r)
    c.r = c.out
    c.run()
    torch.cuda.synchronize()
    assert torch.equal(c.out, apart.out)
    first = apart.out.clone()
    for fill in (0, 0x7F):                               # whatever the workspace holds
        apart.workspace.fill_(fill)
        apart.out.fill_(3.0)
        apart.run()
        torch.cuda.synchronize()
        assert torch.equal(apart.out, first)


def test_numbers_that_are_none_stay_in_their_rows():
    for R, N, K in ((5, 64, 128), (40, 96, 320), (300, 512, 256)):
        c, clean = (Adapted(R, N, K, 16, 3, "own") for _ in range(2))
        clean.run()
        c.x[2, 5], c.x[R - 1, 0] = float("nan"), float("inf")
        c.run()
        torch.cuda.synchronize()
        keep = [i for i in range(R) if i not in (2, R - 1)]
        assert torch.equal(c.out[keep], clean.out[keep])
        assert bool(torch.isnan(c.out[2]).all()) and not bool(torch.isfinite(c.out[R - 1]).any())


def test_streams_graphs_and_fewer_rows():
    c = Adapted(70, 640, 256, 16, 6, "random", residual=True)
    c.run()
    torch.cuda.synchronize()
    want = c.out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.out.fill_(3.0)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run()
    side.synchronize()
    assert torch.equal(c.out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    # the index of a captured call is read at every replay
    for pattern in ("own", "none", "one", "random"):
        index = index_of(pattern, 70, 6)
        fresh = Adapted(70, 640, 256, 16, 6, "own", residual=True, seed=len(pattern))
        c.index.copy_(torch.from_numpy(index.astype(np.int32)))
        c.x.copy_(fresh.x)
        c.down.copy_(fresh.down), c.up.copy_(fresh.up), c.scale.copy_(fresh.scale)
        c.out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        got = c.out.clone()
        c.check()
        c.run()
        torch.cuda.synchronize()
        assert torch.equal(c.out, got)
    c.out.fill_(3.0)
    c.R = 33
    c.run()
    torch.cuda.synchronize()
    assert bool((c.out[33:] == 3.0).all()) and not bool((c.out[:33] == 3.0).all())


def test_two_streams_with_a_workspace_each():
    cases = [Adapted(300, 1024, 512, 16, 6, "random", seed=s) for s in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(4):
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                c.run()
    for c in cases:
        c.check()


def test_rows_of_one_adapter_do_not_depend_on_the_others():
    """A row's result has the same bits whatever its neighbours' adapters are, but for the order in which its own adapter comes in a tile."""
    a, b = (Adapted(300, 512, 256, 16, 8, "one") for _ in range(2))
    a.run()
    b.index[1::2] = -1
    b.run()
    torch.cuda.synchronize()
    assert torch.equal(a.out[0::2], b.out[0::2])


def test_offsets_beyond_32_bits():
    """Adapters whose A and B begin behind 2^31 elements."""
    import paper_2512_21487_amd as pkg
    n, rank, N, K, R = 300, 128, 64, 65536, 20
    down = torch.zeros((n, rank, K), dtype=torch.bfloat16, device="cuda")
    small = Adapted(R, N, K, rank, 1, "one", out32=True)
    down[n - 1] = small.down[0]
    up = torch.zeros((n, N, rank), dtype=torch.bfloat16, device="cuda")
    up[n - 1] = small.up[0]
    scale = torch.ones(n, device="cuda")
    scale[n - 1] = small.scale[0]
    small.run()
    out = torch.zeros_like(small.out)
    pkg.linear_adapters(small.cfg, pkg.AdapterConfig(n_adapters=n, rank=rank), small.x, small.w, torch.full((R,), n - 1, dtype=torch.int32, device="cuda"), down,
                        up, scale, out=out, workspace=small.workspace)
    torch.cuda.synchronize()
    assert torch.equal(out, small.out)
    small.check()


@pytest.mark.parametrize("R,N,K,name", [(800, 2048, 1024, "tiles"), (800, 2048, 1023, "copies"), (5000, 72, 4096, "shared reduction")])
def test_offsets_beyond_32_bits_of_many_rows(R, N, K, name):
    """The same where the product's reduction goes on, in tiles of each kind: the last of so many adapters that A, B or both begin behind 2^32 bytes."""
    import paper_2512_21487_amd as pkg
    rank, n = 128, 2 ** 32 // (256 * max(N, K)) + 3
    small = Adapted(R, N, K, rank, 1, "one", out32=True)
    down, up = (torch.zeros((n, *s), dtype=torch.bfloat16, device="cuda") for s in ((rank, K), (N, rank)))
    down[n - 1], up[n - 1] = small.down[0], small.up[0]
    scale = torch.ones(n, device="cuda")
    scale[n - 1] = small.scale[0]
    small.run()
    out = torch.zeros_like(small.out)
    adapters = pkg.AdapterConfig(n_adapters=n, rank=rank)
    workspace = torch.empty(pkg.linear_adapters_workspace_bytes(small.cfg, adapters, R), dtype=torch.uint8, device="cuda")
    pkg.linear_adapters(small.cfg, adapters, small.x, small.w, torch.full((R,), n - 1, dtype=torch.int32, device="cuda"), down, up, scale, out=out, workspace=workspace)
    torch.cuda.synchronize()
    assert torch.equal(out, small.out)
    small.check()


def test_rows_whose_products_lie_beyond_32_bits():
    """So many rows that x, x A^T and the lists pass 2^32 bytes, or 2^30; the first, some in the middle and the last."""
    import paper_2512_21487_amd as pkg
    R, N, K, rank, n = 2 ** 25 + 77, 16, 72, 8, 3
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.empty((R, K), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    w, down, up = (torch.empty(s, dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.2, generator=gen) for s in ((N, K), (n, rank, K), (n, N, rank)))
    index = torch.randint(-1, n, (R,), dtype=torch.int32, device="cuda", generator=gen)
    cfg, adapters = pkg.LinearConfig(in_features=K, out_features=N), pkg.AdapterConfig(n_adapters=n, rank=rank)
    workspace = torch.empty(pkg.linear_adapters_workspace_bytes(cfg, adapters, R), dtype=torch.uint8, device="cuda")
    out = torch.full((R + 1, N), 9.0, dtype=torch.bfloat16, device="cuda")
    pkg.linear_adapters(cfg, adapters, x, w, index, down, up, out=out, workspace=workspace, n_rows=R)
    torch.cuda.synchronize()
    for at in (0, R // 2, R - 2000):
        rows = slice(at, at + 2000)
        v, of = x[rows].double(), index[rows]
        want, size = v @ w.double().t(), v.abs() @ w.double().abs().t()
        for a in range(n):
            mine = of == a
            want[mine] += (v[mine] @ down[a].double().t()) @ up[a].double().t()
            size[mine] += (v[mine].abs() @ down[a].double().abs().t()) @ up[a].double().abs().t()
        # what the parts of x A^T leave, fp32 sums, and a rounding to bf16
        bound = size * (2.0 ** -16 + (K + 24) * 2.0 ** -24)
        assert bool(((out[rows].double() - want).abs() <= bound + 2.0 ** -8 * (want.abs() + bound)).all())
    assert bool((out[R] == 9.0).all())


def test_no_rows_and_refused_memory():
    import paper_2512_21487_amd as pkg
    c = Adapted(8, 32, 64, 16, 2, "own")
    assert pkg.linear_adapters_workspace_bytes(c.cfg, c.adapters, 0) == 0
    c.R = 0
    c.run()
    torch.cuda.synchronize()
    assert bool((c.out == 3.0).all())
    c.R = 8
    call = lambda **kw: pkg.linear_adapters(c.cfg, c.adapters, **dict(dict(x=c.x, weight=c.w, index=c.index, down=c.down, up=c.up, out=c.out, workspace=c.workspace), **kw))
    with pytest.raises(pkg.MoeEpError, match="workspace has"):
        call(workspace=c.workspace[:c.need - 16])
    with pytest.raises(pkg.MoeEpError, match="aligned to 16"):
        call(workspace=c.workspace[8:])
    with pytest.raises(pkg.MoeEpError, match="overlap"):
        call(workspace=c.up.data_ptr(), workspace_bytes=c.need)
    with pytest.raises(ValueError, match="index"):
        call(index=c.index[:7])
    with pytest.raises(ValueError, match="workspace"):
        call(workspace=torch.zeros(1 << 16, dtype=torch.uint8))
    with pytest.raises(pkg.MoeEpError, match="down"):
        call(down=np.zeros(2 * 16 * 64, np.uint16).ctypes.data)
    call()
    c.scale = None
    c.check()
