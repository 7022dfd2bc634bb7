"""Every kernel that moe_ep_linear_adapters launches: which one a shape runs on is asserted, as the launch itself chooses."""
import pytest

from adapter_shapes import GROUPED, MANY, OFF, launched
from test_gpu_adapters import Adapted
from test_gpu_linear import ACTS

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def on(name, c, pads=(0, 0)):
    if torch.cuda.get_device_properties(0).multi_processor_count != 256:
        pytest.skip("shapes for 256 compute units")
    assert launched(c.R, c.N, c.K, c.rank, c.n, pads=pads, x=c.x.data_ptr(), w=c.w.data_ptr()) == name


@pytest.mark.parametrize("name,R,N,K", [(name, *s) for name in MANY for s in MANY[name]])
@pytest.mark.parametrize("pattern", ["runs", "own", "some"])
def test_many_rows(name, R, N, K, pattern):
    """Without an activation and with one, in both types; tiles of one adapter, of all, and of some rows that have one."""
    i = ("runs", "own", "some").index(pattern)
    for rank, n, out32, act in ((16, 5, False, "none"), (24, 9, True, ACTS[1 + (R + i) % 4]), (128, 3, False, ACTS[1 + (R + i + 1) % 4]), (64, 2, True, "none")):
        c = Adapted(R, N, K, rank, n, pattern, out32=out32, bias=rank != 16, residual=rank != 24, name=act, seed=i)
        on(name, c)
        c.run()
        c.check()


@pytest.mark.parametrize("name", sorted(OFF))
@pytest.mark.parametrize("pattern", ["runs", "some"])
def test_rows_whose_first_alone_is_off_16_bytes(name, pattern):
    for out32, act in ((False, "silu"), (True, "none")):
        c = Adapted(*OFF[name], 24, 9, pattern, out32=out32, bias=True, residual=True, name=act, shifts=(1, 0, 0, 0))
        on(name, c)
        c.run()
        c.check()


@pytest.mark.parametrize("name,R,N,K", [(name, *s) for name in GROUPED for s in GROUPED[name]])
@pytest.mark.parametrize("pattern", ["random", "own", "none"])
def test_grouped_rows(name, R, N, K, pattern):
    for out32, act in ((False, "gelu_tanh"), (True, "none")):
        c = Adapted(R, N, K, 24, 7, pattern, out32=out32, bias=True, residual=out32, name=act)
        on(name, c)
        c.run()
        c.check()


@pytest.mark.parametrize("name,R,N,K", [("split 32x16", 900, 72, 4096), ("split 64x32 by 4", 800, 2048, 64), ("split 64x32 by 4", 800, 2100, 72), ("tiles 64x64, copies", 1531, 1409, 203)])
def test_offsets_beyond_32_bits(name, R, N, K):
    """The last of so many adapters that its A, or its B, begins behind 2^32 bytes."""
    import paper_2512_21487_amd as pkg
    rank, n = 128, 2 ** 32 // (256 * max(N, K)) + 3
    small = Adapted(R, N, K, rank, 1, "one", out32=True)
    on(name, small)
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


@pytest.mark.parametrize("name,R,N,K", [("tiles 128x128, copies", 3951, 961, 523), ("tiles 256x192, copies", 3717, 3165, 65), ("tiles 256x256, copies", 4980, 2305, 67),
                                        ("tiles 128x128, copies", 8012, 450, 520), ("tiles 256x256, copies", 8223, 1349, 328)])
@pytest.mark.parametrize("pads", [(3, 0, 0, 0), (0, 5, 0, 0), (7, 7, 3, 1)])
def test_rows_that_are_copied(name, R, N, K, pads):
    """x, W or both; a reduction that is whole pieces of 16 bytes in rows that are not, and one that is not."""
    for shifts in ((0, 0, 0, 0), (1, 3, 0, 0)):
        c = Adapted(R, N, K, 16, 5, "runs", bias=True, residual=True, pads=pads, shifts=shifts)
        if shifts[0] == 0:                               # (an operand that is not copied goes into tiles from 16 bytes only)
            on(name, c, pads=pads[:2])
        c.run()
        c.check()


@pytest.mark.parametrize("name,R,N,K", [(name, *MANY[name][-1]) for name in MANY] + [("off: " + name, *OFF[name]) for name in sorted(OFF)])
@pytest.mark.parametrize("out32", [False, True])
def test_a_broken_adapter_on_every_kernel(name, R, N, K, out32):
    """B of one adapter is NaN in the first and the last column, A of another in one number; rows of others have what their formula gives, the broken ones' NaN where it does, residual in place."""
    off = name.startswith("off: ")
    c = Adapted(R, N, K, 16, 5, "own", out32=out32, bias=True, residual=True, name="gelu", shifts=(1, 0, 0, 0) if off else (0, 0, 0, 0))
    on(name[5:] if off else name, c)
    want, bound = c.want()
    c.up[1, 0], c.up[1, N - 1], c.down[3, 15, 0] = float("nan"), float("nan"), float("nan")
    none = torch.zeros((R, N), dtype=torch.bool, device="cuda")
    none[c.index == 1, 0] = none[c.index == 1, N - 1] = True
    none[c.index == 3] = True
    c.out.copy_(c.r)
    c.r = c.out
    c.run()
    torch.cuda.synchronize()
    got = c.out.double()
    assert torch.equal(torch.isnan(got), none)
    assert bool((((got - want).abs() / bound)[~none] <= 1.0).all())
