"""moe_ep_linear_adapters where the result is known to the last bit, and where adapters or rows hold numbers that are none."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R,N,K", [(1, 96, 72), (33, 200, 130), (300, 512, 256), (700, 96, 65), (800, 40, 300), (800, 520, 203), (1100, 1030, 328), (2600, 1500, 576), (4200, 1400, 128)])
@pytest.mark.parametrize("rank", [8, 16, 24, 64, 72, 128])
@pytest.mark.parametrize("out32", [False, True])
def test_x_a_counts_to_24_bits(R, N, K, rank, out32):
    """x A^T = 1 + 2^-9 + 2^-18, of which x W^T takes 1 + 2^-9 away: the result is 2^-18, and with x A^T in 16 bits 0.  Nothing rounds in whichever order: all are multiples of 2^-18 below 2."""
    import paper_2512_21487_amd as pkg
    n = 3
    x, w = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((R, K), (N, K)))
    down, up = (torch.zeros((n, *s), dtype=torch.bfloat16, device="cuda") for s in ((rank, K), (N, rank)))
    at = torch.tensor([0, K // 2, K - 1], device="cuda")
    x[:, at] = 1.0
    w[:, at[0]], w[:, at[1]] = -1.0, -2.0 ** -9
    for i, v in enumerate((0.5, 2.0 ** -10, 2.0 ** -19)):
        down[:, :, at[i]] = v
    for a in range(n):                                   # each adapter reads a rank of its own
        up[a, :, (0, rank // 2, rank - 1)[a]] = 1.0
    index = torch.arange(R, device="cuda", dtype=torch.int32) * 4 // R - 1
    index[0] = n - 1
    cfg, adapters = pkg.LinearConfig(in_features=K, out_features=N, out_type=int(out32)), pkg.AdapterConfig(n_adapters=n, rank=rank)
    workspace = torch.full((pkg.linear_adapters_workspace_bytes(cfg, adapters, R),), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.zeros((R, N), dtype=torch.float32 if out32 else torch.bfloat16, device="cuda")
    pkg.linear_adapters(cfg, adapters, x, w, index, down, up, torch.full((n,), 2.0, device="cuda"), out=out, workspace=workspace)
    torch.cuda.synchronize()
    alone = -(1.0 + 2.0 ** -9)
    want = torch.where(index >= 0, 2.0 ** -18, alone)[:, None].to(out.dtype).expand(R, N)
    assert torch.equal(out, want)


# rows, columns, reduction: shared reductions, tiles of every size, through registers and from copies
MANY = [(800, 40, 300), (780, 520, 203), (800, 1030, 328), (900, 300, 4096), (1100, 1030, 72), (2600, 1500, 576), (3000, 2100, 65), (3800, 3130, 128), (4100, 2930, 128), (4100, 1400, 1024), (1531, 1409, 136)]


@pytest.mark.parametrize("R,N,K", MANY + [(40, 300, 200), (700, 300, 200)])
@pytest.mark.parametrize("residual", ["none", "apart", "in place"])
def test_a_broken_adapter_spoils_its_own_rows_alone(R, N, K, residual):
    """Two of six adapters hold numbers that are none, in A, in some columns of B, in their scale; rows of the others, and without one, have what their formula gives."""
    from test_gpu_adapters import Adapted
    i = R % 5
    c = Adapted(R, N, K, (8, 16, 24, 64, 128)[i], 6, "random" if R % 2 else "runs", out32=i == 1, bias=True, residual=residual != "none", name=("none", "gelu_tanh", "gelu", "silu", "none")[i], seed=3)
    for t in (c.down, c.up, c.scale):                    # adapters that no row had are some that rows have now
        t.nan_to_num_(nan=0.1)
    c.index[5::97] = -1                                  # runs of one adapter meet others all the same
    c.index[7::61] = 1
    c.index[11::53] = 4
    want, bound = c.want()
    inf, nan = float("inf"), float("nan")
    gone = torch.zeros((R, N), dtype=torch.bool, device="cuda")
    if i % 2:
        c.down[1, 3, K // 2] = nan
        gone[c.index == 1] = True
    else:
        c.up[1, N // 3:N // 3 + 5] = nan
        gone[c.index == 1, N // 3:N // 3 + 5] = True
    c.up[4, :, 2] = inf if i in (0, 4) else nan          # (activations of minus infinity are numbers)
    if i == 3:
        c.up[4, :, 2], c.scale[4] = 1.0, nan
    gone[c.index == 4] = True
    if residual == "in place":
        c.out.copy_(c.r)
        c.r = c.out
    c.run()
    torch.cuda.synchronize()
    got = c.out.double()
    assert bool(torch.isfinite(got[~gone]).all())
    assert bool((((got - want).abs() / bound)[~gone] <= 1.0).all())
    assert not bool(torch.isfinite(got[gone]).any())


@pytest.mark.parametrize("R,N,K", MANY)
def test_rows_with_numbers_that_are_none_leave_the_others_their_bits(R, N, K):
    from test_gpu_adapters import Adapted
    c, clean = (Adapted(R, N, K, 16, 5, "runs", bias=True, residual=True) for _ in range(2))
    clean.run()
    bad = torch.tensor([2, R // 2, R - 1], device="cuda")
    c.x[2, K - 1], c.x[R // 2, 0], c.x[R - 1, K // 2] = float("nan"), float("inf"), -float("inf")
    c.run()
    torch.cuda.synchronize()
    keep = torch.ones(R, dtype=torch.bool, device="cuda")
    keep[bad] = False
    assert torch.equal(c.out[keep], clean.out[keep]) and not bool(torch.isfinite(c.out[bad]).any())
