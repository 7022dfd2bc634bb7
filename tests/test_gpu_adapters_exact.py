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
