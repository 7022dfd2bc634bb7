"""Every kernel of moe_ep_linear with every epilogue: which one a shape runs on is asserted, so that a rule that moves moves no test away unseen."""
import pytest

from linear_shapes import ALL, KERNELS, SHAPES, kernel_of
from test_gpu_linear import ACTS, Case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def runs_on(name, R, N, K, w32):
    n_cu = torch.cuda.get_device_properties(0).multi_processor_count
    if n_cu != 256:
        pytest.skip("shapes for 256 compute units")
    assert kernel_of(R, N, K, w32, n_cu) == name


@pytest.mark.parametrize("name,R,N,K,w32", ALL)
def test_every_epilogue(name, R, N, K, w32):
    """Activations in both result types; without a residual, with one, and with one in place of the result, which has the bits of one apart."""
    runs_on(name, R, N, K, w32)
    for i, act in enumerate(ACTS):
        for out32 in (False, True):
            how = ("none", "apart", "in place")[(i + out32) % 3]
            c = Case(R, N, K, w32=w32, out32=out32, bias=i != 2, residual=how != "none", name=act, seed=i)
            if how == "in place":
                apart = Case(R, N, K, w32=w32, out32=out32, bias=i != 2, residual=True, name=act, seed=i)
                apart.run()
                apart.check()
                c.out.copy_(c.r)
                c.r = c.out
                c.run()
                torch.cuda.synchronize()
                assert torch.equal(c.out, apart.out)
            else:
                c.run()
                c.check()


@pytest.mark.parametrize("name,R,N,K,w32", [(name, *s) for name in KERNELS for s in SHAPES[name] if s[3] and s[2] % 32 == 0] + [("rows 1x1", 8, 61, 128, True)])
def test_fp32_weights_count_to_the_last_bit_on_every_kernel_that_takes_them(name, R, N, K, w32):
    """1 + 2^-8 + 2^-23 is three bf16 numbers, 1, 2^-8 and 2^-23: without the third the sums are 0.  No sum rounds, in whichever order a matrix instruction adds its 32
    products to what it has, a multiple of 2^-19: sums of 1 are multiples of 2^-19 below 32, of 2^-8 too, and those of 2^-23 are small; one product after the other,
    all are multiples of 2^-23 below 2."""
    import paper_2512_21487_amd as pkg
    runs_on(name, R, N, K, w32)
    w = torch.empty((N, K), device="cuda")
    w[:, 0::2] = 1.0 + 2.0 ** -8
    w[:, 1::2] = -(1.0 + 2.0 ** -8 + 2.0 ** -23)
    x = torch.ones((R, K), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros((R, N), device="cuda")
    pkg.linear(pkg.LinearConfig(in_features=K, out_features=N, weight_type=pkg.F32, out_type=pkg.F32), x, w, out=out)
    torch.cuda.synchronize()
    assert bool((out == -(K // 2) * 2.0 ** -23).all())


@pytest.mark.parametrize("name,R,N,K,w32", ALL)
def test_activations_of_numbers_that_are_huge_or_infinite(name, R, N, K, w32):
    """A pre-activation of plus infinity, or that overflows, is one of every activation; a huge one is itself, a huge negative one 0 but without an activation."""
    import paper_2512_21487_amd as pkg
    runs_on(name, R, N, K, w32)
    huge = (float("inf"), 1e30, -1e30, 3e38, -3e38)
    for out32 in (False, True):
        for act in ACTS:
            c = Case(R, N, K, w32=w32, out32=out32, bias=True, name=act)
            cols = range(0, 10, 2)
            for n, v in zip(cols, huge):
                c.b[n] = v
            if not w32:                                   # 3e38 + 3e38 in the sum
                c.w[1, :2] = 2.0
                c.x[R - 1, :2] = 3e38
            c.run()
            torch.cuda.synchronize()
            for n, v in zip(cols, huge):
                got = c.out[:R - 1, n].double()
                if v > 0 or act == "none":
                    want = torch.full_like(got, v) if not out32 else torch.full_like(got, float(torch.tensor(v, dtype=torch.float32)))
                    assert torch.equal(got, want) if v == float("inf") else bool(((got - want).abs() <= 2.0 ** -8 * abs(v)).all())
                else:
                    assert bool((got == 0).all())
            if not w32:
                assert float(c.out[R - 1, 1]) == float("inf")
            assert bool(torch.isfinite(c.out[:R - 1, 10:]).all()) and bool(torch.isfinite(c.out[:R - 1, 1::2]).all())
