"""Which kernel a product runs on (host only): the shapes that the GPU tests take reach every kernel, on both sides of every rule."""
import pytest

from linear_shapes import ALL, KERNELS, SHAPES, kernel_of


@pytest.mark.parametrize("name,R,N,K,w32", ALL)
def test_shapes_of_the_gpu_tests(name, R, N, K, w32):
    assert kernel_of(R, N, K, w32) == name


def test_every_kernel_has_a_shape():
    assert set(SHAPES) == set(KERNELS)
    for name in KERNELS:
        if "rows" in name or "split" in name:
            assert {w32 for *_, w32 in SHAPES[name]} == {False, True}
        if "tiles" in name:
            assert {K % 64 == 0 for _, _, K, _ in SHAPES[name]} == {False, True}


def test_operands_that_are_not_on_16_bytes_do_not_go_into_tiles():
    assert kernel_of(700, 513, 1408) == "tiles 64x64"
    for how in (dict(x=0x1008), dict(w=0x1002), dict(ldx=1412), dict(ldw=1409)):
        assert "tiles" not in kernel_of(700, 513, 1408, **how)
    assert kernel_of(700, 513, 1408, True).startswith("split")
