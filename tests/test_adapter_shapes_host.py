"""Which kernel a product with adapters runs on (host only): the shapes that the GPU tests take reach every one, as the launch itself chooses."""
import pytest

from adapter_shapes import GATHERED, GROUPED, MANY, OFF, launched
from linear_shapes import KERNELS


@pytest.mark.parametrize("name,R,N,K", [(name, *s) for name in MANY for s in MANY[name]])
def test_shapes_of_many_rows(name, R, N, K):
    assert R > GATHERED and launched(R, N, K, 16, 5) == name


@pytest.mark.parametrize("name", sorted(OFF))
def test_shapes_whose_first_row_is_off_16_bytes(name):
    assert launched(*OFF[name], 24, 9, x=0x1002) == name


@pytest.mark.parametrize("name,R,N,K", [(name, *s) for name in GROUPED for s in GROUPED[name]])
def test_shapes_of_rows_that_are_grouped(name, R, N, K):
    assert R <= GATHERED and launched(R, N, K, 24, 7) == name


def test_every_kernel_has_a_shape():
    products = {k for k in KERNELS if not k.startswith("rows")}
    assert {n for n in MANY if "copies" not in n} | set(OFF) == products
    assert {n for n in MANY if "copies" in n} == {n + ", copies" for n in products if n.startswith("tiles")}
    assert set(GROUPED) == products | {"rows of 16", "rows of 32"}
    for shapes in (MANY, GROUPED):
        for name, each in shapes.items():
            if name.startswith("tiles") and "copies" not in name:
                assert {K % 64 == 0 for _, _, K in each} == {False, True}
            if name.startswith("tiles"):
                assert any(K > 256 for _, _, K in each)


def test_rows_are_copied_only_in_front_of_tiles_that_direct_loads_fill():
    assert launched(4100, 1300, 523, 16, 5).endswith(", copies")
    assert launched(4100, 1300, 520, 16, 5, pads=(3, 0)).endswith(", copies") and launched(4100, 1300, 520, 16, 5, pads=(0, 5)).endswith(", copies")
    assert launched(4100, 1300, 520, 16, 5, pads=(8, 8)).startswith("tiles") and not launched(4100, 1300, 520, 16, 5, pads=(8, 8)).endswith("copies")
    for R, N, K in ((600, 1100, 129), (800, 1100, 129), (4100, 700, 65), (1531, 1409, 131)):
        assert "copies" not in launched(R, N, K, 16, 5)
