"""moe_ep_linear_adapters: structs, workspace sizes and refusals, all of them before any HIP call."""
import ctypes
import os
import re

import pytest

import paper_2512_21487_amd as pkg
from linear_shapes import ALL, kernel_of, KERNELS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A, B, C, D, E, F, G, H, I = (0x10000000 * i for i in range(1, 10))   # never read


def test_struct_matches_header():
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "moe_ep.h")).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} moe_ep_adapter_config;", header).group(1)
    fields = re.findall(r"(\w+)\s+(\w+)\s*;", body)
    assert [n for _, n in fields] == [f[0] for f in pkg.AdapterConfig._fields_]
    assert {t for t, _ in fields} == {"int32_t"}


def configs(linear=None, **kw):
    return (pkg.LinearConfig(**dict(dict(in_features=64, out_features=32), **(linear or {}))), pkg.AdapterConfig(**dict(dict(n_adapters=4, rank=16), **kw)))


@pytest.mark.parametrize("linear,bad,word", [
    ({}, dict(n_adapters=0), "n_adapters"), ({}, dict(n_adapters=(1 << 20) + 1), "n_adapters"), ({}, dict(rank=0), "rank"), ({}, dict(rank=4), "rank"),
    ({}, dict(rank=12), "rank"), ({}, dict(rank=136), "rank"), ({}, dict(rank=-8), "rank"), (dict(weight_type=1), {}, "weight_type"),
    (dict(in_features=0), {}, "in_features"), (dict(activation=9), {}, "activation")])
def test_configurations_that_are_refused(linear, bad, word):
    both = configs(linear, **bad)
    rc, why = pkg.validate_linear_adapters(*both)
    assert rc == -1 and word in why
    assert pkg.linear_adapters_workspace_bytes(*both, 8) == 0


def test_configurations_that_are_taken():
    for linear, good in (({}, {}), ({}, dict(n_adapters=1, rank=8)), ({}, dict(n_adapters=1 << 20, rank=128)), (dict(out_type=1), dict(rank=24))):
        assert pkg.validate_linear_adapters(*configs(linear, **good)) == (0, "ok")


def tiles_of(kernel):
    """Rows of a tile of each kernel, 0 of dot products (csrc/kernels.h)."""
    if kernel.startswith("rows"):
        return 0
    return int(re.search(r"(\d+)x\d+", kernel).group(1))


def test_workspaces_hold_every_rows_products_and_every_list():
    lib = pkg.load_library()
    for name in KERNELS:
        assert lib._ZN6moe_ep16linear_tile_rowsEi(KERNELS.index(name)) == tiles_of(name)
    for out_type, parts in ((0, 2), (1, 3)):
        for rank in (8, 16, 24, 64, 128):
            both = configs(dict(out_type=out_type), rank=rank)
            width = (parts * rank + 63) // 64 * 64
            before = 0
            for R in list(range(1, 600)) + [1023, 4096, 65537, 1 << 20, 1 << 30]:
                need = pkg.linear_adapters_workspace_bytes(*both, R)
                assert need >= before
                before = need
                for tile in (16, 32, 64, 128, 192, 256):
                    assert need >= R * (width + 8) * 2 + -(-R // tile) * (1 + tile * (1 + -(-tile // 32))) * 4
    assert pkg.linear_adapters_workspace_bytes(*configs(), 0) == 0
    assert pkg.linear_adapters_workspace_bytes(*configs(), (1 << 30) + 1) == 0


def call(kw, linear=None, **cfg):
    pkg.linear_adapters(*configs(linear, **cfg), **dict(dict(x=A, weight=B, index=C, down=D, up=E, out=F, workspace=G, workspace_bytes=1 << 20, n_rows=8, stream=0), **kw))


@pytest.mark.parametrize("kw,word", [
    (dict(x=None), "x, weight"), (dict(weight=None), "x, weight"), (dict(out=None), "x, weight"), (dict(index=None), "index, down"), (dict(down=None), "index, down"),
    (dict(up=None), "index, down"), (dict(workspace=None), "index, down"), (dict(n_rows=-1), "n_rows"), (dict(n_rows=(1 << 30) + 1), "n_rows"),
    (dict(x=A + 1), "aligned"), (dict(index=C + 2), "aligned"), (dict(down=D + 1), "aligned"), (dict(up=E + 8), "aligned to 16"), (dict(scale=H + 2), "aligned"),
    (dict(workspace=G + 8), "aligned to 16"), (dict(workspace_bytes=100), "workspace has 100 bytes"), (dict(out=A), "out must not overlap x"),
    (dict(out=C), "out must not overlap index"), (dict(out=D + 64), "out must not overlap down"), (dict(out=E), "out must not overlap up"),
    (dict(scale=F), "out must not overlap scale"), (dict(workspace=A), "workspace must not overlap x"), (dict(workspace=B), "workspace must not overlap weight"),
    (dict(workspace=F), "overlap"), (dict(workspace=C), "workspace must not overlap index"), (dict(bias=G), "workspace must not overlap bias"),
    (dict(residual=G), "workspace must not overlap residual"), (dict(scale=G), "workspace must not overlap scale")])
def test_calls_that_are_refused(kw, word):
    with pytest.raises(pkg.MoeEpError, match=word):
        call(kw)


def test_no_rows_is_nothing():
    call(dict(n_rows=0))


def test_tensors_that_are_refused():
    torch = pytest.importorskip("torch")
    z = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype)
    for name, t in (("x", z(8, 64, dtype=torch.float16)), ("index", z(8, dtype=torch.int64)), ("index", z(8, dtype=torch.float32)), ("down", z(4, 16, 64, dtype=torch.float16)),
                    ("up", z(4, 16, 16)), ("scale", z(4, dtype=torch.int32)), ("workspace", z(1 << 16, dtype=torch.uint8)), ("index", z(8, dtype=torch.int32))):
        kw = {name: t}
        if name == "workspace":
            kw["workspace_bytes"] = None
        with pytest.raises(ValueError, match=name):
            call(kw)
    with pytest.raises(ValueError, match="workspace_bytes"):
        call(dict(workspace_bytes=None))


@pytest.mark.parametrize("name,shape,fits", [
    ("down", (4, 16, 64), True), ("down", (5, 16, 64), True), ("down", (64, 64), True), ("down", (4 * 16 * 64,), True), ("down", (4, 64, 16), False), ("down", (4, 32, 64), False),
    ("down", (16, 4, 64), False), ("down", (4, 16, 128), False), ("down", (3, 16, 64), False), ("down", (4, 1024), False), ("down", (1, 4, 16, 64), False),
    ("up", (4, 32, 16), True), ("up", (6, 32, 16), True), ("up", (128, 16), True), ("up", (4, 16, 32), False), ("up", (16, 128), False), ("up", (4, 64, 16), False),
    ("up", (4, 32, 32), False), ("up", (3, 32, 16), False)])
def test_adapters_whose_shape_is_another(name, shape, fits):
    """As many elements in another order would give other numbers."""
    torch = pytest.importorskip("torch")
    both = dict(down=D, up=E)
    both[name] = torch.zeros(shape, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match=name) as ei:   # one that fits is refused for being on the host
        call(both)
    assert ("must be [" in str(ei.value)) == (not fits)


def test_more_workspace_than_the_tensor_has():
    """A number of bytes beside a tensor is no licence to write behind it."""
    torch = pytest.importorskip("torch")
    small = torch.zeros(1 << 10, dtype=torch.uint8)
    with pytest.raises(ValueError, match="workspace has 1024 bytes"):
        call(dict(workspace=small, workspace_bytes=1 << 20))
    with pytest.raises(ValueError, match="contiguous"):
        call(dict(workspace=torch.zeros((8, 64), dtype=torch.uint8)[:, :32], workspace_bytes=64))
    with pytest.raises(ValueError, match="workspace"):   # one that fits is refused for being on the host
        call(dict(workspace=small, workspace_bytes=1 << 10))
