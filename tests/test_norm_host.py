"""moe_ep_norm: struct, exported constants and refusals, all of them before any HIP call."""
import ctypes
import os
import re

import pytest

import paper_2512_21487_amd as pkg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SIZES = {"int32_t": 4, "float": 4, "int64_t": 8}
A, B, C, D, E, F = (0x10000000 * i for i in range(1, 7))   # never read


def test_struct_and_constants_match_header():
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "moe_ep.h")).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} moe_ep_norm_config;", header).group(1)
    fields = re.findall(r"(\w+)\s+(\w+)\s*;", body)
    assert [n for _, n in fields] == [f[0] for f in pkg.NormConfig._fields_]
    assert [SIZES[t] for t, _ in fields] == [ctypes.sizeof(f[1]) for f in pkg.NormConfig._fields_]
    for name, value in re.findall(r"MOE_EP_((?:NORM|GATE)_\w+) = (\d)", header):
        assert getattr(pkg, name) == int(value)


def config(**kw):
    return pkg.NormConfig(**dict(dict(features=64, norm_before=pkg.NORM_RMS), **kw))


@pytest.mark.parametrize("bad,word", [
    (dict(features=0), "features"), (dict(features=32769), "features"), (dict(norm_after=3), "norm_after"), (dict(norm_after=-1), "norm_after"),
    (dict(norm_before=3), "norm_before"), (dict(block_type=2), "block_type"), (dict(stream_type=-1), "stream_type"), (dict(out_type=2), "out_type"),
    (dict(weight_type=2), "weight_type"), (dict(gate_type=2), "gate_type"), (dict(gate_form=3), "gate_form"), (dict(gate_per_row=2), "gate_per_row"),
    (dict(eps=0.0), "eps"), (dict(eps=-1e-6), "eps"), (dict(eps=1.5), "eps"), (dict(eps=float("nan")), "eps"),
    (dict(block_scale=float("inf")), "block_scale"), (dict(residual_scale=float("nan")), "residual_scale"), (dict(weight_offset=float("inf")), "weight_offset"),
    (dict(block_stride=63), "block_stride"), (dict(residual_stride=63), "residual_stride"), (dict(gate_stride=63), "gate_stride"),
    (dict(gate_per_row=1, gate_stride=-1), "gate_stride"), (dict(sum_stride=63), "sum_stride"), (dict(out_stride=(1 << 22) + 1), "out_stride"), (dict(device=-1), "device")])
def test_norms_that_are_refused(bad, word):
    rc, why = pkg.validate_norm(config(**bad))
    assert rc == -1 and word in why


def test_norms_that_are_taken():
    for good in (dict(), dict(features=1), dict(features=32768), dict(norm_before=0, eps=0.0), dict(gate_per_row=1, gate_stride=1), dict(block_scale=0.0),
                 dict(residual_scale=-2.0), dict(weight_offset=1.0), dict(eps=1e-20), dict(eps=1.0), dict(block_stride=1 << 22)):
        assert pkg.validate_norm(config(**good)) == (0, "ok")
    cfg = pkg.NormConfig(features=4)
    assert (cfg.block_scale, cfg.residual_scale, cfg.weight_offset) == (1.0, 1.0, 0.0) and cfg.eps == ctypes.c_float(1e-6).value
    with pytest.raises(ValueError, match="features"):
        cfg.features = 1 << 33


def call(kw, **cfg):
    pkg.norm(config(**cfg), **dict(dict(block=A, out=B, n_rows=4, stream=0), **kw))


@pytest.mark.parametrize("kw,cfg,word", [
    (dict(block=None), {}, "block"), (dict(out=None), {}, "out must"), (dict(), dict(norm_before=0), "out must"),
    (dict(out=None), dict(norm_before=0), "sum and out"), (dict(out=None, sum=C, before_weight=D), dict(norm_before=0), "before_weight"),
    (dict(n_rows=-1), {}, "n_rows"), (dict(n_rows=(1 << 30) + 1), {}, "n_rows"), (dict(block=A + 1), {}, "aligned"), (dict(sum=C + 1), {}, "aligned"),
    (dict(before_weight=C + 2), dict(weight_type=1), "aligned"), (dict(gate=C + 2), dict(gate_type=1, gate_per_row=1), "aligned"),
    (dict(sum=B), {}, "overlap"), (dict(out=A + 64), {}, "out must not overlap block"), (dict(out=A), dict(out_type=1), "out must not overlap block"),
    (dict(out=A), dict(out_stride=128), "out must not overlap block"), (dict(residual=C, sum=C + 128), {}, "sum must not overlap residual"),
    (dict(residual=C, sum=C), dict(sum_stride=128), "sum must not overlap residual"), (dict(sum=A), {}, "sum must not overlap block"),
    (dict(residual=C, out=C), {}, "out must not overlap residual"), (dict(gate=C, sum=C), {}, "sum must not overlap gate"),
    (dict(before_weight=B), {}, "out must not overlap before_weight"), (dict(after_bias=C, sum=C), {}, "sum must not overlap after_bias")])
def test_calls_that_are_refused(kw, cfg, word):
    with pytest.raises(pkg.MoeEpError, match=word):
        call(kw, **cfg)


def test_no_rows_is_nothing():
    call(dict(n_rows=0))


def test_tensors_that_are_refused():
    torch = pytest.importorskip("torch")
    z = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype)
    for name, t in (("block", z(4, 64, dtype=torch.float16)), ("residual", z(4, 64, dtype=torch.float32)), ("gate", z(4, 64, dtype=torch.float16)),
                    ("after_weight", z(64, dtype=torch.float16)), ("before_bias", z(64, dtype=torch.int32)), ("sum", z(4, 64, dtype=torch.float16)),
                    ("out", z(4, 64, dtype=torch.float16))):
        with pytest.raises(ValueError, match=name):
            call({name: t})
    with pytest.raises(ValueError, match="gate"):
        call(dict(gate=z(4, dtype=torch.float32)), gate_per_row=1)
    with pytest.raises(ValueError, match="device tensor"):
        call(dict(gate=z(4)), gate_per_row=1)


def test_which_kernel_a_row_runs_on():
    """The shapes of the GPU tests reach every one, on both sides of the number of compute units where that decides."""
    of = pkg.load_library()._ZN6moe_ep14norm_kernel_ofEiii
    names = ("1x1", "2x1", "4x1", "8x1", "16x1", "8x2", "16x2", "16x4")   # csrc/kernels.h
    got = {(R, M): names[of(R, M, 256)] for M in (1, 512, 513, 1024, 1025, 2048, 2049, 4096, 4097, 8192, 8193, 16384, 16385, 32768) for R in (1, 256, 257, 5000)}
    for (R, M), name in got.items():
        wavefronts, turns = (int(n) for n in name.split("x"))
        assert wavefronts * turns * 512 >= M
        assert (name == "16x1") == (4096 < M <= 8192 and R <= 256)
    assert set(got.values()) == set(names)
