"""The operators' tensor arguments in the binding: types that the call does not read are refused before any HIP call."""
import pytest

import paper_2512_21487_amd as pkg

torch = pytest.importorskip("torch")

A, B, C, D, E = (0x10000000 * i for i in range(1, 6))   # never read


def zeros(*shape, dtype):
    return torch.zeros(shape, dtype=dtype)


def linear(**kw):
    cfg = pkg.LinearConfig(in_features=64, out_features=32, weight_type=kw.pop("weight_type", pkg.BF16), out_type=kw.pop("out_type", pkg.BF16))
    pkg.linear(cfg, **dict(dict(x=A, weight=B, out=C, n_rows=4, stream=0), **kw))


def route(**kw):
    rule = pkg.Routing(n_experts=64, top_k=6, score_type=kw.pop("score_type", pkg.F32))
    pkg.route(rule, **dict(dict(scores=A, idx=B, w=C, n_tokens=4, stream=0), **kw))


@pytest.mark.parametrize("call,name,shape,dtype,how", [
    (linear, "x", (4, 64), torch.float16, {}), (linear, "weight", (32, 64), torch.float16, {}), (linear, "out", (4, 32), torch.float16, {}),
    (linear, "residual", (4, 32), torch.float16, {}), (linear, "weight", (32, 64), torch.int32, dict(weight_type=pkg.F32)),
    (linear, "bias", (32,), torch.int32, {}), (linear, "out", (4, 32), torch.int32, dict(out_type=pkg.F32)),
    (linear, "residual", (4, 32), torch.int32, dict(out_type=pkg.F32)),
    (route, "scores", (4, 64), torch.float16, dict(score_type=pkg.BF16)), (route, "scores", (4, 64), torch.int32, {}),
    (route, "bias", (64,), torch.int32, {}), (route, "idx", (4, 6), torch.float32, {}), (route, "w", (4, 6), torch.int32, {}),
    (route, "token_mask", (4,), torch.float8_e4m3fn, {})])
def test_types_of_the_right_size_that_are_not_read(call, name, shape, dtype, how):
    with pytest.raises(ValueError, match=f"{name} .*{str(dtype).split('.')[1]}"):
        call(**{name: zeros(*shape, dtype=dtype)}, **how)


@pytest.mark.parametrize("call,name,shape,dtype,how", [
    (linear, "x", (4, 64), torch.bfloat16, {}), (linear, "x", (4, 64), torch.int16, {}), (linear, "weight", (32, 64), torch.uint16, {}),
    (linear, "weight", (32, 64), torch.float32, dict(weight_type=pkg.F32)), (linear, "bias", (32,), torch.float32, {}),
    (route, "scores", (4, 64), torch.int16, dict(score_type=pkg.BF16)), (route, "idx", (4, 6), torch.int32, {}), (route, "token_mask", (4,), torch.bool, {}),
    (route, "token_mask", (4,), torch.uint8, {}), (route, "token_mask", (4,), torch.int8, {})])
def test_types_that_are_read(call, name, shape, dtype, how):
    """bf16 may come as 16-bit integers that hold its bits; what is refused here is that these are no device tensors."""
    with pytest.raises(ValueError, match="device tensor"):
        call(**{name: zeros(*shape, dtype=dtype)}, **how)


def test_the_bias_of_a_context_is_checked_alike():
    class Context:   # set_routing's own part, without a library call
        cfg = pkg.MoeEpConfig(n_experts=8)

    with pytest.raises(ValueError, match="bias .*int32"):
        pkg.MoeEp.set_routing(Context(), pkg.Routing(n_experts=8, top_k=2, score_type=pkg.F32), torch.zeros(8, dtype=torch.int32))


def test_unknown_types_are_named_by_the_call():
    with pytest.raises(pkg.MoeEpError, match="score_type"):
        route(score_type=7)
    with pytest.raises(pkg.MoeEpError, match="weight_type"):
        linear(weight_type=7)
    with pytest.raises(pkg.MoeEpError, match="out_type"):
        linear(out_type=-1)


class On:
    """A tensor as if on another GPU."""

    def __init__(self, t, device):
        self._t, self._device, self.is_cuda, self.device = t, device, True, torch.device("cuda", device)

    def get_device(self):
        return self._device

    def __getattr__(self, name):
        return getattr(self._t, name)


@pytest.mark.parametrize("call,name,shape,dtype", [
    (linear, "x", (4, 64), torch.bfloat16), (linear, "weight", (32, 64), torch.bfloat16), (linear, "bias", (32,), torch.float32),
    (linear, "residual", (4, 32), torch.bfloat16), (linear, "out", (4, 32), torch.bfloat16), (route, "scores", (4, 64), torch.float32),
    (route, "bias", (64,), torch.float32), (route, "token_mask", (4,), torch.uint8), (route, "idx", (4, 6), torch.int32), (route, "w", (4, 6), torch.float32)])
def test_tensors_of_another_device(call, name, shape, dtype, monkeypatch):
    """A config that was not told of a device runs on the first one, and on its stream."""
    monkeypatch.setattr(torch.cuda, "device_count", lambda: 2)
    with pytest.raises(ValueError, match=f"{name} is on cuda:1, .* device 0"):
        call(**{name: On(zeros(*shape, dtype=dtype), 1)})
    with pytest.raises(pkg.MoeEpError):   # of this one: there is no GPU here, or it is no memory of one
        call(**{name: On(zeros(*shape, dtype=dtype), 0)})


def test_counts_of_rows_that_32_bits_do_not_hold():
    for n in (2 ** 32, 2 ** 32 + 4, 2 ** 31, -2 ** 32 + 4):
        with pytest.raises(pkg.MoeEpError, match="n_rows must be in 0..2.30") as ei:
            linear(n_rows=n)
        assert ei.value.code == -1
        with pytest.raises(pkg.MoeEpError, match="n_tokens must be in 0..2.30") as ei:
            route(n_tokens=n)
        assert ei.value.code == -1


@pytest.mark.parametrize("make,name,value", [
    (pkg.LinearConfig, "in_features", 2 ** 32 + 64), (pkg.LinearConfig, "out_features", 2 ** 31), (pkg.LinearConfig, "x_stride", 2 ** 64 + 64),
    (pkg.LinearConfig, "activation", -2 ** 32 + 1), (pkg.Routing, "n_experts", 2 ** 32 + 8), (pkg.Routing, "score_stride", 2 ** 63)])
def test_fields_that_do_not_hold_a_number(make, name, value):
    with pytest.raises(ValueError, match=name):
        make(**{name: value})
    made = make(device=1)
    with pytest.raises(ValueError, match=name):
        setattr(made, name, value)
    assert getattr(made, name) == 0 and made.device == 1
