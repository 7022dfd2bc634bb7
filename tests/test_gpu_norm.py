"""moe_ep_norm against its formula in float64."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

KINDS, FORMS = ("none", "rms", "layer"), ("as_is", "sigmoid", "silu")


def normal(gen, shape, std, wide):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=gen).to(torch.float32 if wide else torch.bfloat16)


def n_of(kind, x, weight, bias, offset, eps):
    """The norm in float64, and what fp32 is off by: dx, the error x comes with, goes through; sums of M squares, the mean's sum and a few steps of the rest."""
    M = x[0].shape[1]
    u = 2.0 ** -24
    v, dv = x
    if kind != "none":
        mean = v.mean(dim=1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
        # a sum over M numbers in lanes and wavefronts: at most M / 64 + 16 additions one behind another
        depth = M / 64 + 16
        dmean = depth * u * v.abs().mean(dim=1, keepdim=True) + dv.mean(dim=1, keepdim=True) if kind == "layer" else mean
        c = v - mean
        dc = dv + dmean + 2 * u * (v.abs() + mean.abs())
        power = (c * c).mean(dim=1, keepdim=True)
        # relative error of the mean square, by Cauchy and Schwarz on its first-order term, and its second-order term
        off = (dc * dc).mean(dim=1, keepdim=True)
        dpower = 2 * torch.sqrt(power * off) + off + (depth + 4) * u * power
        r = 1.0 / torch.sqrt(power + eps)
        # the square root halves a small relative error; (1 - e)^-1/2 - 1 <= e for e <= 0.6
        dr = r * (dpower / (power + eps) + 4 * u)
        v, dv = c * r, dc * r + (c.abs() + dc) * dr + 2 * u * c.abs() * r
    if weight is not None:
        w = weight.double() + offset
        dv = dv * w.abs() + v.abs() * (u * (weight.double().abs() + abs(offset))) + 2 * u * (v * w).abs()
        v = v * w
    if bias is not None:
        v = v + bias.double()
        dv = dv + u * v.abs()
    return v, dv


class Case:
    def __init__(self, R, M, *, after="none", before="rms", weights=True, biases=False, offset=0.0, gate="none", form="as_is", residual=True, block_scale=1.0,
                 residual_scale=1.0, block32=False, stream32=False, out32=False, weight32=False, gate32=False, sums=True, pads=(0, 0, 0, 0, 0), shift=0,
                 eps=1e-6, seed=0, std=1.0):
        """pads: elements between rows of block, residual, gate, sum, out; shift: elements before their first."""
        import paper_2512_21487_amd as pkg
        gen = torch.Generator(device="cuda").manual_seed(seed + R + 7 * M)

        def rows(cols, pad, wide, fill):
            flat = torch.full((shift + R * (cols + pad),), fill, device="cuda", dtype=torch.float32 if wide else torch.bfloat16)
            return flat, flat[shift:].view(R, cols + pad)[:, :cols]

        # what lies beside the operands is no number: nothing of it may reach a result
        def operand(cols, pad, std, wide):
            _, view = rows(cols, pad, wide, float("nan"))
            view.copy_(normal(gen, (R, cols), std, wide))
            return view

        def vector(there, mean, std):
            if not there:
                return None
            guarded = torch.full((M + 16,), float("nan"), device="cuda", dtype=torch.float32 if weight32 else torch.bfloat16)
            guarded[:M] = normal(gen, (M,), std, True) + mean
            return guarded[:M]

        self.block = operand(M, pads[0], std, block32)
        self.residual = operand(M, pads[1], 3.0, stream32) if residual else None
        self.gate = None if gate == "none" else operand(1 if gate == "row" else M, pads[2], 1.5, gate32)
        self.aw, self.ab = vector(weights, 1.0 - offset, 0.3), vector(biases, 0.0, 0.1)
        self.bw, self.bb = vector(weights and before != "none", 1.0 - offset, 0.3), vector(biases and before != "none", 0.0, 0.1)
        self.sum_flat, self.sum = rows(M, pads[3], stream32, 3.0) if sums or before == "none" else (None, None)
        self.out_flat, self.out = rows(M, pads[4], out32, 5.0) if before != "none" else (None, None)
        self.R, self.M, self.how = R, M, dict(after=after, before=before, offset=offset, form=form, block_scale=block_scale, residual_scale=residual_scale, eps=eps)
        self.cfg = pkg.NormConfig(features=M, norm_after=KINDS.index(after), norm_before=KINDS.index(before), block_type=int(block32), stream_type=int(stream32),
                                  out_type=int(out32), weight_type=int(weight32), gate_type=int(gate32), gate_form=FORMS.index(form),
                                  gate_per_row=int(gate == "row"), eps=eps, block_scale=block_scale, residual_scale=residual_scale, weight_offset=offset,
                                  block_stride=M + pads[0], residual_stride=M + pads[1], gate_stride=(1 if gate == "row" else M) + pads[2],
                                  sum_stride=M + pads[3], out_stride=M + pads[4])

    def run(self, stream=None):
        import paper_2512_21487_amd as pkg
        pkg.norm(self.cfg, self.block, self.residual, self.gate, self.aw, self.ab, self.bw, self.bb, sum=self.sum, out=self.out, n_rows=self.R, stream=stream)

    def want(self):
        how, u = self.how, 2.0 ** -24
        eps, one, two = (float(torch.tensor(how[k], dtype=torch.float32)) for k in ("eps", "block_scale", "residual_scale"))
        v = self.block.double()
        z, dz = n_of(how["after"], (v, torch.zeros_like(v)), self.aw, self.ab, how["offset"], eps)
        if self.gate is not None:
            g = self.gate.double()
            f = g if how["form"] == "as_is" else torch.sigmoid(g) if how["form"] == "sigmoid" else g * torch.sigmoid(g)
            # exp of an argument that is rounded (half a step of |g| log2 e) and a step of exp2 and reciprocal each
            df = 0.0 * f if how["form"] == "as_is" else f.abs() * u * (2 * g.abs() + 8)
            z, dz = z * f, dz * f.abs() + z.abs() * df + dz * df + 2 * u * (z * f).abs()
        h, dh = one * z, abs(one) * dz + 2 * u * (one * z).abs()
        if self.residual is not None:
            h = h + two * self.residual.double()
            dh = dh + u * h.abs()
        got = {"sum": (h, dh)}
        if self.out is not None:
            got["out"] = n_of(how["before"], (h, dh), self.bw, self.bb, how["offset"], eps)
        return got

    def check(self):
        torch.cuda.synchronize()
        want = self.want()
        for name, flat, view in (("sum", self.sum_flat, self.sum), ("out", self.out_flat, self.out)):
            if view is None:
                continue
            v, dv = want[name]
            bound = dv + (v.abs() + dv) * (2.0 ** -24 if view.dtype == torch.float32 else 2.0 ** -8) + 1e-37
            got = view.double()
            assert bool(torch.isfinite(got).all()), name
            worst = float(((got - v).abs() / bound).max())
            assert worst <= 1.0, f"{name}: {worst} times the bound"
            if flat is not None:
                # nothing but the results was written
                whole = torch.full_like(flat, 3.0 if name == "sum" else 5.0)
                whole[view.storage_offset():].view(self.R, -1)[:, :self.M] = view
                assert torch.equal(whole, flat), name


SIZES = [1, 2, 7, 8, 9, 61, 64, 511, 512, 513, 1024, 1409, 2048, 2055, 4096, 5120, 5121, 8192, 8200, 16384, 20000, 32767, 32768]


@pytest.mark.parametrize("M", SIZES)
@pytest.mark.parametrize("R", [1, 3, 5, 70])
def test_sizes(R, M):
    for wide in (False, True):
        c = Case(R, M, after="rms", before="layer", biases=True, gate="element", form="silu", block32=wide, stream32=wide, out32=wide, gate32=wide, weight32=wide,
                 residual=R != 3)
        c.run()
        c.check()
    c = Case(R, M)
    c.run()
    c.check()


@pytest.mark.parametrize("R,M", [(300, 64), (2100, 64), (2500, 520), (5000, 1024), (257, 1409), (2049, 2048), (1100, 4096), (1500, 5120), (700, 7168), (300, 16384), (257, 30000)])
def test_many_rows(R, M):
    for how in (dict(), dict(after="layer", before="rms", gate="row", form="sigmoid", stream32=True, residual_scale=0.5)):
        c = Case(R, M, **how)
        c.run()
        c.check()


@pytest.mark.parametrize("after", KINDS)
@pytest.mark.parametrize("before", KINDS)
@pytest.mark.parametrize("gate,form", [("none", "as_is")] + [(g, f) for g in ("row", "element") for f in FORMS])
@pytest.mark.parametrize("weights,biases,offset", [(False, False, 1.0), (True, False, 1.0), (True, True, 0.0), (False, True, 0.0)])
@pytest.mark.parametrize("residual", [False, True])
def test_forms(after, before, gate, form, weights, biases, offset, residual):
    for R, M, sums in ((5, 192, True), (9, 1409, before == "none")):
        c = Case(R, M, after=after, before=before, gate=gate, form=form, weights=weights, biases=biases, offset=offset, residual=residual, sums=sums,
                 block_scale=0.22, residual_scale=-0.5)
        c.run()
        c.check()


@pytest.mark.parametrize("block32", [False, True])
@pytest.mark.parametrize("stream32", [False, True])
@pytest.mark.parametrize("out32", [False, True])
@pytest.mark.parametrize("weight32,gate32", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("M,gate", [(640, "element"), (333, "row")])
def test_types(block32, stream32, out32, weight32, gate32, M, gate):
    c = Case(11, M, after="rms", gate=gate, form="sigmoid", block32=block32, stream32=stream32, out32=out32, weight32=weight32, gate32=gate32, biases=True)
    c.run()
    c.check()


@pytest.mark.parametrize("pads", [(8, 8, 8, 8, 8), (1, 0, 0, 0, 0), (0, 3, 0, 0, 0), (0, 0, 5, 0, 0), (0, 0, 0, 7, 0), (0, 0, 0, 0, 9), (4, 12, 20, 36, 1)])
@pytest.mark.parametrize("shift", [0, 1, 4])
@pytest.mark.parametrize("M", [130, 2048, 5119])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("gate", ["row", "element"])
def test_strides_and_alignments(pads, shift, M, wide, gate):
    c = Case(6, M, after="rms", gate=gate, pads=pads, shift=shift, block32=wide, stream32=wide, out32=wide, gate32=wide)
    c.run()
    c.check()


@pytest.mark.parametrize("R,M", [(5, 64), (9, 1409), (300, 2048), (2100, 5120), (7, 16384)])
@pytest.mark.parametrize("wide", [False, True])
def test_results_in_place(R, M, wide):
    """The sum in place of the residual and the norm in place of the block have the bits of results apart."""
    how = dict(after="rms", gate="element", form="silu", block32=wide, stream32=wide, out32=wide)
    apart, c = Case(R, M, **how), Case(R, M, **how)
    apart.run()
    apart.check()
    c.sum, c.out = c.residual, c.block
    c.run()
    torch.cuda.synchronize()
    assert torch.equal(c.sum, apart.sum) and torch.equal(c.out, apart.out)


def test_the_same_bits_again_and_rows_by_themselves():
    c = Case(600, 1409, after="layer", gate="row", form="silu")
    c.run()
    torch.cuda.synchronize()
    first = (c.sum.clone(), c.out.clone())
    for _ in range(3):
        c.run()
        torch.cuda.synchronize()
        assert torch.equal(c.sum, first[0]) and torch.equal(c.out, first[1])
    c.R = 200                                            # fewer rows: those behind stay as they are
    c.sum.fill_(3.0)
    c.out.fill_(5.0)
    c.run()
    torch.cuda.synchronize()
    assert torch.equal(c.sum[:200], first[0][:200]) and bool((c.sum[200:] == 3.0).all())
    assert torch.equal(c.out[:200], first[1][:200]) and bool((c.out[200:] == 5.0).all())


@pytest.mark.parametrize("M", [96, 2048, 9000])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_rows_beyond_fp32_in_their_squares(M, kind):
    """Numbers of 1e30 and of the largest bf16: their squares and sums leave fp32, the norm does not.  Small numbers beside them keep their places."""
    import paper_2512_21487_amd as pkg
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = normal(gen, (6, M), 1.0, True)
    x[0] *= 1e30
    x[1] *= 5e37
    x[2] = 3.3895e38
    x[3] *= 1e-15
    x[4, 0] = 1e32
    x[5] = 0.0
    out = torch.empty((6, M), device="cuda")
    pkg.norm(pkg.NormConfig(features=M, norm_before=KINDS.index(kind), block_type=1, out_type=1, eps=1e-6), x, out=out)
    torch.cuda.synchronize()
    v = x.double()
    c = v - v.mean(dim=1, keepdim=True) if kind == "layer" else v
    want = c / torch.sqrt((c * c).mean(dim=1, keepdim=True) + 1e-6)
    u = 2.0 ** -24
    bound = want.abs() * u * (M / 64 + 32)
    if kind == "layer":
        # the mean is off by its sum's steps and its own; equal numbers leave that alone, which may be more than they are apart
        size = v.abs().mean(dim=1, keepdim=True) * u * (M / 64 + 32)
        power = torch.sqrt((c * c).mean(dim=1, keepdim=True) + 1e-6)
        bound = bound + size / power + want.abs() * size / power
    ok = (out.double() - want).abs() <= bound + 1e-37
    rows = [0, 1, 3, 4, 5] if kind == "layer" else range(6)
    assert bool(ok[list(rows)].all())
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("M", [8, 64, 512, 1024, 2048, 4096, 8192, 16384, 32768])
def test_equal_numbers_beyond_fp32_in_their_sum(M):
    """Powers of two, whose sums and mean are exact in any order: nothing is left of them, and the bias is the result."""
    import paper_2512_21487_amd as pkg
    for rows in (3, 300):
        x = torch.full((rows, M), 2.0 ** 127, device="cuda")
        x[1] = -2.0 ** 120
        bias = torch.arange(M, device="cuda", dtype=torch.float32) - 3.0
        for eps in (1e-20, 1e-6, 1.0):
            out, total = torch.empty_like(x), torch.empty_like(x)
            pkg.norm(pkg.NormConfig(features=M, norm_before=pkg.NORM_LAYER, block_type=1, out_type=1, weight_type=1, eps=eps), x, before_bias=bias, out=out)
            pkg.norm(pkg.NormConfig(features=M, norm_after=pkg.NORM_LAYER, block_type=1, stream_type=1, weight_type=1, eps=eps), x, after_bias=bias, sum=total)
            torch.cuda.synchronize()
            assert torch.equal(out, bias.expand_as(out)) and torch.equal(total, bias.expand_as(out))


def test_numbers_that_are_none_stay_in_their_rows():
    import paper_2512_21487_amd as pkg
    inf, nan = float("inf"), float("nan")
    for M in (64, 4096):
        c, clean = Case(9, M), Case(9, M)
        clean.run()
        c.block[1, 3], c.block[4, M - 1], c.residual[6, 0] = nan, inf, -inf
        c.run()
        torch.cuda.synchronize()
        keep = [0, 2, 3, 5, 7, 8]
        assert torch.equal(c.out[keep], clean.out[keep]) and torch.equal(c.sum[keep], clean.sum[keep])
        assert bool(torch.isnan(c.out[1]).all())
        for row, at in ((4, M - 1), (6, 0)):             # infinite mean square: 0, and infinity over infinity
            assert bool(torch.isnan(c.out[row, at])) and int((c.out[row] == 0).sum()) == M - 1
            assert bool(torch.isinf(c.sum[row, at])) and int(torch.isinf(c.sum[row]).sum()) == 1
    # a closed gate takes a block's finite numbers out, whatever they are
    c = Case(4, 256, before="none", gate="row", form="sigmoid", gate32=True, weights=False)
    c.gate.fill_(-1e4)
    c.run()
    torch.cuda.synchronize()
    assert torch.equal(c.sum, c.residual)


def test_streams_and_graphs():
    c = Case(33, 2048, after="rms", gate="row", form="sigmoid")
    side = torch.cuda.Stream()
    c.run()
    torch.cuda.synchronize()
    want = (c.sum.clone(), c.out.clone())
    c.sum.zero_(), c.out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run()
    side.synchronize()
    assert torch.equal(c.sum, want[0]) and torch.equal(c.out, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    fresh = Case(33, 2048, after="rms", gate="row", form="sigmoid", seed=9)
    for source in (fresh, c, fresh):
        if source is not c:
            c.block.copy_(fresh.block), c.residual.copy_(fresh.residual), c.gate.copy_(fresh.gate)
        c.sum.zero_(), c.out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = (c.sum.clone(), c.out.clone())
        c.run()
        torch.cuda.synchronize()
        assert torch.equal(got[0], c.sum) and torch.equal(got[1], c.out)
        c.check()


def test_offsets_beyond_32_bits():
    """Rows that begin behind 2^31 elements, and behind 2^32 bytes, of every operand."""
    import paper_2512_21487_amd as pkg
    R, M, stride = 520, 64, 1 << 22
    flat = torch.zeros(R * stride, dtype=torch.bfloat16, device="cuda")
    wide = flat.view(R, stride)
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, r = normal(gen, (R, M), 1.0, False), normal(gen, (R, M), 1.0, False)
    block, residual, total, out = (wide[:, at:at + M] for at in (0, 128, 256, 384))
    block.copy_(x), residual.copy_(r)
    pkg.norm(pkg.NormConfig(features=M, norm_before=pkg.NORM_RMS, block_stride=stride, residual_stride=stride, sum_stride=stride, out_stride=stride),
             block, residual, sum=total, out=out)
    want_sum, want = torch.empty_like(x), torch.empty_like(x)
    pkg.norm(pkg.NormConfig(features=M, norm_before=pkg.NORM_RMS), x, r, sum=want_sum, out=want)
    torch.cuda.synchronize()
    assert torch.equal(total, want_sum) and torch.equal(out, want)
    assert not bool(wide[:, 512:600].any())


def test_more_rows_than_a_grid_has_rows_of_threads():
    """2^32 threads are a grid dimension's; a wavefront has a row."""
    import paper_2512_21487_amd as pkg
    R, M = 2 ** 26 + 5, 8
    x = torch.randint(-3, 4, (R, M), device="cuda", dtype=torch.int8).to(torch.bfloat16)
    out = torch.full((R + 1, M), 9.0, dtype=torch.bfloat16, device="cuda")
    pkg.norm(pkg.NormConfig(features=M, norm_before=pkg.NORM_RMS), x, out=out, n_rows=R)
    torch.cuda.synchronize()
    for rows in (slice(0, 1000), slice(R // 2, R // 2 + 1000), slice(R - 1000, R)):
        v = x[rows].double()
        want = v / torch.sqrt(v.square().mean(dim=1, keepdim=True) + 1e-6)
        assert bool(((out[rows].double() - want).abs() <= 1.01 * 2.0 ** -8 * want.abs()).all())   # a rounding to bf16
    assert bool(torch.isfinite(out).all()) and bool((out[R] == 9.0).all())


def test_no_rows_and_refused_memory():
    import paper_2512_21487_amd as pkg
    cfg = pkg.NormConfig(features=64, norm_before=pkg.NORM_RMS)
    x, y = torch.zeros((8, 64), dtype=torch.bfloat16, device="cuda"), torch.full((8, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    assert pkg.norm(cfg, x, out=y, n_rows=0) == 0
    torch.cuda.synchronize()
    assert bool((y == 7.0).all())
    with pytest.raises(ValueError):
        pkg.norm(cfg, x[:, :60], out=y)
    with pytest.raises(ValueError):
        pkg.norm(cfg, x, out=y.cpu())
    host = torch.zeros(8 * 64, dtype=torch.bfloat16)
    with pytest.raises(pkg.MoeEpError, match="out"):
        pkg.norm(cfg, x, out=host.data_ptr())
    with pytest.raises(pkg.MoeEpError, match="overlap"):
        pkg.norm(cfg, x, sum=y, out=y)
    with pytest.raises(pkg.MoeEpError, match="block"):   # an allocation that ends before
        small = torch.zeros(64, dtype=torch.bfloat16, device="cuda")
        pkg.norm(cfg, small.data_ptr(), out=y.data_ptr() + (1 << 44), n_rows=1 << 24)
    before = torch.cuda.current_device()
    with pytest.raises(pkg.MoeEpError) as ei:
        pkg.norm(pkg.NormConfig(features=64, norm_before=pkg.NORM_RMS, device=63), x.data_ptr(), out=y.data_ptr(), n_rows=8)
    assert ei.value.code == -3 and torch.cuda.current_device() == before
