"""moe_ep_route against the rule in float64: choices exactly, weights within the rounding of fp32."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

FMAX, BF_LOWEST = np.finfo(np.float32).max, -3.3895313892515355e38


def by_rule(scores, bias, mask, *, k, groups=1, top_groups=1, top2=False, sigmoid=False, renorm=True, scale=1.0, lowest=-FMAX):
    """(idx, w) of the documented rule; scores as float64 values of what the kernel reads."""
    T, E = scores.shape
    gone = ~(scores > lowest)
    if bias is not None:
        gone = gone | ~(bias > -np.inf)[None, :]
    if mask is not None:
        gone = gone | (mask == 0)[:, None]
    s = np.where(gone, -np.inf, np.minimum(scores, FMAX))
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        if sigmoid:
            p = 1.0 / (1.0 + np.exp(-s))
        else:
            top = s.max(axis=1, keepdims=True)
            p = np.where(gone, 0.0, np.exp(s - np.where(np.isfinite(top), top, 0.0)))
            total = p.sum(axis=1, keepdims=True)
            p = p / np.where(total > 0, total, 1.0)
        c = np.where(gone, -np.inf, p + (bias.astype(np.float64) if bias is not None else 0.0))
    order = (c if bias is not None else s).copy()
    if groups > 1:
        S = E // groups
        for t in range(T):
            value = np.full(groups, -np.inf)
            for g in range(groups):
                members = c if (bias is not None or top2) else s
                m = np.sort(members[t, g * S:(g + 1) * S])[::-1]
                value[g] = m[0] + (m[1] if top2 and S > 1 and m[1] > -np.inf else 0.0)
            kept = np.argsort(-value, kind="stable")[:top_groups]
            for g in range(groups):
                if g not in kept:
                    order[t, g * S:(g + 1) * S] = -np.inf
    idx = np.argsort(-order, axis=1, kind="stable")[:, :k].astype(np.int32)
    full = np.take_along_axis(order, idx, 1) > -np.inf
    w = np.where(full, np.take_along_axis(p, idx, 1), 0.0)
    if renorm:   # by logarithms: every p of a choice may be too small even for float64
        si = np.where(full, np.take_along_axis(s, idx, 1), -np.inf)
        log_p = np.minimum(si, 0.0) - np.log1p(np.exp(-np.abs(si))) if sigmoid else si
        top = log_p.max(axis=1, keepdims=True)
        w = np.where(full, np.exp(log_p - np.where(top > -np.inf, top, 0.0)), 0.0)
        total = w.sum(axis=1, keepdims=True)
        w = w / np.where(total > 0, total, 1.0)
    return np.where(full, idx, -1), w * scale


def weight_bound(scores, k):
    """Relative: exp of a rounded difference is off by the difference's rounding, half a step of up to the scores' range; exp and
    division are within two steps each; sums of k or E numbers in a tree add a half step per level (k in turn at most)."""
    finite = scores[np.isfinite(scores) & (np.abs(scores) < 1e30)]
    span = float(finite.max() - finite.min()) if finite.size else 0.0
    return (span / 2 + k + 16) * 2.0 ** -23


def run(scores, bias=None, mask=None, *, k, groups=1, top_groups=1, top2=False, sigmoid=False, renorm=True, scale=1.0, bf16=False, stride=0,
        stream=None):
    import paper_2512_21487_amd as pkg
    T, E = scores.shape
    wide = torch.full((T, stride or E), 7.5, dtype=torch.float32)
    wide[:, :E] = torch.from_numpy(np.ascontiguousarray(scores, dtype=np.float32))
    dev = wide.cuda().to(torch.bfloat16 if bf16 else torch.float32)
    b = torch.from_numpy(bias).cuda() if bias is not None else None
    m = torch.from_numpy(mask).cuda() if mask is not None else None
    # what lies behind the last token stays as it was
    idx = torch.full(((T + 2) * k,), 12345, dtype=torch.int32, device="cuda")
    w = torch.full(((T + 2) * k,), 0.25, dtype=torch.float32, device="cuda")
    rule = pkg.Routing(n_experts=E, top_k=k, n_groups=groups, top_groups=top_groups, group_score=int(top2), score=int(sigmoid),
                       renormalise=int(renorm), scale=scale, score_type=pkg.BF16 if bf16 else pkg.F32, score_stride=stride)
    torch.cuda.synchronize()
    pkg.route(rule, dev[:, :E], b, m, n_tokens=T, idx=idx, w=w, stream=stream)
    torch.cuda.synchronize()
    assert bool((idx[T * k:] == 12345).all()) and bool((w[T * k:] == 0.25).all())
    read = dev[:, :E].double().cpu().numpy()
    return read, idx[:T * k].view(T, k).cpu().numpy(), w[:T * k].view(T, k).cpu().numpy()


def check(scores, bias=None, mask=None, **kw):
    how = {n: kw[n] for n in ("k", "groups", "top_groups", "top2", "sigmoid", "renorm", "scale") if n in kw}
    read, idx, w = run(scores, bias, mask, **kw)
    want_idx, want_w = by_rule(read, bias, mask, lowest=BF_LOWEST if kw.get("bf16") else -FMAX, **how)
    assert np.array_equal(idx, want_idx)
    bound = weight_bound(read, how["k"])
    assert np.all(np.abs(w - want_w) <= bound * want_w + 1e-37)
    assert np.all(w[idx < 0] == 0.0)


def normal(T, E, seed):
    return np.random.default_rng(seed).standard_normal((T, E)).astype(np.float32)


@pytest.mark.parametrize("T", [1, 2, 3, 4, 7, 16, 33, 64, 1001])
@pytest.mark.parametrize("E,k", [(1, 1), (2, 2), (7, 3), (16, 8), (61, 5), (64, 6), (65, 16), (128, 8), (160, 6), (255, 9), (256, 8), (512, 64)])
@pytest.mark.parametrize("sigmoid,with_bias", [(False, False), (False, True), (True, False), (True, True)])
def test_choice_over_all_experts(T, E, k, sigmoid, with_bias):
    s = normal(T, E, 1000 * E + T)
    bias = (0.05 * normal(1, E, E)[0]) if with_bias else None
    check(s, bias, k=k, sigmoid=sigmoid, renorm=(T + E) % 2 == 0, scale=2.5 if E % 2 else 1.0)


@pytest.mark.parametrize("E,groups,top_groups,k", [(8, 8, 3, 3), (16, 2, 1, 8), (64, 16, 2, 7), (64, 64, 8, 8), (96, 3, 2, 5), (160, 8, 3, 6),
                                                   (256, 8, 4, 8), (256, 4, 2, 16), (256, 32, 5, 8), (512, 16, 16, 32), (488, 8, 7, 8)])
@pytest.mark.parametrize("top2", [False, True])
@pytest.mark.parametrize("sigmoid,with_bias", [(False, False), (True, False), (True, True), (False, True)])
def test_choice_inside_groups(E, groups, top_groups, k, top2, sigmoid, with_bias):
    for T in (1, 37, 300):
        s = normal(T, E, E + T + groups)
        bias = (0.1 * normal(1, E, E)[0]) if with_bias else None
        check(s, bias, k=k, groups=groups, top_groups=top_groups, top2=top2, sigmoid=sigmoid, renorm=True, scale=1.5)


@pytest.mark.parametrize("E,groups,top_groups,k", [(128, 1, 1, 8), (61, 1, 1, 5), (160, 8, 3, 6)])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("extra", [0, 1, 3, 8, 64])
def test_types_and_rows_that_lie_apart(E, groups, top_groups, k, bf16, extra):
    """Equal scores are common in bf16: the lower expert goes first."""
    s = normal(200, E, E + extra)
    check(s, None, k=k, groups=groups, top_groups=top_groups, bf16=bf16, stride=E + extra)
    check(s, 0.05 * normal(1, E, 3)[0], k=k, groups=groups, top_groups=top_groups, top2=True, sigmoid=True, bf16=bf16, stride=E + extra)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("groups,top_groups,top2", [(1, 1, False), (4, 2, False), (4, 2, True)])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("bf16", [False, True])
def test_experts_and_tokens_that_are_not_there(sigmoid, groups, top_groups, top2, with_bias, bf16):
    T, E, k = 96, 32, 6
    rng = np.random.default_rng(5)
    s = normal(T, E, 6)
    s[0] = -np.inf                                   # nobody is there
    s[1] = np.nan
    s[2] = BF_LOWEST if bf16 else -FMAX
    s[3, 3:] = -np.inf                               # fewer than k
    s[4, 1:] = np.nan                                # one
    s[5, : E // 2] = -np.inf                         # whole groups
    s[6] = np.inf                                    # all alike, the largest number
    s[7, 4] = np.inf
    s[8] = 0.0
    s[8, ::2] = -0.0                                 # both zeros are equal
    s[9] = -1e4                                      # p of the sigmoid is 0 in every type
    s[10] = 1e4
    s[11:20][rng.random((9, E)) < 0.7] = -np.inf
    bias = None
    if with_bias:
        bias = 0.05 * normal(1, E, 7)[0]
        bias[3], bias[9], bias[30], bias[31] = np.nan, -np.inf, np.inf, 1e30
    mask = (rng.random(T) < 0.8).astype(np.uint8) * 3
    mask[:12] = 1
    check(s, bias, mask, k=k, groups=groups, top_groups=top_groups, top2=top2, sigmoid=sigmoid, bf16=bf16)
    check(s[20:], bias, np.zeros(T - 20, np.uint8), k=k, groups=groups, top_groups=top_groups, top2=top2, sigmoid=sigmoid, bf16=bf16)


def test_values_that_fp32_cannot_tell_apart():
    """Pairs of experts whose p + bias differ by less than fp32 resolves, within the choice and at its end."""
    T, E, k = 3000, 64, 4
    rng = np.random.default_rng(11)
    s = np.full((T, E), -6.0, np.float32) - rng.random((T, E)).astype(np.float32)
    bias = np.zeros(E, np.float32)
    bias[1::2] = 0.125
    sig = lambda v: 1.0 / (1.0 + np.exp(-np.asarray(v, np.float64)))
    pairs = [(0, 1), (10, 21), (40, 7)]
    for n, (a, b) in enumerate(pairs):               # three pairs of close values: the fourth place is inside the second pair
        s[:, a] = (2.0 - n + 0.1 * rng.random(T)).astype(np.float32)
        target = sig(s[:, a]) + bias[a] - bias[b]
        s[:, b] = np.log(target / (1.0 - target)).astype(np.float32)
    near = np.abs((sig(s[:, 0]) + bias[0]) - (sig(s[:, 1]) + bias[1]))
    assert np.median(near) < 2.0 ** -24 and np.all(near > 0)
    check(s, bias, k=k, sigmoid=True)
    check(s, bias, k=3, sigmoid=True)


def test_groups_that_fp32_cannot_tell_apart():
    """Two groups whose sums of two values differ by less than fp32 resolves."""
    T, E = 2000, 64
    rng = np.random.default_rng(12)
    s = np.full((T, E), -4.0, np.float32) - rng.random((T, E)).astype(np.float32)
    sig = lambda v: 1.0 / (1.0 + np.exp(-np.asarray(v, np.float64)))
    s[:, 2], s[:, 5] = (1.0 + 0.1 * rng.random((2, T))).astype(np.float32)
    s[:, 33] = (1.05 + 0.02 * rng.random(T)).astype(np.float32)
    rest = sig(s[:, 2]) + sig(s[:, 5]) - sig(s[:, 33])
    s[:, 34] = np.log(rest / (1.0 - rest)).astype(np.float32)
    for bias in (None, np.full(E, 0.25, np.float32)):
        check(s, bias, k=2, groups=8, top_groups=1, top2=True, sigmoid=True)
        check(s, bias, k=5, groups=8, top_groups=4, top2=True, sigmoid=True)


def test_equal_values_in_every_place():
    for E, groups, top_groups in ((128, 1, 1), (256, 8, 4), (61, 1, 1)):
        s = np.zeros((50, E), np.float32)
        s[10:] = np.round(normal(40, E, 3) * 2) / 2
        for bias in (None, np.zeros(E, np.float32)):
            for sigmoid in (False, True):
                check(s, bias, k=8, groups=groups, top_groups=top_groups, top2=True, sigmoid=sigmoid)


def test_weights_of_choices_that_are_improbable():
    """A bias can choose experts whose p is below what fp32 holds; renormalised weights are still their proportions."""
    s = normal(64, 32, 9)
    s[:, 8:] += 90.0
    bias = np.zeros(32, np.float32)
    bias[:8] = 4.0
    check(s, bias, k=4)
    s = normal(64, 32, 10) - 95.0
    check(s, bias, k=4, sigmoid=True)


def test_streams_graphs_and_repeats():
    import paper_2512_21487_amd as pkg
    T, E, k = 513, 128, 8
    rule = pkg.Routing(n_experts=E, top_k=k, score=pkg.SCORE_SIGMOID, renormalise=1, score_type=pkg.F32)
    a, b = torch.from_numpy(normal(T, E, 21)).cuda(), torch.from_numpy(normal(T, E, 22)).cuda()
    bias = torch.from_numpy(0.05 * normal(1, E, 23)[0]).cuda()
    new = lambda: (torch.zeros((T, k), dtype=torch.int32, device="cuda"), torch.zeros((T, k), device="cuda"))
    want = {}
    for n, s in (("a", a), ("b", b)):
        idx, w = new()
        pkg.route(rule, s, bias, idx=idx, w=w)
        torch.cuda.synchronize()
        want[n] = (idx, w)
    side = [torch.cuda.Stream() for _ in range(2)]
    got = {n: new() for n in "ab"}
    torch.cuda.synchronize()
    for _ in range(5):                               # two streams at once
        for st, (n, s) in zip(side, (("a", a), ("b", b))):
            pkg.route(rule, s, bias, idx=got[n][0], w=got[n][1], stream=st.cuda_stream)
    torch.cuda.synchronize()
    for n in "ab":
        assert torch.equal(got[n][0], want[n][0]) and torch.equal(got[n][1], want[n][1])
    held, (idx, w) = a.clone(), new()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pkg.route(rule, held, bias, idx=idx, w=w)
    for n, s in (("a", a), ("b", b), ("a", a)):
        held.copy_(s)
        other = new()
        pkg.route(rule, b, bias, idx=other[0], w=other[1])   # eager work between the replays
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(idx, want[n][0]) and torch.equal(w, want[n][1])


def test_buffers_that_are_too_small_or_elsewhere():
    import paper_2512_21487_amd as pkg
    rule = pkg.Routing(n_experts=64, top_k=6, score_type=pkg.F32)
    s = torch.zeros((8, 64), device="cuda")
    idx, w = torch.zeros(48, dtype=torch.int32, device="cuda"), torch.zeros(48, device="cuda")
    with pytest.raises(ValueError):
        pkg.route(rule, s, idx=idx[:40], w=w)
    with pytest.raises(ValueError):
        pkg.route(rule, s[:, :60], idx=idx, w=w)
    host = np.zeros((8, 64), np.float32)
    with pytest.raises(pkg.MoeEpError, match="scores"):
        pkg.route(rule, host.ctypes.data, n_tokens=8, idx=idx, w=w)
    before = torch.cuda.current_device()
    with pytest.raises(pkg.MoeEpError) as ei:
        pkg.route(pkg.Routing(n_experts=64, top_k=6, score_type=pkg.F32, device=63), s, idx=idx, w=w)
    assert ei.value.code == -3 and torch.cuda.current_device() == before
    pkg.route(rule, s, idx=idx, w=w)
    torch.cuda.synchronize()
    assert idx.view(8, 6)[0].tolist() == [0, 1, 2, 3, 4, 5]


@pytest.mark.parametrize("T", [8191, 8192, 8193, 9001])
@pytest.mark.parametrize("E,groups,top_groups,k", [(64, 1, 1, 6), (61, 1, 1, 8), (128, 8, 3, 8), (160, 2, 1, 5), (256, 1, 1, 8), (256, 16, 4, 8)])
@pytest.mark.parametrize("sigmoid,with_bias,top2", [(False, False, False), (True, True, True), (False, True, False), (False, False, True)])
def test_many_tokens(T, E, groups, top_groups, k, sigmoid, with_bias, top2):
    """Fewer lanes have a token from some number of tokens on.  Rows of every kind among ordinary ones: nobody there, few, equal, huge."""
    s = normal(T, E, T + E)
    if E % 2:                                        # equal scores, as bf16 has many
        s = np.round(s * 16) / 16
    s[5::97, 2:] = -np.inf
    s[6::101] = np.nan
    s[7::103] = 0.25
    s[8::107, ::2] = -FMAX
    s[9::109] = np.inf
    s[10::113] = -1e4
    bias = None
    if with_bias:
        bias = 0.05 * normal(1, E, 7)[0]
        bias[3], bias[E // 2] = -np.inf, bias[1]
    mask = (np.random.default_rng(T).random(T) < 0.9).astype(np.uint8)
    check(s, bias, mask if k < 8 else None, k=k, groups=groups, top_groups=top_groups, top2=top2, sigmoid=sigmoid, renorm=True, scale=1.5)


@pytest.mark.parametrize("T,E,groups", [(2 ** 29 + 5, 2, 1), (2 ** 26 + 5, 3, 3)])
def test_more_tokens_than_a_grid_has_rows_of_threads(T, E, groups):
    """2^32 threads are a grid dimension's; eight lanes, or a wavefront, have a token."""
    import paper_2512_21487_amd as pkg
    s = torch.randint(0, 7, (T, E), device="cuda", dtype=torch.int8).to(torch.bfloat16)
    idx = torch.full((T + 1, 1), 9, dtype=torch.int32, device="cuda")
    w = torch.full((T + 1, 1), 9.0, dtype=torch.float32, device="cuda")
    pkg.route(pkg.Routing(n_experts=E, top_k=1, n_groups=groups, top_groups=1, renormalise=1, scale=1.5, score_type=pkg.BF16), s, n_tokens=T, idx=idx, w=w)
    want = torch.zeros(T, dtype=torch.int32, device="cuda")
    best = s[:, 0].clone()
    for e in range(1, E):
        more = s[:, e] > best
        want[more] = e
        best = torch.maximum(best, s[:, e])
    torch.cuda.synchronize()
    assert torch.equal(idx[:T, 0], want) and bool((w[:T] == 1.5).all())
    assert int(idx[T]) == 9 and float(w[T]) == 9.0
