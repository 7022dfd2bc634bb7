"""moe_ep_route where its fp32 selection is furthest from the rule in float64: biases near the ends of fp32."""
import numpy as np
import pytest

from test_gpu_route import BF_LOWEST, FMAX, by_rule, check, normal, run

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("E,groups,top_groups,k", [(61, 1, 1, 6), (72, 8, 8, 5), (128, 1, 1, 8), (256, 4, 2, 8), (512, 1, 1, 16)])
@pytest.mark.parametrize("T", [33, 8300])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_slots_left_to_biases_near_the_lowest_number(E, groups, top_groups, k, T, sigmoid):
    """Experts that the lowest finite biases put last come before those that are not there, of which no slot may be made."""
    s = normal(T, E, E + T)
    s[3::5] = 0.25                                    # alike: the lower expert
    s[4::7, E // 2 + 1] = -np.inf                     # one expert that is not there
    s[5::7, E // 3:] = np.nan
    for lowest in (-FMAX, np.float32(-FMAX * (1 - 2.0 ** -22)), np.float32(-3e38)):
        bias = np.full(E, lowest, np.float32)
        bias[::E // 4] = 0.05 * normal(1, E, 5)[0, ::E // 4]
        check(s, bias, k=k, groups=groups, top_groups=top_groups, sigmoid=sigmoid)
        bias[1], bias[E - 1] = -np.inf, np.nan
        check(s, bias, k=k, groups=groups, top_groups=top_groups, sigmoid=sigmoid)


def groups_rule(s, bias, *, S, top_groups, k, sigmoid):
    """idx of the rule with GROUP_TOP2 in float64, for groups of S >= 2 experts."""
    T, E = s.shape
    s = np.where(s > -FMAX, s.astype(np.float64), -np.inf)
    if sigmoid:
        p = 1.0 / (1.0 + np.exp(-s))
    else:
        p = np.exp(s - s.max(axis=1, keepdims=True))
        p = p / p.sum(axis=1, keepdims=True)
    c = np.where(s > -np.inf, p + bias.astype(np.float64), -np.inf)
    best = -np.sort(-c.reshape(T, E // S, S), axis=2)[:, :, :2]
    value = np.where(best[:, :, 1] > -np.inf, best.sum(axis=2), best[:, :, 0])
    kept = np.argsort(-value, axis=1, kind="stable")[:, :top_groups]
    stays = np.zeros(value.shape, bool)
    np.put_along_axis(stays, kept, True, 1)
    c = np.where(np.repeat(stays, S, axis=1), c, -np.inf)
    idx = np.argsort(-c, axis=1, kind="stable")[:, :k]
    return np.where(np.take_along_axis(c, idx, 1) > -np.inf, idx, -1)


@pytest.mark.parametrize("E,groups", [(32, 8), (64, 4), (24, 3)])
@pytest.mark.parametrize("T", [50, 8500])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_groups_whose_sum_is_beyond_fp32(E, groups, T, sigmoid):
    """Two lowest biases add up to what fp32 does not hold; such a group still comes before one without an expert, and two largest before two smaller ones."""
    S = E // groups
    s = normal(T, E, E + T)
    s[:, :S] = -np.inf                                # the first group has no expert
    s[2::3, S:2 * S - 1] = np.nan                     # the second but one, sometimes
    keep = min(S, 5)
    s[:, 2 * S + keep:3 * S] = -np.inf
    bias = np.full(E, -FMAX, np.float32)
    bias[2 * S:3 * S] = 0.1
    for top_groups, k in ((2, keep + 1), (1, 2)):
        _, idx, _ = run(s, bias, k=k, groups=groups, top_groups=top_groups, top2=True, sigmoid=sigmoid)
        assert np.array_equal(idx, groups_rule(s, bias, S=S, top_groups=top_groups, k=k, sigmoid=sigmoid))
    bias = np.linspace(2e38, 3.4e38, E).astype(np.float32)
    bias[E // 2:] = bias[:E // 2][::-1]
    _, idx, _ = run(s, bias, k=2, groups=groups, top_groups=1, top2=True, sigmoid=sigmoid)
    assert np.array_equal(idx, groups_rule(s, bias, S=S, top_groups=1, k=2, sigmoid=sigmoid))


@pytest.mark.parametrize("opposite", [64.3, 1000.0, 3e5])
@pytest.mark.parametrize("T", [8000, 30000])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_groups_whose_two_best_nearly_cancel(opposite, T, sigmoid):
    """A group's sum may be far smaller than the two numbers that were rounded for it."""
    E, S = 16, 2
    s = normal(T, E, 31)
    # one of many such tokens: in fp32 the second group's sum is the larger one
    s[0] = np.float32([-0.98689717, 0.34717762, -0.43605295, -0.14113410] * 4)
    bias = np.tile(np.float32([opposite, -(opposite - 0.4)]), E // S)
    for top_groups, k in ((1, 2), (3, 5)):
        _, idx, _ = run(s, bias, k=k, groups=E // S, top_groups=top_groups, top2=True, sigmoid=sigmoid)
        assert np.array_equal(idx, groups_rule(s, bias, S=S, top_groups=top_groups, k=k, sigmoid=sigmoid))


# p is less than a step of fp32 beside a bias of 1, or a sigmoid's 1 but for one that double alone holds
def steps_below_fp32(rng, T, E, sigmoid):
    if sigmoid:
        return rng.choice(np.float32([20.0, 24.0, 30.5, 33.0, 36.0, 41.25, 50.25, np.inf]), (T, E)), np.full(E, 1.0, np.float32)
    s = rng.choice(np.float32([-19.0, -19.5, -20.0, -20.5, -21.0, -22.0]), (T, E))
    s[:, E // 2] = 0.0                                # most of the sum; never chosen
    bias = np.full(E, 1.0, np.float32)
    bias[E // 2] = -3.0
    return s, bias


@pytest.mark.parametrize("E,k,there", [(20, 5, 8), (64, 3, 7), (64, 1, 5), (128, 6, 8), (96, 10, 16)])
@pytest.mark.parametrize("T", [2000, 9000])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_a_better_expert_behind_some_that_are_alike(E, k, there, T, sigmoid):
    """The last slot and those next to it may be alike and one behind them be ahead of all in double."""
    rng = np.random.default_rng(E + k)
    s, bias = steps_below_fp32(rng, T, E, sigmoid)
    order = np.argsort(rng.random((T, E)), axis=1)
    np.put_along_axis(s, order[:, there:], -np.inf, 1)
    check(s, bias, k=k, sigmoid=sigmoid)
    # in every token alike but for the last one, so that no other pair of a token beside it has the order looked at
    np.put_along_axis(s, order[:, :there], np.float32(30.5 if sigmoid else -19.5), 1)
    np.put_along_axis(s, order[:, :there].max(axis=1, keepdims=True), np.float32(41.25 if sigmoid else -19.0), 1)
    check(s, bias, k=k, sigmoid=sigmoid)


@pytest.mark.parametrize("E,k", [(20, 5), (61, 8), (64, 3), (128, 8), (96, 12)])
@pytest.mark.parametrize("T", [2000, 9000])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_experts_alike_that_only_double_tells_from_others(E, k, T, sigmoid):
    """Of several experts with one score one may be the last that fp32 keeps, and be ahead of the rest in double: the others come with it."""
    rng = np.random.default_rng(E + k)
    s, bias = steps_below_fp32(rng, T, E, sigmoid)
    s[rng.random((T, E)) < 1.0 - (k + 4.0) / E] = -np.inf   # about as many as the lists are long
    check(s, bias, k=k, sigmoid=sigmoid)


@pytest.mark.parametrize("E,k", [(12, 4), (64, 6)])
@pytest.mark.parametrize("T", [3000, 9000])
def test_softmax_values_a_step_of_double_apart(E, k, T):
    """Which of two values, equal or a step of double apart, is the larger one is also what double says, with a sum in double."""
    rng = np.random.default_rng(E)
    s = np.full((T, E), -40.0, np.float32)
    s[:, :3] = 0.3 * rng.standard_normal((T, 3))      # most of the sum; never chosen
    near = (np.float32(-23.5).view(np.int32) + rng.integers(0, 40, (T, 8))).astype(np.int32).view(np.float32)
    s[:, 4:12] = near                                 # p of 2^-35 or so: a step of the score is half a step of 1 + p
    bias = np.full(E, -5.0, np.float32)
    bias[4:12] = 1.0
    check(s, bias, k=k)


def test_choices_by_rules_and_values_of_all_kinds():
    """Rules and shapes drawn at random, scores and biases from tiny to the ends of fp32, many of them equal, infinite or not there."""
    rng = np.random.default_rng(77)
    pick = lambda *a: a[rng.integers(len(a))]
    for _ in range(150):
        G = pick(1, 1, 1, 2, 3, 4, 8, 16, 32)
        S = max(1, min(int(pick(1, 2, 3, 4, 8, 9, 16, 32, 61, 128)), 512 // G))
        E, top_groups, T = G * S, int(rng.integers(1, G + 1)), int(pick(1, 7, 65, 200))
        k = int(rng.integers(1, min(pick(8, 8, 16, 64), S * top_groups) + 1))
        s = (rng.standard_normal((T, E)) * pick(1e-6, 0.05, 1, 1, 8, 50, 1e4, 1e37)).astype(np.float32)
        if rng.random() < 0.3:
            s = np.round(s * 4) / 4
        if rng.random() < 0.4:
            s[rng.random((T, E)) < pick(0.02, 0.5, 0.95)] = pick(-np.inf, np.nan, -FMAX)
        if rng.random() < 0.2:
            s[rng.random((T, E)) < 0.05] = np.inf
        bias = None
        if rng.random() < 0.75:
            bias = np.clip(rng.standard_normal(E) * pick(0.0, 1e-7, 0.05, 0.05, 1, 64, 1000, 1e6, 1e30, 1e38), -3.4e38, 3.4e38).astype(np.float32)
            if rng.random() < 0.3:
                bias[rng.random(E) < pick(0.1, 0.7, 0.95)] = pick(-FMAX, FMAX, np.inf, -np.inf, np.nan, -3e38, 0.0)
        how = dict(k=k, groups=G, top_groups=top_groups, top2=bool(rng.random() < 0.6), sigmoid=bool(rng.random() < 0.5), renorm=True)
        bf16 = bool(rng.random() < 0.3)
        read, idx, w = run(s, bias, bf16=bf16, **how)
        want, _ = by_rule(read, bias, None, lowest=BF_LOWEST if bf16 else -FMAX, **how)
        assert np.array_equal(idx, want), how
        assert np.all(w >= 0.0) and np.all(w[idx < 0] == 0.0)
