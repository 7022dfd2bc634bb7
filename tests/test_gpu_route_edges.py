"""moe_ep_route where its fp32 selection is furthest from the rule in float64: biases near the ends of fp32."""
import numpy as np
import pytest

from test_gpu_route import FMAX, check, normal

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
