"""The bound of continuation_values: a plain attention that rounds as the kernels do is within it, one with a mistake planted is not."""
import numpy as np
import pytest

from tests import continuation_oracle as orc
from tests import continuation_values as val


def rounded(q, k, v, scale, tile=128, v_used=None):
    """The running softmax over tiles with bf16 weights for the product and unrounded ones for the sum (v_used: the values that it takes instead)."""
    v_used = v if v_used is None else v_used
    G, D = q.shape
    m, z, o = np.full(G, -np.inf), np.zeros(G), np.zeros((G, D))
    for t in range(0, len(k), tile):
        s = q @ k[t:t + tile].T * scale
        new = np.maximum(m, s.max(-1))
        a, p = np.exp(m - new), np.exp(s - new[:, None])
        z, o, m = z * a + p.sum(-1), o * a[:, None] + orc.to_bf16(p) @ v_used[t:t + tile], new
    return orc.to_bf16(o / z[:, None])


def data(n, seed, places):
    rng = np.random.default_rng(seed)
    q, k, v = (orc.to_bf16(rng.standard_normal(s)) for s in ((4, 128), (n, 128), (n, 128)))
    v[places] = orc.to_bf16(v[places] * 64)
    return q, k, v


@pytest.mark.parametrize("n", [1, 2, 65, 500, 4000, 16500])
def test_rounding_alone_is_within_the_bound(n):
    for seed in range(3):
        places = [i for i in (0, 63, 64, 127, 128, n // 2, n - 1) if i < n]
        q, k, v = data(n, seed, places)
        assert val.check(rounded(q, k, v, 128 ** -0.5), q, k, v, 128 ** -0.5).all()


@pytest.mark.parametrize("n", [500, 4000, 16500])
@pytest.mark.parametrize("what", ["lost", "exchanged", "twice", "neighbour"])
def test_one_value_row_out_of_place_is_not(n, what):
    places = [127, 128, n // 2, n - 1]
    q, k, v = data(n, 7, places)
    for i in places:
        wrong = v.copy()
        if what == "lost":
            wrong[i] = 0
        elif what == "exchanged":
            j = i - 1 if i == n - 1 else i + 1
            wrong[[i, j]] = wrong[[j, i]]
        elif what == "twice":
            wrong[i - 2] = v[i]
        else:
            wrong[i] = v[i - 3]
        assert not val.check(rounded(q, k, v, 128 ** -0.5, v_used=wrong), q, k, v, 128 ** -0.5).all(), i
