"""The window attention and rotary oracles against small hand-made cases and
differences (CPU only)."""
import numpy as np
import pytest

from oracle import rope as orope
from oracle import window as owin


def test_visible_keys_by_hand():
    # 5 queries over 7 keys: query 0 lies at position 2
    assert owin.visible(0, 5, 7, 1, 0, 0).tolist() == [1, 2]
    assert owin.visible(4, 5, 7, 1, 0, 1).tolist() == [0, 5, 6]
    assert owin.visible(1, 5, 7, 0, 2, 2).tolist() == [0, 1, 3, 4, 5]
    assert owin.visible(4, 5, 7, -1, -1, 0).tolist() == list(range(7))
    # more queries than keys: the first ones lie before the first key
    assert owin.visible(0, 5, 3, 4, 0, 2).tolist() == []
    assert owin.visible(1, 5, 3, 4, 1, 0).tolist() == [0]


def test_one_visible_key_returns_its_value():
    rng = np.random.default_rng(0)
    q, k, v = (rng.standard_normal((1, 3, 1, 4)) for _ in range(3))
    r = owin.window_attention(q, k, v, 0, 0, 0)
    assert np.allclose(r["o"], v) and np.allclose(r["lse"][0, 0], (q * k).sum(-1)[0, :, 0] / 2)


def test_masked_values_enter_no_sum():
    rng = np.random.default_rng(1)
    q, k, v = (rng.standard_normal((1, 4, 1, 4)) for _ in range(3))
    k[0, 0], v[0, 0] = np.nan, np.inf
    r = owin.window_attention(q[:, 2:], k, v, 1, 0, 0)  # positions 2 and 3 see keys 1 to 3
    assert np.all(np.isfinite(r["o"]))


@pytest.mark.parametrize("name", ["q", "k", "v"])
def test_gradients_match_differences(name):
    rng = np.random.default_rng(2)
    x = dict(q=rng.standard_normal((2, 5, 4, 6)), k=rng.standard_normal((2, 7, 2, 6)), v=rng.standard_normal((2, 7, 2, 6)))
    do = rng.standard_normal(x["q"].shape)
    lens = dict(q_len=[5, 3], kv_len=[7, 2])

    def loss():
        o = owin.window_attention(x["q"], x["k"], x["v"], 2, 1, 1, **lens)["o"]
        return float(np.nansum(o * do))

    g = owin.window_attention(x["q"], x["k"], x["v"], 2, 1, 1, do=do, **lens)["d" + name]
    for at in [(0, 0, 0, 0), (0, 2, 1, 3), (0, 4, 0, 5), (1, 1, 1, 2)]:
        keep = x[name][at]
        d = []
        for s in (1e-5, -1e-5):
            x[name][at] = keep + s
            d.append(loss())
        x[name][at] = keep
        assert abs((d[0] - d[1]) / 2e-5 - g[at]) < 1e-7, (at, g[at])


def test_rotation_by_hand_and_inverse():
    x = np.array([[[1.0, 0.0, 2.0, 3.0, 5.0, 7.0]]])
    y = orope.rotate(x, [[2], [1]], [np.pi / 4, np.pi], (1, 1), True)
    assert np.allclose(y[0, 0], [0, 1, -2, -3, 5, 7])
    z = orope.rotate(x, [[2], [1]], [np.pi / 4, np.pi], (1, 1), False)
    assert np.allclose(z[0, 0], [-2, -0.0, 1, -3, 5, 7])
    assert np.allclose(orope.rotate(y, [[2], [1]], [np.pi / 4, np.pi], (1, 1), True, inverse=True), x)
    pos, inside = orope.grid_positions(8, (1, 2, 3), (4, 0, 0))
    assert pos[:, 5].tolist() == [4, 1, 2] and inside.tolist() == [True] * 6 + [False] * 2
