"""Checks of the serving oracle itself (CPU): the rotation and its transposed map, the 8-bit format, the cache."""
import math

import numpy as np
import pytest
import torch

from oracle import prism_oracle as orc
from oracle import serving_oracle as so


def test_interleaved_full_rotation_is_the_papers():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((3, 17, 128))
    for yarn in (None, (32768, 4.0, 1.0, 32.0)):
        theta = orc.rope_frequencies(128, 1e6, yarn=yarn)
        np.testing.assert_allclose(so.frequencies(1e6, 128, yarn), theta, rtol=1e-13)
        np.testing.assert_allclose(so.rotate(x, np.arange(17) + 1000, theta, False), orc.apply_rope(x, theta, 1000), atol=1e-12)


def test_half_layout_is_interleaved_with_dims_moved():
    rng = np.random.default_rng(1)
    x, rot = rng.standard_normal((2, 9, 64)), 48
    theta = so.frequencies(1e4, rot)
    order = np.r_[np.arange(0, rot, 2), np.arange(1, rot, 2), np.arange(rot, 64)]      # dim of the half layout -> interleaved dim
    inter = so.rotate(x, np.arange(9), theta, False)
    half = so.rotate(x[..., order], np.arange(9), theta, True)
    np.testing.assert_allclose(half, inter[..., order], atol=1e-13)


@pytest.mark.parametrize("half", [False, True])
def test_backward_is_the_gradient(half):
    """Against differences of the forward map, which is linear: exact up to rounding."""
    rng = np.random.default_rng(2)
    x, g = rng.standard_normal((1, 3, 64)), rng.standard_normal((1, 3, 64))
    theta, pos = so.frequencies(1e4, 32), np.array([5, 0, 70000])
    back = so.rotate(g, pos, theta, half, 1.3, backward=True)
    step = 1e-3
    for at in [(0, 0, 0), (0, 0, 17), (0, 1, 3), (0, 2, 31), (0, 2, 40)]:
        up, down = x.copy(), x.copy()
        up[at] += step
        down[at] -= step
        diff = (so.rotate(up, pos, theta, half, 1.3) - so.rotate(down, pos, theta, half, 1.3)) / (2 * step)
        assert abs((diff * g).sum() - back[at]) < 1e-10


def test_e4m3_rounding_is_torchs():
    rng = np.random.default_rng(3)
    x = np.concatenate([rng.standard_normal(4000) * 2.0 ** rng.integers(-12, 8, 4000), so.e4m3_values(),
                        (so.e4m3_values()[1:] + so.e4m3_values()[:-1]) / 2, [np.nan, 0.0, -0.0, 1e-9]])
    x = x[~(np.abs(x) > 448)]
    ref = torch.from_numpy(x).float().to(torch.float8_e4m3fn).double().numpy()
    got = so.to_e4m3(x.astype(np.float32).astype(np.float64))
    np.testing.assert_array_equal(got, ref)


def test_scales():
    assert so.scale_for(0.0) == 2.0 ** -120
    assert so.scale_for(448.0) == 1.0 and so.scale_for(448.0001) == 2.0 and so.scale_for(447.0) == 1.0
    assert so.scale_for(224.0) == 0.5 and so.scale_for(3.5) == 2.0 ** -7


def test_attention_against_softmax_and_empty_rows():
    rng = np.random.default_rng(4)
    k, v = rng.standard_normal((3, 2, 32, 64)), rng.standard_normal((3, 2, 32, 64))
    table = np.array([[2, 0], [1, -1]])
    q = rng.standard_normal((4, 4, 64))
    out, lse, _, _ = so.attention(q, k, v, [40, 1], [0, 2, 3], table)
    kk = np.concatenate([k[2, 1], k[0, 1, :8]])
    vv = np.concatenate([v[2, 1], v[0, 1, :8]])
    x = kk @ q[3, 1] / 8.0
    p = np.exp(x) / np.exp(x).sum()
    np.testing.assert_allclose(out[3, 1], p @ vv, atol=1e-12)
    assert math.isclose(lse[3, 1], math.log(np.exp(x).sum()), rel_tol=1e-12)
    np.testing.assert_allclose(out[0, 2], v[1, 0, 0], atol=1e-12)
    assert np.isnan(out[:, 3]).all()                                     # no sequence's row
    out, lse, _, _ = so.attention(q, k, v, [0, 33], [0, 1, 2], table)    # nothing there; a position without a page
    assert (out[:, 0] == 0).all() and (lse[:, 0] == -np.inf).all() and np.isfinite(lse[:, 1]).all()


def test_window_and_sinks():
    ok = so.visible(10, 12, 4, 2)
    assert list(np.flatnonzero(ok)) == [0, 1, 7, 8, 9, 10]
    assert list(np.flatnonzero(so.visible(2, 12, 4, 2))) == [0, 1, 2]
    assert not so.visible(-1, 12, 4, 2).any()


def test_append_scale_grows_and_starts_anew():
    pages, scales = np.full((2, 1, 32, 64), 3.0), np.array([[0.5], [64.0]])
    x = np.full((1, 3, 64), 100.0)
    table = np.array([[0], [1]])
    out, s, new, moved = so.append_e4m3(pages, scales, x, [6, 2], [0, 1, 3], table)
    assert s[0, 0] == 0.5 and not moved[0].any() and out[0, 0, 5, 0] == 200.0            # large enough: kept
    assert s[1, 0] == 0.25 and new[1, 0, :2].all() and out[1, 0, 0, 0] == 400.0           # first token: anew
    out, s, new, moved = so.append_e4m3(pages, scales * 0.125, x, [6, 2], [0, 1, 3], table)
    assert s[0, 0] == 0.25 and moved[0, 0, :5].all() and out[0, 0, 0, 0] == 0.75 and out[0, 0, 6, 0] == 3.0
