"""The 4-bit format and the log probabilities of the oracle: properties of their definitions (no GPU)."""
import numpy as np
import pytest

from oracle import cache_q4


def test_scales_are_the_least_that_reach_the_largest_value():
    rng = np.random.RandomState(0)
    x = rng.randn(200, 32) * 10.0 ** rng.uniform(-40, 37, (200, 1))
    x[0] = 0
    x = np.float32(x).astype(np.float64)
    s = cache_q4.scales(x)
    a = np.abs(x).max(-1)
    assert s[0] == 0 and (7 * s >= a).all()
    m, e = np.frexp(s[1:])
    step = np.maximum(np.ldexp(1.0, e - 5), 2.0 ** -130)
    assert np.array_equal(np.rint(s[1:] / step) * step, s[1:])   # five bits
    below = s[1:] - np.where(m == 0.5, np.maximum(step / 2, 2.0 ** -130), step)
    assert (7 * below < a[1:]).all()


def test_values_are_bfloat16_and_within_half_a_step():
    import torch
    rng = np.random.RandomState(1)
    x = np.float32(rng.randn(64, 128) * np.exp(rng.randn(64, 1)))
    y = cache_q4.values(x)
    assert np.array_equal(torch.from_numpy(y).to(torch.bfloat16).double().numpy(), y)
    step = np.repeat(cache_q4.scales(x.reshape(64, 4, 32).astype(np.float64)), 32, -1)
    assert (np.abs(y - x) <= step / 2).all()
    assert np.array_equal(cache_q4.values(y), y)     # what is read back is held as it is


def test_ties_go_to_the_even_code():
    x = np.zeros((1, 32))
    x[0, :8] = [7, 0.5, 1.5, 2.5, -0.5, -1.5, -6.5, 6.5]         # scale 1
    c, s = cache_q4.quantise(x)
    assert s[0, 0] == 1 and c[0, 0, :8].tolist() == [7, 0, 2, 2, 0, -2, -6, 6]


@pytest.mark.parametrize("page,d", [(16, 64), (32, 128)])
def test_bytes_and_back(page, d):
    x = np.random.RandomState(2).randn(2, 3, page, d)
    b = cache_q4.pack(x)
    assert b.shape == (2, 3, page * d * 9 // 16)
    np.testing.assert_array_equal(cache_q4.unpack(b, page, d), cache_q4.values(x))
    # element 8 w + 2 k + h of a slot's first group at bits 16 h + 4 k of word w
    c, _ = cache_q4.quantise(x)
    w = b[1, 2, :d // 2].view("<u4")
    assert [(int(w[1]) >> (16 * h + 4 * k)) & 15 for k in range(4) for h in range(2)] == (c[1, 2, 0, 0, 8:16] + 8).tolist()


def test_logprobs_of_a_known_row():
    z = np.log(np.array([[0.5, 0.25, 0.125, 0.125], [0.0, 1, 1, 1]]).clip(1e-300))
    z[1, 0] = -np.inf
    lp, h, top, tl = cache_q4.logprobs(z, [1, -1], 1.0, 3)
    np.testing.assert_allclose(lp[0], np.log(0.25))
    np.testing.assert_allclose(h[0], 1.75 * np.log(2))
    assert top[0].tolist() == [0, 1, 2] and top[1].tolist() == [-1] * 3 and h[1] == 0 and np.isneginf(lp[1])
    np.testing.assert_allclose(tl[0], np.log([0.5, 0.25, 0.125]))
