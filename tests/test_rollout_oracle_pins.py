"""Pins for the oracle of the rollout's calls: library routines, other ways to write the same, differences.  CPU only."""
import numpy as np
import pytest
import torch

from oracle import qk_producer_oracle as P
from oracle import rollout_oracle as R

PAIRS = (4, 3, 1)


def _case(L=6, H=3, d=16, seed=0):
    rng = np.random.default_rng(seed)
    return (rng.standard_normal((L, H * d)), 1.0 + 0.1 * rng.standard_normal(H * d), rng.integers(-50, 50, (L, 3)),
            rng.uniform(0.01, 1.0, d // 2), rng.standard_normal((H, L, d)))


@pytest.mark.parametrize("across", [False, True])
@pytest.mark.parametrize("pairing", [0, 1])
def test_forward_is_the_producer_with_its_angle_tables(across, pairing):
    x, g, pos, freq, _ = _case()
    theta = R.angles(pos, freq, PAIRS)
    for l in range(6):       # pairs 0..3 by time, 4..6 by height, 7 by width
        assert theta[l, 3] == pos[l, 0] * freq[3] and theta[l, 4] == pos[l, 1] * freq[4] and theta[l, 7] == pos[l, 2] * freq[7]
    want = P.qk_norm_rope(x, g, np.cos(theta), np.sin(theta), 3, eps=1e-6, across_heads=across,
                          pairing="half" if pairing else "interleaved")
    assert np.allclose(R.rope_axes(x, g, theta, 3, 1e-6, across, pairing), want, atol=1e-13)


@pytest.mark.parametrize("across", [False, True])
@pytest.mark.parametrize("pairing", [0, 1])
def test_gradients_against_differences(across, pairing):
    x, g, pos, freq, dY = _case(L=3, H=2)
    theta = R.angles(pos, freq, PAIRS)
    f = lambda x, g: float((R.rope_axes(x, g, theta, 2, 1e-3, across, pairing) * dY).sum())
    dX, dg, *_ = R.rope_axes_backward(x, g, theta, 2, 1e-3, across, pairing, dY)
    h = 1e-6                  # central differences: off by h^2 times a third derivative, and by rounding / h
    for at in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[at] = h
        assert abs((f(x + e, g) - f(x - e, g)) / (2 * h) - dX[at]) < 1e-7
    for c in range(len(g)):
        e = np.zeros_like(g)
        e[c] = h
        assert abs((f(x, g + e) - f(x, g - e)) / (2 * h) - dg[c]) < 1e-7


def test_four_bit_values_are_the_nearest_on_the_grid():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 64)) * 10.0 ** rng.integers(-6, 6, (50, 1))
    code, scale = R.quantise(x)
    v = R.values(code, scale).reshape(50, 2, 32)
    s = 2.0 ** (scale.astype(float) - 127.0)
    top = np.abs(x).reshape(50, 2, 32).max(-1)
    assert np.all(top <= 7 * s) and np.all(top > 3.5 * s)
    z = np.abs(x.reshape(50, 2, 32)) / s[..., None]
    step = np.where(z < 2, 0.5, np.where(z < 4, 1.0, 2.0))
    assert np.all(np.abs(v - x.reshape(50, 2, 32)) <= 0.5 * step * s[..., None] * (1 + 1e-12))


def test_four_bit_ties_signs_and_special_groups():
    x = np.zeros((1, 32))
    x[0, :16] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -7.0]
    code, scale = R.quantise(x)
    assert scale[0, 0] == 127 and list(code[0, :16]) == [0, 2, 2, 4, 4, 6, 6, 7, 8, 10, 10, 12, 12, 14, 14, 15]
    assert list(code[0, 16:]) == [0] * 16
    code, scale = R.quantise(np.zeros((1, 64)))
    assert list(scale[0]) == [1, 1] and not code.any()
    x = np.ones((1, 64))
    x[0, 3] = np.inf
    x[0, 40] = np.nan
    code, scale = R.quantise(x)
    assert list(scale[0]) == [255, 255] and not code.any() and np.isnan(R.values(code, scale)).all()


def test_cache_bytes_go_where_they_belong():
    H, cap, d = 2, 5, 64
    parts, size = R.cache_parts(H, cap, d)
    assert parts == (0, 512, 1024, 1280) and size == 1536
    cache = np.full(size, 7, dtype=np.uint8)
    K = np.zeros((H, 1, d))
    K[1, 0, 33] = 6.0
    R.cache_write(cache, H, cap, d, 3, K, -K)
    k = 32 * (cap + 3) + 16                      # head 1, token 3, channels 32 and 33
    assert cache[k] == 7 * 16 and cache[512 + k] == 15 * 16 + 8 and cache[1024 + 2 * (cap + 3) + 1] == 127
    back = R.cache_read(cache, H, cap, d, 3, 4)
    assert np.array_equal(back[0], K) and np.array_equal(back[1], -K)
    assert (cache == 7).sum() == size - 2 * H * (32 + 2)


def test_attention_matches_library():
    rng = np.random.default_rng(2)
    Q, K, V = rng.standard_normal((5, 8)), rng.standard_normal((11, 8)), rng.standard_normal((11, 8))
    want = torch.nn.functional.scaled_dot_product_attention(*(torch.from_numpy(t)[None] for t in (Q, K, V)), scale=0.3)[0].numpy()
    assert np.allclose(R.attention(Q, K, V, 0.3)[0], want, atol=1e-13)
    assert np.array_equal(R.block_tokens([1, -1, 4, 0, 6], 70, 2, 6), np.r_[64:70, 140:204, 0:64])
