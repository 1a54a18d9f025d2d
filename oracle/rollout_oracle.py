"""CPU oracle for the calls of a long rollout: rotary positions over three axes with RMSNorm and their gradients, the 4-bit
cache, and attention over it.  TEST INFRASTRUCTURE ONLY; it shares no code with the GPU library.

* RMSNorm and rotation as in ``qk_producer_oracle``, the angle of pair i being pos[token, axis(i)] * freq[i]; the gradients
  are written from z = R(-theta) dY, n = x / r, u = z g: dg = sum z n, dx = (u - n mean(u n)) / r.
* The cache holds 32 channels of a token as a scale 2^e and signed values of 0, 0.5, 1, 1.5, 2, 3, 4, 6: e is the smallest integer, at
  least -126, with max|x| <= 7 * 2^e; a value goes to the nearest, a tie to the one with an even place in that row.
* Attention is softmax(q . k * scale) v over the tokens given, in binary64.
"""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def angles(pos: np.ndarray, freq: np.ndarray, pairs) -> np.ndarray:
    """[L, d/2] in binary64."""
    axis = np.repeat(np.arange(3), pairs)
    return np.asarray(pos, dtype=np.float64)[:, axis] * np.asarray(freq, dtype=np.float64)


def _split(y, pairing):
    half = y.shape[-1] // 2
    return (y[..., 0::2], y[..., 1::2]) if pairing == 0 else (y[..., :half], y[..., half:])


def _join(a, b, pairing):
    if pairing:
        return np.concatenate((a, b), -1)
    out = np.empty(a.shape[:-1] + (2 * a.shape[-1],))
    out[..., 0::2], out[..., 1::2] = a, b
    return out


def rotate(y, theta, pairing):
    """Channel pairs of y [L, H, d] turned by theta [L, d/2]."""
    c, s = np.cos(theta)[:, None], np.sin(theta)[:, None]
    a, b = _split(np.asarray(y, dtype=np.float64), pairing)
    return _join(a * c - b * s, a * s + b * c, pairing)


def _norm(x, heads, eps, across):
    """x [L, H*d] -> (n [L, H, d], 1/r [L, H or 1, 1])."""
    x = np.asarray(x, dtype=np.float64).reshape(len(x), heads, -1)
    over = (1, 2) if across else (2,)
    inv = 1.0 / np.sqrt((x * x).mean(over, keepdims=True) + eps)
    return x * inv, inv


def rope_axes(x, g, theta, heads, eps, across, pairing):
    """[H, L, d]."""
    n, _ = _norm(x, heads, eps, across)
    return rotate(n * np.asarray(g, dtype=np.float64).reshape(heads, -1), theta, pairing).transpose(1, 0, 2)


def rope_axes_backward(x, g, theta, heads, eps, across, pairing, dY):
    """(dX [L, H*d], dg [H*d]) and how large the terms are that each was added up from (for error bounds)."""
    n, inv = _norm(x, heads, eps, across)
    w = np.asarray(g, dtype=np.float64).reshape(heads, -1)
    dY = np.asarray(dY, dtype=np.float64).transpose(1, 0, 2)
    z = rotate(dY, -theta, pairing)
    a, b = _split(np.abs(dY), pairing)
    size = _join(a + b, a + b, pairing)
    over = (1, 2) if across else (2,)
    u = z * w
    dX = inv * (u - n * (u * n).mean(over, keepdims=True))
    big = inv * (size * abs(w) + abs(n) * (size * abs(w) * abs(n)).mean(over, keepdims=True))
    return dX.reshape(len(x), -1), (z * n).sum(0).ravel(), big.reshape(len(x), -1), (size * abs(n)).sum(0).ravel()


def quantise(x):
    """x [..., d] -> (codes uint8 [..., d] of 0 .. 15, scale bytes uint8 [..., d/32])."""
    x = np.asarray(x, dtype=np.float64)
    v = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    top = np.abs(v).max(-1)
    fine = np.isfinite(v).all(-1)
    e = np.full(top.shape, -126)
    for k in range(-126, 128):            # the smallest that fits
        e = np.where(np.where(fine, top, 0.0) > 7.0 * 2.0 ** k, k + 1, e)
    with np.errstate(invalid="ignore"):
        z = np.where(fine[..., None], v * 2.0 ** -e[..., None].astype(np.float64), 0.0)
    dist = np.abs(np.abs(z)[..., None] - GRID)
    least = dist.min(-1, keepdims=True)
    near = dist == least
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
    code = code + 8 * (np.signbit(z) & fine[..., None])
    return code.reshape(x.shape).astype(np.uint8), np.where(fine, e + 127, 255).astype(np.uint8)


def values(codes, scales):
    """What codes and scale bytes stand for, binary64."""
    v = np.where(codes & 8, -1.0, 1.0) * GRID[codes & 7]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127.0))
    return (v.reshape(v.shape[:-1] + (v.shape[-1] // 32, 32)) * s[..., None]).reshape(v.shape)


def cache_parts(heads, capacity, d):
    """Byte offsets of the codes of K and V and of their scales, and the size of a cache."""
    up = lambda n: -(-n // 256) * 256
    codes, scales = up(heads * capacity * d // 2), up(heads * capacity * d // 32)
    return (0, codes, 2 * codes, 2 * codes + scales), 2 * (codes + scales)


def cache_write(cache, heads, capacity, d, first, K, V):
    """Lay K and V [H, L, d] into the bytes of a cache (uint8 [size])."""
    at, _ = cache_parts(heads, capacity, d)
    last = first + K.shape[1]
    for i, x in enumerate((K, V)):
        code, scale = quantise(x)
        cache[at[i]:at[i] + heads * capacity * d // 2].reshape(heads, capacity, d // 2)[:, first:last] = \
            code[..., 0::2] + 16 * code[..., 1::2]
        cache[at[2 + i]:at[2 + i] + heads * capacity * d // 32].reshape(heads, capacity, d // 32)[:, first:last] = scale


def cache_read(cache, heads, capacity, d, first, last):
    """(K, V) [H, last - first, d], binary64."""
    at, _ = cache_parts(heads, capacity, d)
    out = []
    for i in range(2):
        b = cache[at[i]:at[i] + heads * capacity * d // 2].reshape(heads, capacity, d // 2)[:, first:last]
        code = np.stack((b & 15, b >> 4), -1).reshape(heads, last - first, d)
        scale = cache[at[2 + i]:at[2 + i] + heads * capacity * d // 32].reshape(heads, capacity, d // 32)[:, first:last]
        out.append(values(code, scale))
    return out


def attention(Q, K, V, scale):
    """Rows of softmax(Q K^T scale) V [q, d], the mean of |v| under the same weights, and the largest sum of |q k| scale."""
    if len(K) == 0:
        return np.zeros(Q.shape), np.zeros(Q.shape), 0.0
    s = Q @ K.T * scale
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    return p @ V, p @ np.abs(V), float((np.abs(Q) @ np.abs(K).T).max() * scale)


def block_tokens(ids, n, nb, n_k):
    """Tokens of the KV blocks listed, invalid ids left out."""
    got = [np.arange(c // nb * n + c % nb * 64, c // nb * n + min(n, (c % nb + 1) * 64)) for c in ids if 0 <= c < n_k]
    return np.concatenate(got) if got else np.zeros(0, dtype=int)
