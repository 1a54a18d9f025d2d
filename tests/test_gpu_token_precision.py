"""Up to 16 query rows over the 4-bit cache: the probabilities go into their product in two bfloat16 parts, so that the output's own rounding is
what is left.

Bar.  A probability p is hi + lo, hi = p rounded to bfloat16 (off by at most 2^-8 p), lo = p - hi (exact in float32, for both are multiples of p's last
place) rounded to bfloat16: off by 2^-8 of 2^-8 p, 2^-16 p.  Numerator and sum take the same parts, so O is off by 2^-16 (A + |O|), A the mean of |v|, and
by the output's half step 2^-8 |O|; the float32 terms are those of test_gpu_kvq."""
import numpy as np
import pytest

from oracle import rollout_oracle as R
from test_gpu_kvq import _cache, _np, _rand, gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def _close(got, Q, K, V, scale):
    ref, size, terms = R.attention(Q, K, V, scale)
    T, d = len(K), Q.shape[1]
    bar = (2.0 ** -8 + 2.0 ** -16) * np.abs(ref) + (2.0 ** -16 + 2 * (d + 8) * 2.0 ** -24 * terms + (T + 300) * 2.0 ** -24) * size + 1e-37
    assert np.all(np.abs(got - ref) <= bar), (float((np.abs(got - ref) / bar).max()), T)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,rows,cached,extra,qscale", [(2, 1, 77, 1, 1.0), (12, 1, 2500, 0, 1.0), (3, 16, 1301, 70, 1.0), (2, 9, 4111, 3, 8.0), (40, 3, 700, 5, 0.1)])
def test_few_rows_lose_nothing_but_the_outputs_rounding(gpu, d, H, rows, cached, extra, qscale):  # noqa: F811
    torch, lf = gpu
    print(f"token H={H} d={d} rows={rows} cached={cached} extra={extra} qscale={qscale}", flush=True)
    Q = _rand(torch, 1, H, rows, d, scale=qscale)
    K, V = _rand(torch, 2, H, cached, d), _rand(torch, 3, H, cached, d)
    Kx, Vx = _rand(torch, 4, H, extra, d), _rand(torch, 5, H, extra, d)
    dev, host = _cache(gpu, H, cached, d, K, V)
    O = lf.lf_token_attn_kvq(Q.cuda(), dev, cached, cached, K=Kx.cuda(), V=Vx.cuda())
    rk, rv = R.cache_read(host, H, cached, d, 0, cached)
    for h in range(H):
        _close(_np(O[h]), _np(Q[h]), np.concatenate((rk[h], _np(Kx[h]))), np.concatenate((rv[h], _np(Vx[h]))), d ** -0.5)


def test_a_score_far_above_the_reference(gpu):  # noqa: F811
    """A later tile whose probabilities overflow against the first tile's maximum: they are made again before their parts are taken."""
    torch, lf = gpu
    H, d, T = 2, 128, 900
    K, V, Q = _rand(torch, 1, H, T, d), _rand(torch, 2, H, T, d), _rand(torch, 3, H, 5, d, scale=30.0)
    K[:, :700] *= 0.001
    dev, host = _cache(gpu, H, T, d, K, V)
    O = lf.lf_token_attn_kvq(Q.cuda(), dev, T, T)
    rk, rv = R.cache_read(host, H, T, d, 0, T)
    for h in range(H):
        _close(_np(O[h]), _np(Q[h]), rk[h], rv[h], d ** -0.5)
