"""Calls at the edges of what the rollout's entry points take, on the GPU."""
import pytest

from test_gpu_kvq import _cache, _check, _np, _rand, gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def test_places_that_do_not_fit_are_refused_and_nothing_is_written(gpu):  # noqa: F811
    torch, lf = gpu
    H, d, T = 2, 64, 70
    K = _rand(torch, 1, H, 4, d).cuda()
    cache = torch.randint(0, 256, (lf.lf_kvq_bytes(H, d, T),), generator=torch.Generator().manual_seed(2), dtype=torch.uint8).cuda()
    before, idx = cache.clone(), torch.zeros((H, 1, 1), dtype=torch.int32, device="cuda")
    for call in (lambda: lf.lf_kvq_append(K, K, cache, T, 2 ** 32), lambda: lf.lf_kvq_append(K, K, cache, T + 2 ** 32, 0),
                 lambda: lf.lf_kvq_read(cache, H, d, T, 2 ** 32, 4), lambda: lf.lf_token_attn_kvq(K, cache, T, 2 ** 32 + 4),
                 lambda: lf.lf_sparse_attn_kvq(K, cache, T, 2 ** 32 + 4, idx, 4, 64)):
        with pytest.raises(ValueError, match="32 bits"):
            call()
    torch.cuda.synchronize()
    assert torch.equal(cache, before)


def test_rows_behind_the_cache_at_an_odd_address_without_a_row(gpu):  # noqa: F811
    torch, lf = gpu
    H, d, T = 2, 64, 70
    dev, host = _cache(gpu, H, T, d, _rand(torch, 1, H, T, d), _rand(torch, 2, H, T, d))
    Q, none = _rand(torch, 3, H, 2, d).cuda(), torch.zeros(9 * d, dtype=torch.bfloat16, device="cuda")[3:].as_strided((H, 0, d), (d, d, 1))
    want = lf.lf_token_attn_kvq(Q, dev, T, T)
    assert torch.equal(lf.lf_token_attn_kvq(Q, dev, T, T, K=none, V=none), want)
