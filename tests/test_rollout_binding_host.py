"""Sizes and places that do not fit the int32 fields of the C structures: refused by the binding of the rollout's calls (ctypes
would drop their upper bits, and the call would run on other tokens).  No GPU: the refusal comes before anything else is looked at."""
import pytest
import torch

from paper_2602_04789_amd import lf

BIG = (2 ** 31, 2 ** 32, 2 ** 32 + 4, -2 ** 31 - 1, -2 ** 32 + 4)


@pytest.mark.parametrize("big", BIG)
def test_calls_refuse_what_does_not_fit(big):
    X, Y = torch.zeros(4, 128, dtype=torch.bfloat16), torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    g, pos, freq = torch.ones(128), torch.zeros(4, 3, dtype=torch.int32), torch.ones(32, dtype=torch.float64)
    cache, idx = torch.zeros(4096, dtype=torch.uint8), torch.zeros((2, 1, 1), dtype=torch.int32)
    calls = [lambda: lf.lf_kvq_append(Y, Y, cache, 8, big), lambda: lf.lf_kvq_append(Y, Y, cache, big, 0)]
    for at in range(1, 6):          # heads, head_dim, capacity, first, tokens
        args = [cache, 2, 64, 8, 0, 4]
        args[at] = big
        calls.append(lambda args=args: lf.lf_kvq_read(*args, K=Y, V=Y))
    for at in (2, 3, 5, 6):         # capacity, kv_len, frame_len, block
        args = [Y, cache, 8, 8, idx, 4, 64]
        args[at] = big
        calls.append(lambda args=args: lf.lf_sparse_attn_kvq(*args))
    calls += [lambda: lf.lf_token_attn_kvq(Y, cache, big, 4), lambda: lf.lf_token_attn_kvq(Y, cache, 8, big)]
    for call in (lf.lf_qk_norm_rope_axes, lf.lf_qk_norm_rope_axes_bwd):
        for pairs in ((big, 10, 10), (12, big, 10), (12, 10, big)):
            calls.append(lambda call=call, pairs=pairs: call(X, g, pos, freq, pairs, 2, Y))
        calls += [lambda call=call: call(X, g, pos, freq, (12, 10, 10), 2, Y, pairing=big),
                  lambda call=call: call(X, g, pos, freq, (12, 10, 10), big, Y)]
    for k, call in enumerate(calls):
        with pytest.raises(ValueError, match="32 bits"):
            call()
            print("taken:", k)


@pytest.mark.parametrize("big", BIG)
def test_sizes_of_what_does_not_fit_are_zero(big):
    for f, args in ((lf.lf_kvq_bytes, (2, 64, 100)), (lf.lf_qk_norm_rope_axes_bwd_workspace_bytes, (2, 64, 100)),
                    (lf.lf_sparse_attn_kvq_workspace_bytes, (2, 64, 64, 64, 64, 64 * 100, 90)),
                    (lf.lf_token_attn_kvq_workspace_bytes, (2, 64, 5, 5000, 5))):
        assert f(*args) > 0
        for at in range(len(args)):
            assert f(*args[:at], big, *args[at + 1:]) == 0, (f.__name__, at)
