"""Layouts of what the rollout's calls write: rows of two heads that share an element are refused (they would be written by two
workgroups), every other layout is taken as far as the next check, here a pointer that is refused.  No GPU, nothing is enqueued."""
import ctypes as C
import os
import random

import pytest

from paper_2602_04789_amd import lf

FAKE = 0x10000
SHAPE, ALIGN, WORKSPACE = -2, -5, -6


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(lf.library_path()):
        from paper_2602_04789_amd import build
        build.build()
    return lf.load()


def _overlap(heads, stride_head, tokens, stride_tok, d):
    """By laying the rows out."""
    seen = set()
    for h in range(heads):
        for t in range(tokens):
            for at in range(h * stride_head + t * stride_tok, h * stride_head + t * stride_tok + d, 8):
                if at in seen:
                    return True
                seen.add(at)
    return False


def _calls(lib, heads, stride_head, tokens, stride_tok, d):
    """The status of each call that writes such a tensor, and the one that it has where the layout is fine."""
    ap = lf.lf_axes_shape(heads, d, tokens, 0, 0, (d // 2, 0, 0), 1e-6, 0, heads * d, stride_tok, stride_head)
    yield lib.lf_qk_norm_rope_axes(FAKE, FAKE, FAKE, FAKE, C.byref(ap), FAKE + 2, None), ALIGN
    cs = lf.lf_kvq_shape(heads, d, 5000, 0)
    ok = (d, d * tokens)
    for k, v in (((stride_tok, stride_head), ok), (ok, (stride_tok, stride_head))):
        rows = lf.lf_kvq_rows(0, tokens, *k, *v)
        yield lib.lf_kvq_read(None, 0, C.byref(cs), C.byref(rows), FAKE, FAKE, None), WORKSPACE
    sh = lf.lf_shape(heads, d, tokens, 64, tokens, tokens, 0, 0, *ok, *ok, *ok, stride_tok, stride_head)
    yield lib.lf_sparse_attn_kvq(FAKE, None, 0, C.byref(cs), None, None, C.byref(sh), FAKE, 1, 0.0, FAKE, None, 0, None), WORKSPACE
    if tokens <= 64:
        ts = lf.lf_token_shape(heads, d, tokens, 5, 0, 0, *ok, *ok, *ok, stride_tok, stride_head)
        yield lib.lf_token_attn_kvq(FAKE, None, 0, C.byref(cs), None, None, C.byref(ts), 0.0, FAKE, None, 0, None), WORKSPACE


def test_rows_that_share_elements_are_refused(lib):
    rng = random.Random(0)
    both = [0, 0]
    for _ in range(3000):
        d, heads, tokens = rng.choice([64, 128]), rng.randint(1, 6), rng.randint(1, 6)
        stride_tok, stride_head = d + 8 * rng.randint(0, 5 * d // 8), 8 * rng.randint(0, 6 * d // 8)
        bad = _overlap(heads, stride_head, tokens, stride_tok, d)
        both[bad] += 1
        for status, fine in _calls(lib, heads, stride_head, tokens, stride_tok, d):
            assert status == (SHAPE if bad else fine), (heads, stride_head, tokens, stride_tok, d)
    assert min(both) > 500


@pytest.mark.parametrize("heads,stride_head,tokens,stride_tok,d,bad", [
    (2, 64, 2, 64, 64, True),                       # head 1's first token is head 0's second
    (12, 128 * 4679, 4680, 128, 128, True), (12, 128 * 4680, 4680, 128, 128, False),        # a head begins on the last token of the one before
    (12, 128, 4680, 1536, 128, False), (13, 128, 4680, 1536, 128, True),                    # token-major rows
    (2, 3 * 64, 100, 2 * 64, 64, False),            # heads between each other's tokens
    (256, 64, 1, 64, 64, False), (256, 56, 1, 64, 64, True),
    (3, (2 ** 63 - 1) // 8 * 8, 3, (2 ** 63 - 1) // 8 * 8, 64, True), (2, 2 ** 62, 4, 2 ** 60, 64, False), (2, 2 ** 62, 5, 2 ** 60, 64, True),
    (128, 2 ** 62, 4, 2 ** 60, 64, False)])
def test_named_layouts(lib, heads, stride_head, tokens, stride_tok, d, bad):
    for k, (status, fine) in enumerate(_calls(lib, heads, stride_head, tokens, stride_tok, d)):
        assert status == (SHAPE if bad else fine), k


def test_rows_behind_the_cache_are_not_looked_at_where_there_are_none(lib):
    """extra_len = 0: K and V may be anything, a slice without a row at an odd address among it; the next check is the workspace's."""
    cs = lf.lf_kvq_shape(12, 128, 32760, 0)
    nbytes = lf.lf_kvq_bytes(12, 128, 32760)
    for extra, ptr, status in ((0, FAKE + 2, WORKSPACE), (0, None, WORKSPACE), (1, FAKE + 2, ALIGN), (1, FAKE, WORKSPACE), (1, None, -1)):
        for K, V in ((ptr, FAKE), (FAKE, ptr), (ptr, ptr)):
            ts = lf.lf_token_shape(12, 128, 1, 32760, extra, 0, 128, 128, 128, 128, 128, 128, 128, 128)
            assert lib.lf_token_attn_kvq(FAKE, FAKE, nbytes, C.byref(cs), K, V, C.byref(ts), 0.0, FAKE, None, 0, None) == status, (extra, K, V)


def test_range_of_eps(lib):
    """What the producer and its gradients take for eps: from 0 on, nothing that is not finite."""
    for eps, taken in ((0.0, True), (-0.0, True), (1e-45, True), (1e-6, True), (1.0, True), (3.4e38, True), (-1e-45, False), (-1.0, False),
                       (float("inf"), False), (float("-inf"), False), (float("nan"), False)):
        p = lf.lf_axes_shape(12, 128, 4680, 0, 0, (22, 21, 21), eps, 0, 1536, 128, 128 * 4680)
        assert (lib.lf_qk_norm_rope_axes_bwd_workspace_bytes(C.byref(p)) > 0) == taken, eps
        want = ALIGN if taken else SHAPE
        assert lib.lf_qk_norm_rope_axes(FAKE, FAKE, FAKE, FAKE, C.byref(p), FAKE + 2, None) == want, eps
        assert lib.lf_qk_norm_rope_axes_bwd(FAKE, FAKE, FAKE, FAKE, C.byref(p), FAKE, FAKE + 2, FAKE, FAKE, 1 << 30, None) == want, eps
