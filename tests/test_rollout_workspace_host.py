"""The list attention's scratch over a growing cache, as lf.h states it: a call's size can be less than a shorter one's, a buffer with the
largest of the sizes serves all, and no size is beyond the bounds given there.  No GPU: calls are stopped by the pointer check behind the scratch's."""
import ctypes as C
import os
import random

import pytest

from paper_2602_04789_amd import lf

FAKE = 0x10000


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(lf.library_path()):
        from paper_2602_04789_amd import build
        build.build()
    return lf.load()


def _status(lib, H, d, n, q, kv, length, size):
    """Of a call with that much scratch, at an address that is refused (-5) if the size is not (-6)."""
    cs = lf.lf_kvq_shape(H, d, kv, 0)
    sh = lf.lf_shape(H, d, n, 64, q, kv, 0, 0, *((d, d * q) * 4))
    return lib.lf_sparse_attn_kvq(FAKE, FAKE, lf.lf_kvq_bytes(H, d, kv), C.byref(cs), FAKE, FAKE, C.byref(sh), FAKE, length, 0.0, FAKE,
                                  FAKE + 16, size, None)


def test_one_buffer_for_a_rollout_with_lists_of_one_length(lib):
    H, d, n, q, length = 12, 128, 1560, 3 * 1560, 20
    need = {kv: lf.lf_sparse_attn_kvq_workspace_bytes(H, d, n, 64, q, kv, length) for kv in range(2 * q, 8 * q, q)}
    assert need[2 * q] == 2 * H * 2 * q * d * 2 and need[7 * q] == 0          # written in bfloat16 first; converted as it is read
    most = max(need.values())
    for kv in need:
        if need[kv]:
            assert _status(lib, H, d, n, q, kv, length, most) == -5 and _status(lib, H, d, n, q, kv, length, need[kv] - 1) == -6


def test_sizes_are_within_their_bounds(lib):
    rng = random.Random(1)
    kinds = set()
    for _ in range(20000):
        H, d, n, f = rng.randint(1, 40), rng.choice([64, 128]), round(8 * 200 ** rng.random()), rng.randint(1, 3)
        F, length = f + rng.randint(0, 40), round(3000 ** rng.random())
        need = lf.lf_sparse_attn_kvq_workspace_bytes(H, d, n, 64, f * n, F * n, length)
        rows = 2 * ((H * F * n * d * 2 + 255) // 256 * 256)
        assert need == rows or need <= 512 * 64 * (d + 2) * 4, (H, d, n, f, F, length)
        kinds.add(2 if need == rows else need > 0)
    assert kinds == {0, 1, 2}
