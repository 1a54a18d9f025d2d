"""eps = 0, the lower end of what the three-axis producer accepts: numbers of tokens that leave threads of the last workgroup without one (such a
thread's sum of squares is 0, its 1 / sqrt(0 + 0) not finite), against the binary64 oracle.  Bars as in test_gpu_rope_axes."""
import pytest

from test_gpu_rope_axes import _run, gpu  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,d", [(1, 64), (2, 64), (5, 64), (12, 128), (40, 128)])
@pytest.mark.parametrize("across", [False, True])
def test_eps_of_zero(gpu, H, d, across):  # noqa: F811
    for L, pairing in ((1, 0), (11, 1), (37, 0)):
        _run(gpu, L, H, d, across, pairing, seed=L + H, eps=0.0)


@pytest.mark.parametrize("across", [False, True])
def test_eps_of_zero_and_many_tokens(gpu, across):  # noqa: F811
    _run(gpu, 1333, 5, 64, across, 1, seed=3, eps=0.0)
    _run(gpu, 4681, 12, 128, across, 0, seed=4, eps=0.0)
