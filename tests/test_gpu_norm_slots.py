"""Gradients of the norm between blocks where group_len or the number of groups goes beyond the tokens: the same shares of rows as without that, so the same bits."""
import ctypes as C

import pytest

from test_gpu_gate_norm import _inputs, _run, gpu  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("L,width", [(300, 320), (1999, 1536), (700, 2048), (300, 8200)])
def test_a_group_longer_than_the_tokens(gpu, L, width):  # noqa: F811
    """Against the oracle, and bit by bit against a group of all tokens."""
    want = _run(gpu, L, width, group_len=L, post=True, seed=1)
    for group_len in (L + 1, 5 * L, (1 << 31) - 1):
        got = _run(gpu, L, width, group_len=group_len, post=True, seed=1)
        assert all(gpu[0].equal(a, b) for a, b in zip(want[:2] + tuple(want[2]), got[:2] + tuple(got[2]))), group_len


@pytest.mark.parametrize("L,width,group_len", [(300, 320, 300), (300, 320, 1 << 20), (1000, 1536, 260), (90, 2056, 7)])
@pytest.mark.parametrize("more", [1, 77])
def test_more_groups_than_the_tokens_fill(gpu, L, width, group_len, more):  # noqa: F811
    """Through the C call, whose tables may have rows that no token belongs to: their gradients are zeros, and nothing else changes."""
    torch, lf = gpu
    live = -(-L // group_len)
    print(f"more groups L={L} width={width} group_len={group_len} groups={live + more}", flush=True)
    t = _inputs(torch, L, width, live + more, False, 2, 0)

    def call(groups):
        X1, _ = lf.lf_gate_norm(t["X"], B=t["B"], gate=t["gate"][:live], post_weight=t["post"], weight=t["weight"], scale=t["scale"][:live], group_len=group_len)
        p = lf.lf_norm_shape(L, width, groups, group_len, lf.LF_BF16, lf.LF_NORM_LAYER, 1e-6, 1.0, *[width] * 4, *[t["gate"].stride(0)] * 3)
        tables = [torch.full((live + more, width), 7.0, device="cuda") for _ in range(3)]
        weights = [torch.full((width,), 7.0, device="cuda") for _ in range(2)]
        dX, dB = torch.full_like(t["X"], 7.0), torch.full_like(t["B"], 7.0)
        n = lf.load().lf_gate_norm_bwd_workspace_bytes(C.byref(p))
        ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
        rc = lf.load().lf_gate_norm_bwd(X1.data_ptr(), t["B"].data_ptr(), t["gate"].data_ptr(), t["post"].data_ptr(), t["weight"].data_ptr(), t["scale"].data_ptr(), None, C.byref(p),
                                        t["dY"].data_ptr(), t["dXout"].data_ptr(), dX.data_ptr(), dB.data_ptr(), tables[0].data_ptr(), weights[0].data_ptr(), weights[1].data_ptr(),
                                        tables[1].data_ptr(), tables[2].data_ptr(), ws.data_ptr(), n, torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        torch.cuda.synchronize()
        return [dX, dB] + weights, tables
    (want, want_tables), (got, tables) = call(live), call(live + more)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    for a, b in zip(want_tables, tables):
        assert torch.equal(a[:live], b[:live]) and (a[live:] == 7.0).all() and (b[live:] == 0.0).all()
