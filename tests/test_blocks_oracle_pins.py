"""Pins for the oracle of the calls around the attention: library routines, other ways to write the same, differentiation.  CPU only."""
import numpy as np
import pytest
import torch

from oracle import blocks_oracle as R


@pytest.mark.parametrize("layer", [True, False])
@pytest.mark.parametrize("post", [True, False])
def test_norm_and_gradients_against_differentiation(layer, post):
    rng = np.random.default_rng(1)
    L, C, starts, rs, eps = 9, 24, [1, 4, 4, 8], 0.7, 1e-3
    g = R.groups_of(L, starts=starts)
    assert list(g) == [-1, 0, 0, 0, 2, 2, 2, 2, -1]
    keep = g >= 0
    t = {k: torch.from_numpy(rng.standard_normal(s)).requires_grad_() for k, s in
         dict(X=(L, C), B=(L, C), gate=(3, C), scale=(3, C), shift=(3, C), weight=(C,), post=(C,)).items()}
    gi = torch.from_numpy(g[keep])
    b = t["B"][keep]
    if post:
        b = torch.nn.functional.rms_norm(b, (C,), t["post"], eps)
    xo = t["X"][keep] + rs * t["gate"][gi] * b
    n = torch.nn.functional.layer_norm(xo, (C,), eps=eps) if layer else torch.nn.functional.rms_norm(xo, (C,), eps=eps)
    y = n * t["weight"] * (1 + t["scale"][gi]) + t["shift"][gi]
    a = {k: v.detach().numpy() for k, v in t.items()}
    Xo = R.gate(a["X"][keep], a["B"][keep], g[keep], a["gate"], a["post"] if post else None, eps, rs)
    assert np.allclose(Xo, xo.detach().numpy(), atol=1e-13)
    assert np.allclose(R.norm(Xo, g[keep], a["weight"], a["scale"], a["shift"], eps, layer), y.detach().numpy(), atol=1e-12)
    dY, dXo = rng.standard_normal(Xo.shape), rng.standard_normal(Xo.shape)
    names = ["X", "B", "gate", "scale", "shift", "weight"] + (["post"] if post else [])
    want = dict(zip(names, torch.autograd.grad((y, xo), [t[k] for k in names], (torch.from_numpy(dY), torch.from_numpy(dXo)))))
    got, size = R.gate_norm_backward(Xo, a["B"][keep], g[keep], 3, a["gate"], a["post"] if post else None, a["weight"], a["scale"], eps, rs, layer, dY, dXo)
    for k, name in (("X", "dX"), ("B", "dB"), ("gate", "dgate"), ("scale", "dscale"), ("shift", "dshift"), ("weight", "dweight"), ("post", "dpost_weight")):
        if k in want:
            w = want[k].numpy()
            w = w[keep] if k in "XB" else w
            assert np.allclose(got[name], w, atol=1e-11), name
            assert np.all(size[name] >= np.abs(got[name]) - 1e-12)
    assert np.all(got["dshift"][1] == 0)


def test_group_of_a_token():
    assert list(R.groups_of(5, group_len=2)) == [0, 0, 1, 1, 2]


@pytest.mark.parametrize("causal,nq,nk,want", [(0, 2, 5, [5, 5]), (1, 3, 3, [1, 2, 3]), (1, 2, 5, [4, 5]), (1, 4, 2, [0, 0, 1, 2]), (3, 6, 6, [3, 3, 3, 6, 6, 6]),
                                               (3, 2, 5, [5, 5]), (4, 7, 7, [4, 4, 4, 4, 7, 7, 7]), (2, 5, 3, [0, 0, 2, 2, 3]), (1, 1, 0, [0])])
def test_what_rows_see(causal, nq, nk, want):
    assert [R.seen(nq, nk, causal, i) for i in range(nq)] == want
    if causal:      # the same as tokens in the chunks up to the one that holds the row's own place
        for i in range(nq):
            p = nk - nq + i
            assert want[i] == sum(1 for j in range(nk) if p >= 0 and j // causal <= p // causal)


@pytest.mark.parametrize("causal", [0, 1, 3])
def test_attention_and_gradients_against_differentiation(causal):
    rng = np.random.default_rng(2)
    H, Hk, d, q_start, kv_start = 4, 2, 8, [1, 4, 4, 9, 10], [0, 5, 7, 10, 10]
    Q, dO = rng.standard_normal((2, H, 12, d))
    K, V = rng.standard_normal((2, Hk, 11, d))
    scale = 0.3
    O, lse2, _, grads, sizes = R.packed_attention(Q, K, V, q_start, kv_start, causal, scale, dO)
    t = [torch.from_numpy(x).requires_grad_() for x in (Q, K, V)]
    total = 0.0
    for b in range(4):
        nq, nk = q_start[b + 1] - q_start[b], kv_start[b + 1] - kv_start[b]
        for i in range(nq):
            n = R.seen(nq, nk, causal, i)
            for h in range(H):
                x = q_start[b] + i
                if n == 0:
                    assert np.all(O[h, x] == 0) and np.isposinf(lse2[h, x])
                    continue
                k = slice(kv_start[b], kv_start[b] + n)
                z = t[1][h // 2, k] @ t[0][h, x] * scale
                o = torch.softmax(z, 0) @ t[2][h // 2, k]
                assert np.allclose(O[h, x], o.detach().numpy(), atol=1e-13)
                assert np.isclose(lse2[h, x], float(torch.logsumexp(z, 0)) / np.log(2.0), atol=1e-12)
                total = total + (o * torch.from_numpy(dO[h, x])).sum()
    for name, got, size, want in zip("QKV", grads, sizes, torch.autograd.grad(total, t)):
        inside = ~np.isnan(got)
        assert np.allclose(got[inside], want.numpy()[inside], atol=1e-12), name
        assert np.all(want.numpy()[~inside] == 0)
        assert np.all(size[inside] >= np.abs(got[inside]) * 0.99 - 1e-12)
    assert np.isnan(O[:, 0]).all() and np.isnan(O[:, 10:]).all() and np.isnan(grads[1][:, 10:]).all()


def test_clip():
    n, f = R.clip([np.array([3.0, 0.0]), np.array([[4.0]])], 2.0, 0.0)
    assert n == 5.0 and f == 0.4 and R.clip([np.array([3.0])], 4.0, 0.0)[1] == 1.0
    assert R.clip([np.array([np.inf])], 4.0, 0.0) == (np.inf, 1.0) and R.clip([], 1.0, 1e-6)[0] == 0.0
