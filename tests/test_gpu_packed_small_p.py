"""dK of the packed attention where the probabilities are small: tokens beside one that takes nearly all of every row, and very many tokens.  P has to keep
its relative precision on the way into dS whatever it is, in every gradient kernel.

Bars.  Element by element as in test_gpu_packed_attn.py.  In the 2-norm, of a token or of all of them, with a rounding to bfloat16 off by at most 2^-8 of the
value, evenly, so 2^-8 / sqrt 3 = 2.26e-3 of it: dS once and the output once; P to no fewer than ten bits, 2^-10 / sqrt 3 = 0.56e-3; and beside
a dominating token s, O = v_s rounded, what that leaves in delta, 2.26e-3 |dO . v_s| against a dP - delta = dO . (v_y - v_s): 2.26e-3 / sqrt 2.
Independent, they are 3.3e-3 without the last one and 3.7e-3 with it; a median over tokens is below that by what a binade leaves."""
import numpy as np
import pytest

from oracle import blocks_oracle as R

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2602_04789_amd import lf
    lf.load()
    return torch, lf


def _np(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("above", [16, 40])
@pytest.mark.parametrize("H,Hk,d,rows,tokens,causal", [(2, 2, 64, 128, 4680, 0), (4, 2, 64, 200, 4680, 1), (2, 2, 128, 128, 4680, 0), (2, 1, 128, 200, 4680, 48),
                                                       (1, 1, 64, 64, 32760, 0), (12, 12, 64, 64, 4680, 0), (8, 8, 128, 64, 4680, 1)])
def test_tokens_beside_a_dominating_one(gpu, above, H, Hk, d, rows, tokens, causal):
    """Token 1 has logits that lie `above` the others' (of standard normal ones): P of the others is e^-above at the most."""
    torch, lf = gpu
    print(f"dominating H={H} Hk={Hk} d={d} rows={rows} tokens={tokens} causal={causal} above={above}", flush=True)
    g = torch.Generator().manual_seed(rows + d)
    r = lambda h, n: torch.randn((h, n, d), generator=g)
    Q, K, V, dO = r(H, rows), r(Hk, tokens), r(Hk, tokens), r(H, rows)
    Q[:, :, 0] = 8.0
    K[:, :, 0] = 0.0
    K[:, 1, 0] = above * d ** 0.5 / 8.0
    Q, K, V, dO = (t.to(torch.bfloat16).cuda() for t in (Q, K, V, dO))
    qs, ks = (torch.tensor([0, n], dtype=torch.int32, device="cuda") for n in (rows, tokens))
    O, lse2 = lf.lf_packed_attn_fwd(Q, K, V, qs, ks, causal=causal)
    dK = _np(lf.lf_packed_attn_bwd(Q, K, V, O, dO, lse2, qs, ks, causal=causal)[1])
    ref, size = (x[1] for x in R.packed_attention(_np(Q), _np(K), _np(V), [0, rows], [0, tokens], causal, d ** -0.5, _np(dO))[3:])
    err = np.abs(dK - ref)
    rel = np.median(np.linalg.norm(dK - ref, axis=-1) / np.linalg.norm(ref, axis=-1))
    bar = 1.1 * HALF * size + HALF * np.abs(ref) + 2.0 ** -110
    print("median of a token's error", rel, "largest of its bar", float((err / bar).max()))
    assert np.all(err <= bar)
    assert rel <= 3.7e-3


@pytest.mark.parametrize("tokens", [4681, 1 << 17, 1 << 20])
def test_many_tokens_share_a_row(gpu, tokens):
    """d = 64, no token above the others: P is some 1 / tokens."""
    torch, lf = gpu
    rows, d = 128, 64
    print(f"many tokens {tokens}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(tokens)
    r = lambda n: torch.randn((1, n, d), generator=g, device="cuda").to(torch.bfloat16)
    Q, K, V, dO = r(rows), r(tokens), r(tokens), r(rows)
    qs, ks = (torch.tensor([0, n], dtype=torch.int32, device="cuda") for n in (rows, tokens))
    O, lse2 = lf.lf_packed_attn_fwd(Q, K, V, qs, ks)
    _, dK, dV = lf.lf_packed_attn_bwd(Q, K, V, O, dO, lse2, qs, ks)
    q, k, v, do = (t[0].double() for t in (Q, K, V, dO))
    p = torch.softmax((q @ k.T.contiguous()) * d ** -0.5, -1)
    ds = do @ v.T.contiguous()
    ds -= (ds * p).sum(-1, keepdim=True)
    ds *= p
    for name, got, want in (("dK", dK, (ds.T.contiguous() @ q) * d ** -0.5), ("dV", dV, p.T.contiguous() @ do)):
        rel = float((got[0].double() - want).norm() / want.norm())
        print(name, rel)
        assert rel <= 3.3e-3, name
