"""The calls around the attention as they are used together: a finetuning step of one block over packed clips, and a row served over what it left."""
import numpy as np
import pytest

from oracle import blocks_oracle as B
from oracle import rollout_oracle as R

pytestmark = pytest.mark.gpu


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


def test_a_finetuning_step_over_packed_clips(gpu):
    """Norm and modulation, three-axis producer of Q and K, attention by chunks, gate onto the stream with the next norm, all gradients back, and their norm clipped.
    Every call's outputs are compared with the binary64 definitions on the inputs that it had, so a wrong hand-over (layout, strides, padding, groups) shows."""
    torch, lf = gpu
    H, d, starts, pad, chunk = 3, 64, [0, 70, 75, 210], 6, 30
    C, n, L, G = H * d, starts[-1], starts[-1] + 6, len(starts) - 1
    g = torch.Generator().manual_seed(0)
    r = lambda *s: torch.randn(s, generator=g).cuda()
    bf = torch.bfloat16
    s = torch.tensor(starts, dtype=torch.int32, device="cuda")
    X, tables = r(L, C), 0.3 * r(G, 5, C)               # float32 stream; shift, scale, gate, next shift, next scale
    Wq, Wk, Wv, Wo = (r(C, C) * C ** -0.5 for _ in range(4))
    gq, gk = 1.0 + 0.1 * r(C), 1.0 + 0.1 * r(C)
    pos = torch.randint(0, 40, (L, 3), generator=g, dtype=torch.int32).cuda()
    freq, pairs = (10000.0 ** -torch.linspace(0, 1, d // 2, dtype=torch.float64)).cuda(), (12, 10, 10)
    Y0 = torch.zeros((L, C), dtype=bf, device="cuda")
    lf.lf_gate_norm(X, scale=tables[:, 1], shift=tables[:, 0], starts=s, Y=Y0)
    x = [(Y0.float() @ W).to(bf) for W in (Wq, Wk, Wv)]
    Q, K = torch.empty((H, L, d), dtype=bf, device="cuda"), torch.empty((H, L, d), dtype=bf, device="cuda")
    lf.lf_qk_norm_rope_axes(x[0], gq, pos, freq, pairs, H, Q)
    lf.lf_qk_norm_rope_axes(x[1], gk, pos, freq, pairs, H, K)
    V = x[2].view(L, H, d).transpose(0, 1)               # token-major, as the projection leaves it
    O = torch.zeros((L, H, d), dtype=bf, device="cuda").transpose(0, 1)
    _, lse2 = lf.lf_packed_attn_fwd(Q, K, V, s, s, causal=chunk, O=O)
    block = (O.transpose(0, 1).reshape(L, C).float() @ Wo).to(bf)
    X1, Y1 = lf.lf_gate_norm(X, B=block, gate=tables[:, 2], scale=tables[:, 4], shift=tables[:, 3], starts=s, Xout=torch.zeros_like(X), Y=torch.zeros_like(Y0))
    # back
    dY1, dX1 = r(L, C).to(bf), r(L, C)
    how = dict(B=block, gate=tables[:, 2], scale=tables[:, 4], starts=s)
    dX, dB, dgate, _, _, dscale1, dshift1 = lf.lf_gate_norm_bwd(X1, dY1, dXout=dX1, dX=torch.zeros_like(X), dB=torch.zeros_like(block), **how)
    dO = (dB.float() @ Wo.T).to(bf).view(L, H, d).transpose(0, 1)
    grads = [torch.zeros((L, H, d), dtype=bf, device="cuda").transpose(0, 1) for _ in range(3)]
    dQ, dK, dV = lf.lf_packed_attn_bwd(Q.transpose(0, 1).contiguous().transpose(0, 1), K.transpose(0, 1).contiguous().transpose(0, 1), V, O, dO, lse2, s, s,
                                       causal=chunk, grads=grads)
    dxq, dgq = lf.lf_qk_norm_rope_axes_bwd(x[0], gq, pos, freq, pairs, H, dQ)
    dxk, dgk = lf.lf_qk_norm_rope_axes_bwd(x[1], gk, pos, freq, pairs, H, dK)
    dxv = dV.transpose(0, 1).reshape(L, C)
    dY0 = sum((t.float() @ W.T) for t, W in ((dxq, Wq), (dxk, Wk), (dxv, Wv))).to(bf)
    dX0, _, _, _, _, dscale0, dshift0 = lf.lf_gate_norm_bwd(X, dY0, dXout=dX, dX=torch.zeros_like(X), scale=tables[:, 1], starts=s)
    params = [(Y0.float().T @ t.float()) for t in (dxq, dxk, dxv)] + [O.transpose(0, 1).reshape(L, C).float().T @ dB.float(), dgq, dgk, dscale0, dshift0, dscale1, dshift1, dgate]
    kept = [p.clone() for p in params]
    norm = lf.lf_grad_clip(params, 1.0)
    torch.cuda.synchronize()
    # each against its definition
    gi, scale = B.groups_of(L, starts=starts), d ** -0.5
    near = lambda a, b, rel: np.linalg.norm(a - b) <= rel * np.linalg.norm(b)
    keep = gi >= 0
    T = _np(tables)
    assert near(_np(Y0)[keep], B.norm(_np(X)[keep], gi[keep], None, T[:, 1], T[:, 0], 1e-6, True), 2.0 ** -8) and (Y0[n:] == 0).all()
    theta = R.angles(pos.cpu().numpy(), freq.cpu().numpy(), pairs)
    assert near(_np(Q), R.rope_axes(_np(x[0]), _np(gq), theta, H, 1e-6, False, 0), 2.0 ** -8)
    ref = B.packed_attention(_np(Q), _np(K), _np(V), starts, starts, chunk, scale, _np(dO))
    assert near(_np(O)[:, :n], ref[0][:, :n], 5e-3) and (O[:, n:] == 0).all()
    for name, a, b in zip(("dQ", "dK", "dV"), (dQ, dK, dV), ref[3]):
        assert near(_np(a)[:, :n], b[:, :n], 6e-3) and (a[:, n:] == 0).all(), name
    assert near(_np(X1)[keep], B.gate(_np(X)[keep], _np(block)[keep], gi[keep], T[:, 2], None, 1e-6, 1.0), 2.0 ** -20) and (X1[n:] == 0).all()
    assert near(_np(Y1)[keep], B.norm(_np(X1)[keep], gi[keep], None, T[:, 4], T[:, 3], 1e-6, True), 2.0 ** -8)
    want, _ = B.gate_norm_backward(_np(X1)[keep], _np(block)[keep], gi[keep], G, T[:, 2], None, None, T[:, 4], 1e-6, 1.0, True, _np(dY1)[keep], _np(dX1)[keep])
    for name, a in (("dX", dX), ("dB", dB), ("dgate", dgate), ("dscale", dscale1), ("dshift", dshift1)):
        a = _np(a)[keep] if name in ("dX", "dB") else _np(kept[-1] if name == "dgate" else kept[-3] if name == "dscale" else kept[-2])
        assert near(a, want[name], 2.0 ** -8), name
    n0, f = B.clip([_np(p) for p in kept], 1.0, 1e-6)
    assert abs(float(norm) - n0) <= 2.0 ** -22 * n0 and f < 1.0
    assert all(near(_np(p), _np(k) * f, 2.0 ** -22) for p, k in zip(params, kept))
    # one more row of every clip, served over the keys and values that the step left: the same as that row inside a longer clip
    q1 = r(H, G, d).to(bf)
    sq = torch.arange(G + 1, dtype=torch.int32, device="cuda")
    got = _np(lf.lf_packed_attn(q1, K, V, sq, s, causal=1))
    want = B.packed_attention(_np(q1), _np(K), _np(V), list(range(G + 1)), starts, 1, scale)[0]
    assert near(got, want, 5e-3)


def test_a_block_gradient_through_autograd(gpu):
    """The calls inside a torch.autograd.Function, as a training program has them: gradients of a small block equal those of the plain formulas to what bfloat16 leaves
    (outputs of 2^-8, a few of them in a row: 2e-2 in the 2-norm)."""
    torch, lf = gpu
    s = torch.tensor([0, 40, 100], dtype=torch.int32, device="cuda")
    bf = torch.bfloat16

    class Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v):
            o, lse2 = lf.lf_packed_attn_fwd(q, k, v, s, s, causal=1)
            ctx.save_for_backward(q, k, v, o, lse2)
            return o

        @staticmethod
        def backward(ctx, do):
            q, k, v, o, lse2 = ctx.saved_tensors
            return lf.lf_packed_attn_bwd(q, k, v, o, do.contiguous(), lse2, s, s, causal=1)

    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w):
            _, y = lf.lf_gate_norm(x, weight=w, starts=s, kind=lf.LF_NORM_RMS)
            ctx.save_for_backward(x, w)
            return y

        @staticmethod
        def backward(ctx, dy):
            x, w = ctx.saved_tensors
            got = lf.lf_gate_norm_bwd(x, dy.contiguous(), weight=w, starts=s, kind=lf.LF_NORM_RMS)
            return got[0], got[4]

    g = torch.Generator().manual_seed(1)
    H, d, n = 2, 64, 100
    x, w = torch.randn((n, H * d), generator=g).cuda().requires_grad_(), (1.0 + 0.1 * torch.randn(H * d, generator=g)).cuda().requires_grad_()
    do = torch.randn((H, n, d), generator=g).to(bf).cuda()
    y = Norm.apply(x, w)
    heads = lambda t: t.view(n, H, d).transpose(0, 1).contiguous()
    o = Attention.apply(heads(y), heads(y), heads(y))
    got = torch.autograd.grad((o * do).sum(), (x, w))

    xd, wd = x.detach().double().requires_grad_(), w.detach().double().requires_grad_()
    yd = xd * torch.rsqrt(xd.square().mean(1, keepdim=True) + 1e-6) * wd
    t = yd.view(n, H, d).transpose(0, 1).contiguous()
    outs = []
    for a, b in ((0, 40), (40, 100)):
        q = t[:, a:b]
        z = (q @ q.transpose(1, 2).contiguous()) * d ** -0.5
        z = z.masked_fill(torch.triu(torch.ones(b - a, b - a, dtype=torch.bool, device="cuda"), 1), -1e300)
        outs.append(torch.softmax(z, -1) @ q)
    want = torch.autograd.grad((torch.cat(outs, 1) * do.double()).sum(), (xd, wd))
    for a, b in zip(got, want):
        assert float((a.double() - b).norm() / b.norm()) <= 2e-2
