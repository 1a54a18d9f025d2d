"""The rollout's calls as a program makes them, one after the other: chunks that are produced, attended over the 4-bit cache and then stored in
it, single query rows over what is held, and a finetuning step through the producer.  Every stage against the binary64 oracle on
what the stage before it left; bars as in the stages' own tests."""
import numpy as np
import pytest

from oracle import rollout_oracle as R
from paper_2602_04789_amd import synth
from test_gpu_kvq import _check
from test_gpu_rope_axes import _rel_ok

pytestmark = pytest.mark.gpu

PAIRS = (12, 10, 10)


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


def _positions(torch, first_frame, frames, n, width):
    l = torch.arange(frames * n)
    return torch.stack((first_frame + l // n, l % n // width, l % n % width), 1).to(torch.int32)


def _produced(torch, lf, X, w, pos, freq, H, Y):
    """RMSNorm and positions into Y, checked."""
    lf.lf_qk_norm_rope_axes(X, w, pos.cuda(), freq.cuda(), PAIRS, H, Y)
    theta = R.angles(pos.numpy(), freq.numpy(), PAIRS)
    ref = R.rope_axes(_np(X), _np(w), theta, H, 1e-6, False, 0)
    n, _ = R._norm(_np(X), H, 1e-6, False)
    a, b = R._split(np.abs(n * _np(w).reshape(H, -1)), 0)
    _rel_ok(_np(Y), ref, R._join(a + b, a + b, 0).transpose(1, 0, 2), 2.0 ** -18)


def test_rollout_over_the_four_bit_cache(gpu):
    torch, lf = gpu
    H, d, n, f, chunks = 3, 64, 100, 2, 4
    nb, q, frames = 2, f * n, f * chunks
    g = torch.Generator().manual_seed(0)
    rand = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).cuda()
    w = (1.0 + 0.1 * torch.randn(H * d, generator=g)).cuda()
    freq = torch.cat([10000.0 ** (-torch.arange(k, dtype=torch.float64) / k) for k in PAIRS])
    sched = synth.Schedule(mode=synth.SCHED_FIXED, n_chunks=chunks, frames_per_chunk=f, frame_len=n, n_sink=1, n_win=1, k_frames=2,
                           ratio_of=synth.OF_HISTORY, current_mandatory=1, first_chunk_dense=0, keep_fixed=0.6)
    cap = frames * n
    held = torch.randint(0, 256, (lf.lf_kvq_bytes(H, d, cap),), generator=g, dtype=torch.uint8).cuda()
    Kc = torch.zeros((H, cap, d), dtype=torch.bfloat16, device="cuda")      # the current chunk's rows at their place, for the pooled keys
    shape = lf.make_shape(Kc[:, :q], Kc, frame_len=n)
    pooled = torch.zeros(lf.lf_kcache_bytes(shape, frames), dtype=torch.uint8, device="cuda")
    for i in range(1, chunks + 1):
        print("chunk", i, flush=True)
        at, kv = (i - 1) * q, i * q
        pos = _positions(torch, (i - 1) * f, f, n, 10)
        Q, V = torch.empty((H, q, d), dtype=torch.bfloat16, device="cuda"), rand(H, q, d)
        K = Kc[:, at:kv]
        _produced(torch, lf, rand(q, H * d), w, pos, freq, H, Q)
        _produced(torch, lf, rand(q, H * d), w, pos, freq, H, K)
        b = lf.lf_chunk_budget(i, sched)
        lists = lf.lf_select_mask_cached(Q, pooled, frames, kv, n, 64, b, Kcache=Kc[:, :kv])
        O = lf.lf_sparse_attn_kvq(Q, held, cap, kv, lists, n, 64, K=K, V=V)
        rk, rv = R.cache_read(held.cpu().numpy(), H, cap, d, 0, at)
        rk, rv = np.concatenate((rk, _np(K)), 1), np.concatenate((rv, _np(V)), 1)
        for h in range(H):
            for r in range(f * nb):
                rows, t = R.block_tokens([r], n, nb, f * nb), R.block_tokens(lists[h, r].tolist(), n, nb, i * f * nb)
                _check(_np(O[h])[rows], _np(Q[h])[rows], rk[h, t], rv[h, t], d ** -0.5)
        # the chunk is finished: its keys and values go into the cache, its means into the pooled keys
        before = held.clone()
        lf.lf_kvq_append(K, V, held, cap, at)
        want = before.cpu().numpy()
        R.cache_write(want, H, cap, d, at, _np(K), _np(V))
        assert np.array_equal(held.cpu().numpy(), want)
        lf.lf_kcache_update(Kc[:, :kv], n, 64, (i - 1) * f, i * f, frames, pooled)
        # a few query rows over everything held so far, and the same chunk once more, now from the cache alone
        rows = rand(H, 5, d)
        rk, rv = R.cache_read(held.cpu().numpy(), H, cap, d, 0, kv)
        T = lf.lf_token_attn_kvq(rows, held, cap, kv)
        A = lf.lf_sparse_attn_kvq(Q, held, cap, kv, lists, n, 64)
        for h in range(H):
            _check(_np(T[h]), _np(rows[h]), rk[h], rv[h], d ** -0.5)
            t = R.block_tokens(lists[h, 0].tolist(), n, nb, i * f * nb)
            _check(_np(A[h])[:64], _np(Q[h])[:64], rk[h, t], rv[h, t], d ** -0.5)


def test_finetuning_step_through_the_producer(gpu):
    """Activations -> Q and K -> attention over lists -> gradients of Q and K -> gradients of the activations and the norm weight."""
    torch, lf = gpu
    H, d, n, f, F = 2, 64, 100, 2, 4
    q, kv = f * n, F * n
    g = torch.Generator().manual_seed(1)
    rand = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).cuda()
    w = (1.0 + 0.1 * torch.randn(H * d, generator=g)).cuda()
    freq = torch.cat([10000.0 ** (-torch.arange(k, dtype=torch.float64) / k) for k in PAIRS])
    Xq, Xk, V, dO = rand(q, H * d), rand(kv, H * d), rand(H, kv, d), rand(H, q, d)
    pos = _positions(torch, 0, F, n, 10)
    Q, K = torch.empty((H, q, d), dtype=torch.bfloat16, device="cuda"), torch.empty((H, kv, d), dtype=torch.bfloat16, device="cuda")
    _produced(torch, lf, Xq, w, pos[kv - q:], freq, H, Q)
    _produced(torch, lf, Xk, w, pos, freq, H, K)
    lists = torch.stack([torch.randperm(F * 2, generator=g)[:5].sort().values for _ in range(H * f * 2)]).to(torch.int32).view(H, f * 2, 5).cuda()
    O, lse = lf.lf_sparse_attn_fwd(Q, K, V, lists, n, 64)
    dQ, dK, dV = lf.lf_sparse_attn_bwd(Q, K, V, O, dO, lse, lists, n, 64)
    for X, p, dY in ((Xq, pos[kv - q:], dQ), (Xk, pos, dK)):
        dX, dw = lf.lf_qk_norm_rope_axes_bwd(X, w, p.cuda(), freq.cuda(), PAIRS, H, dY)
        theta = R.angles(p.numpy(), freq.numpy(), PAIRS)
        rX, rg, sX, sg = R.rope_axes_backward(_np(X), _np(w), theta, H, 1e-6, False, 0, _np(dY))
        _rel_ok(_np(dX), rX, sX, 2.0 ** -17)
        assert np.all(np.abs(_np(dw) - rg) <= 161 * 2.0 ** -24 * sg + 1e-37)
