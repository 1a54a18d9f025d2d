"""Attention over packed sequences and its gradients against their binary64 oracle, through the C ABI.

Bars, element by element, with half a step of bfloat16, 2^-8 of the value (the oracle returns the sums of absolute values A that they are in units of).
  O      every P is rounded to bfloat16, and the row's sum is that of the rounded ones: 2 x 2^-8 of A = sum P |v|; the output's own rounding; scores are
         float32 sums of 128 products at most, off by 2^-17 of sum |q k| scale (some 30 at the most here), and exp2 by 2^-22: 2^-11 of A.
  lse2   scores as above: 2^-12; the sum of rounded P: log2(1 + 2^-8) = 0.0057.
  dV     P once to bfloat16: 1.1 x 2^-8 of A, and the output.    dQ, dK   dS off by P times what O's bfloat16 leaves in delta, and by its own and P's
         rounding; the oracle adds that up: 1.1 x 2^-8 of it, and the output."""
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


def _make(torch, H, L, d, g, layout="heads", scale=1.0, pad=0):
    """[H, L, d] in a larger buffer of 7.0: heads outside tokens, or tokens outside heads."""
    x = (scale * torch.randn((H, L, d), generator=g)).to(torch.bfloat16)
    shape = (H, L + 3, d + pad) if layout == "heads" else (L + 3, H, d + pad)
    buf = torch.full(shape, 7.0, dtype=torch.bfloat16, device="cuda")
    view = (buf if layout == "heads" else buf.transpose(0, 1))[:, 3:, :d]
    view.copy_(x.cuda())
    return view, buf


def _np(t):
    return t.double().cpu().numpy()


def _ok(name, got, ref, size, unit, floor=2.0 ** -30):
    there = ~np.isnan(ref)
    err, bar = np.abs(got - ref)[there], (unit * size + HALF * np.abs(ref))[there] + floor
    assert np.all(err <= bar), (name, float((err / bar).max()))
    return there


def _run(gpu, H, Hk, d, q_start, kv_start, causal, q_len=None, kv_len=None, seed=0, layout="heads", pad=0, key_scale=1.0, softmax_scale=0.0, train=True):
    torch, lf = gpu
    q_len, kv_len = q_len or max(q_start[-1], 1), kv_len or max(kv_start[-1], 1)
    print(f"packed H={H} Hk={Hk} d={d} q={q_start} kv={kv_start} causal={causal} layout={layout} pad={pad}", flush=True)
    g = torch.Generator().manual_seed(seed)
    (Q, _), (K, _), (V, _), (dO, _) = (_make(torch, *a, d, g, layout, s, pad) for *a, s in ((H, q_len, 1.0), (Hk, kv_len, key_scale), (Hk, kv_len, 1.0), (H, q_len, 1.0)))
    O, Obuf = _make(torch, H, q_len, d, g, layout, 0.0, pad)
    Obuf.fill_(7.0)
    qs, ks = (torch.tensor(s, dtype=torch.int32, device="cuda") for s in (q_start, kv_start))
    shape = (H, Hk, d, len(q_start) - 1, q_len, kv_len, causal)
    lse2 = torch.full((H, q_len), 7.0, device="cuda")
    ws = torch.full((max(lf.lf_packed_attn_workspace_bytes(*shape), 256),), 255, dtype=torch.uint8, device="cuda")
    how = dict(causal=causal, softmax_scale=softmax_scale)
    lf.lf_packed_attn_fwd(Q, K, V, qs, ks, O=O, lse2=lse2, workspace=ws, **how)
    O2 = torch.full_like(Obuf, 7.0)
    O2 = (O2 if layout == "heads" else O2.transpose(0, 1))[:, 3:, :d]
    lf.lf_packed_attn(Q, K, V, qs, ks, O=O2, workspace=ws, **how)
    torch.cuda.synchronize()
    assert torch.equal(O, O2)
    scale = softmax_scale or d ** -0.5
    ref = R.packed_attention(_np(Q), _np(K), _np(V), q_start, kv_start, causal, scale, _np(dO) if train else None)
    got = _np(O)
    there = _ok("O", got, ref[0], ref[2], 2 * HALF + 2.0 ** -11)
    assert np.all(got[~there] == 7.0)
    assert (Obuf if layout == "heads" else Obuf.transpose(0, 1))[:, :3].eq(7.0).all() and Obuf[..., d:].eq(7.0).all()
    l, rows = _np(lse2), there.all(-1)
    assert np.array_equal(np.isposinf(l[rows]), np.isposinf(ref[1][rows])) and np.all(l[~rows] == 7.0)
    fine = rows & np.isfinite(ref[1])
    assert np.all(np.abs(l[fine] - ref[1][fine]) <= 0.0057 + 2.0 ** -12 + 2.0 ** -22 * np.abs(ref[1][fine]))
    assert np.all(got[rows & np.isposinf(ref[1])] == 0.0)
    if not train:
        return O, lse2
    big = [torch.full((t.stride(0) * t.shape[0] + t.stride(1) * t.shape[1] + d,), 7.0, dtype=torch.bfloat16, device="cuda").as_strided(t.shape, t.stride()) for t in (Q, K, V)]
    wsb = torch.full((max(lf.lf_packed_attn_bwd_workspace_bytes(*shape), 256),), 255, dtype=torch.uint8, device="cuda")
    lf.lf_packed_attn_bwd(Q, K, V, O, dO, lse2, qs, ks, workspace=wsb, grads=big, **how)
    torch.cuda.synchronize()
    for name, t, r, s in zip(("dQ", "dK", "dV"), big, ref[3], ref[4]):
        there = _ok(name, _np(t), r, s, 1.1 * HALF)
        assert np.all(_np(t)[~there] == 7.0), name
    return O, lse2, big


SEQS = [([0, 1], [0, 1]), ([0, 1], [0, 77]), ([0, 130], [0, 130]), ([0, 3, 3, 70, 71], [0, 5, 9, 9, 200]), ([2, 40, 173, 300], [1, 39, 172, 299]),
        ([0, 300], [0, 63]), ([0, 64, 192], [0, 128, 129]), ([0, 257], [0, 700])]


@pytest.mark.parametrize("seqs", SEQS, ids=lambda s: f"q{s[0]}kv{s[1]}")
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [0, 1, 48])
def test_forward_and_gradients(gpu, seqs, d, causal):
    for H, Hk in ((1, 1), (6, 2)):
        _run(gpu, H, Hk, d, *seqs, causal, q_len=seqs[0][-1] + 5, kv_len=seqs[1][-1] + 7, seed=d + causal, layout="tokens" if H == 6 else "heads", pad=8)


@pytest.mark.parametrize("causal", [2, 31, 32, 33, 64, 65, 128, 200, 1 << 30])
def test_chunks(gpu, causal):
    """Chunks that end before, at and behind the ends of tiles, with rows before their first token's chunk."""
    _run(gpu, 2, 1, 128, [0, 200, 333], [0, 200, 410], causal, seed=causal % 1000)
    _run(gpu, 2, 2, 64, [0, 150], [0, 90], causal, seed=causal % 999)


@pytest.mark.parametrize("n", [31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 255, 256, 257, 260])
def test_lengths_around_tiles(gpu, n):
    _run(gpu, 2, 1, 128, [0, n], [0, n], 1, seed=n)
    _run(gpu, 1, 1, 64, [0, n], [0, n + 1], 1, seed=n)
    _run(gpu, 1, 1, 128, [0, 5, 5 + n], [0, n, n + 3], 0, seed=n)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hk", [(1, 1), (5, 1), (12, 12), (40, 8), (17, 1), (32, 2), (48, 1), (64, 2)])
def test_single_rows_over_a_cache(gpu, H, Hk, d):
    """One row of each of several requests, lengths from none to long ones; more heads to a shared one than a tile has rows."""
    lens = [0, 1, 64, 65, 300, 1027]
    kv = [0] + list(np.cumsum(lens))
    _run(gpu, H, Hk, d, list(range(7)), [int(x) for x in kv], 1, seed=H, train=H <= 12, layout="tokens")


@pytest.mark.parametrize("rows", [2, 5, 16, 31, 32, 33])
@pytest.mark.parametrize("causal", [0, 1, 7])
def test_few_rows(gpu, rows, causal):
    """Both sides of the lines between the kernels of few and of many rows, and of tiles of 16 and 32."""
    _run(gpu, 6, 2, 128, [0, rows, 2 * rows], [0, 400, 3 * rows + 400], causal, seed=rows, train=False)
    _run(gpu, 1, 1, 64, [0, rows], [0, 2500], causal, seed=rows, train=False)


def test_few_rows_in_uneven_sequences(gpu):
    """A mean of few rows, but one sequence with many."""
    starts = [0, 1, 1, 130, 131, 132, 132, 133, 140]
    _run(gpu, 4, 2, 128, starts, [0, 20, 20, 900, 905, 1000, 1001, 1001, 1300], 1, seed=1)
    _run(gpu, 4, 1, 64, starts, [0, 20, 20, 900, 905, 1000, 1001, 1001, 1300], 50, seed=1)


@pytest.mark.parametrize("rows,tokens,causal", [(1, 40000, 1), (16, 9000, 0), (3, 20011, 7000), (40, 12000, 1), (130, 9000, 0), (300, 6001, 1)])
def test_a_long_axis_is_divided_and_joined(gpu, rows, tokens, causal):
    torch, lf = gpu
    H, Hk, d = 2, 1, 128
    assert lf.lf_packed_attn_workspace_bytes(H, Hk, d, 1, rows, tokens, causal) > 0
    _run(gpu, H, Hk, d, [0, rows], [0, tokens], causal, seed=rows, train=False)


def test_many_sequences(gpu):
    rng = np.random.default_rng(0)
    q, kv = np.concatenate([[0], np.cumsum(rng.integers(0, 9, 150))]), np.concatenate([[0], np.cumsum(rng.integers(0, 12, 150))])
    _run(gpu, 2, 1, 64, [int(x) for x in q], [int(x) for x in kv], 1, seed=4)
    q, kv = np.concatenate([[0], np.cumsum(rng.integers(30, 60, 80))]), np.concatenate([[0], np.cumsum(rng.integers(0, 90, 80))])
    _run(gpu, 2, 1, 128, [int(x) for x in q], [int(x) for x in kv], 0, seed=5)


def test_many_tokens_of_few_heads(gpu):
    """Enough tokens for the gradient kernel of 256 tokens a workgroup; three heads share one."""
    _run(gpu, 24, 8, 128, [0, 700, 1033, 1033, 1034, 2201, 4100], [0, 700, 1033, 1034, 1034, 2300, 4199], 1, seed=6, q_len=4103, kv_len=4203)


def test_many_tokens_by_chunks(gpu):
    _run(gpu, 16, 16, 128, [0, 1000, 2100], [0, 1000, 2100], 300, seed=7)


@pytest.mark.parametrize("H,Hk,q,kv,causal,layout,pad", [
    (24, 8, [0, 700, 1400], [0, 3001, 16500], 0, "heads", 0), (24, 8, [2, 702, 1403], [3, 3001, 16500], 0, "tokens", 8), (12, 12, [0, 700, 2100], [0, 0, 16500], 0, "heads", 16), (32, 32, [0, 1100], [0, 8193], 1, "tokens", 8),
    (27, 9, [3, 903, 1290], [5, 9000, 16500], 300, "heads", 24), (36, 9, [3, 903], [5, 16505], 300, "heads", 24), (24, 24, [0, 1500], [0, 16400], 5000, "tokens", 0), (16, 4, [0, 1, 1, 700, 2063], [0, 4000, 4100, 12000, 32900], 0, "tokens", 0),
    (12, 12, [0, 2100, 3074], [0, 1500, 20000], 1, "heads", 0)])
def test_many_rows_of_many_tokens(gpu, H, Hk, q, kv, causal, layout, pad):
    """The kernel of 64 rows a wavefront (8192 tokens or more seen in the mean), and causal calls of such sizes.  In some cases there are rows that see nothing."""
    _run(gpu, H, Hk, 128, q, kv, causal, seed=8, layout=layout, pad=pad, train=False)


@pytest.mark.parametrize("H,Hk,d,q,kv,causal", [(2, 1, 64, [0, 3, 150], [0, 9, 200], 1), (2, 2, 128, [0, 200], [0, 700], 0), (14, 14, 128, [0, 130], [0, 2051], 0)])
def test_the_smallest_scale(gpu, H, Hk, d, q, kv, causal):
    """All logits are 0 but for 1e-30 of something: means, in every gradient kernel."""
    _run(gpu, H, Hk, d, q, kv, causal, seed=13, softmax_scale=1.0000001e-30)


@pytest.mark.parametrize("n", [4200, 8200])
def test_many_rows_of_rising_logits(gpu, n):
    """Keys that grow along the tokens, then the same ones backwards: the reference moves at every tile, or only at the first."""
    torch, lf = gpu
    H, rows, d = 24, 1401, 128
    g = torch.Generator().manual_seed(3)
    u = torch.nn.functional.normalize(torch.randn(d, generator=g), dim=0)
    Q = (11.3 * u).repeat(1, rows, 1).to(torch.bfloat16)
    V = torch.randn((1, n, d), generator=g).to(torch.bfloat16)
    qs, ks = torch.tensor([0, rows], dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda")
    for order in (torch.arange(n), n - torch.arange(n)):
        K = (order[:, None] * u * (0.19 * 4200 / n)).to(torch.bfloat16)[None]
        O = lf.lf_packed_attn(Q.cuda().expand(H, rows, d).contiguous(), K.cuda().expand(H, n, d).contiguous(), V.cuda().expand(H, n, d).contiguous(), qs, ks)
        assert torch.equal(O, O[:1].expand_as(O))
        ref, _, size = R.packed_attention(_np(Q[:, :1]), _np(K), _np(V), [0, 1], [0, n], 0, d ** -0.5)
        # logits of up to 800, as below
        _ok("O", _np(O[:1]), np.broadcast_to(ref, (1, rows, d)), np.broadcast_to(size, (1, rows, d)), 2 * HALF + 2.0 ** -7)


@pytest.mark.parametrize("H,Hk,q,kv,causal", [(14, 14, [0, 600, 600, 1401, 2100], [0, 555, 777, 1300, 2051], 0), (39, 13, [0, 1, 2, 300], [0, 1, 258, 2310], 0),
                                              (118, 118, [0, 64, 700, 771], [0, 64, 700, 771], 1), (88, 44, [0, 1000, 2049], [0, 1000, 2049], 300)])
def test_gradients_of_many_tokens(gpu, H, Hk, q, kv, causal):
    """The gradient kernel of 256 tokens a workgroup: tokens x heads of 28 672 or more, 90 112 where rows see less than all."""
    _run(gpu, H, Hk, 128, q, kv, causal, seed=9)


@pytest.mark.parametrize("d,H,Hk,q,kv,causal", [(128, 64, 32, [0, 64, 500, 1100], [0, 64, 500, 1100], 1), (64, 64, 32, [0, 64, 500, 1100], [0, 64, 500, 1100], 0)])
def test_gradients_of_undivided_workgroups(gpu, d, H, Hk, q, kv, causal):
    """The gradient kernel of 64 tokens a workgroup, with enough of them for the chip."""
    _run(gpu, H, Hk, d, q, kv, causal, seed=10)


@pytest.mark.parametrize("seqs,rows", [(64, 32), (65, 32), (63, 33), (70, 4)])
def test_places_of_full_tiles(gpu, seqs, rows):
    """Sequences of whole tiles, so a place of each of them is left over; more than 64 find their tiles another way."""
    starts = [rows * i for i in range(seqs + 1)]
    for d, H, Hk in ((64, 2, 2), (128, 8, 1)):
        _run(gpu, H, Hk, d, starts, [7 * i + (i // 3) * 40 for i in range(seqs + 1)], 0, seed=11, train=False)
    _run(gpu, 2, 1, 64, [5 * rows * i for i in range(seqs + 1)], [rows * i for i in range(seqs + 1)], 0, seed=12)


def test_larger_keys_and_scales(gpu):
    """Logits of some hundreds: the reference of the softmax moves, and most probabilities vanish."""
    for d in (64, 128):
        for rows in (1, 200):
            _run(gpu, 2, 1, d, [0, rows], [0, 333], 1, seed=rows, key_scale=20.0, train=False)
            _run(gpu, 2, 1, d, [0, rows], [0, 333], 0, seed=rows, softmax_scale=1e-3)


def test_rising_logits_move_the_reference(gpu):
    """Keys that grow along the sequence, so every tile's scores are above those before."""
    torch, lf = gpu
    for rows in (4, 150):
        n, d = 900, 128
        g = torch.Generator().manual_seed(3)
        u = torch.nn.functional.normalize(torch.randn(d, generator=g), dim=0)
        Q = (11.3 * u).repeat(1, rows, 1).to(torch.bfloat16).cuda()
        K = (torch.arange(n)[:, None] * u * 0.9).to(torch.bfloat16)[None].cuda()
        V = torch.randn((1, n, d), generator=g).to(torch.bfloat16).cuda()
        qs, ks = torch.tensor([0, rows], dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda")
        O = lf.lf_packed_attn(Q, K, V, qs, ks, causal=1)
        ref, _, size = R.packed_attention(_np(Q), _np(K), _np(V), [0, rows], [0, n], 1, d ** -0.5)
        # logits of up to 800: products of some 10^4, a float32 score is off by 2^-24 x 8 steps of that, 2^-8 in the exponent
        _ok("O", _np(O), ref, size, 2 * HALF + 2.0 ** -7)


def test_a_row_that_sees_one_token(gpu):
    """It copies the token, and its scores have no gradient: exactly zero, in every kernel."""
    torch, lf = gpu
    for H, Hk, d, starts in ((2, 1, 64, [0, 1, 2]), (2, 1, 128, [0, 1, 2]), (16, 16, 128, list(range(0, 2300)))):
        n = starts[-1]
        g = torch.Generator().manual_seed(n)
        r = lambda h: torch.randn((h, n, d), generator=g).to(torch.bfloat16).cuda()
        Q, K, V, dO = r(H), r(Hk), r(Hk), r(H)
        s = torch.tensor(starts, dtype=torch.int32, device="cuda")
        for causal in (0, 1, 5):
            O, lse2 = lf.lf_packed_attn_fwd(Q, K, V, s, s, causal=causal)
            dQ, dK, dV = lf.lf_packed_attn_bwd(Q, K, V, O, dO, lse2, s, s, causal=causal)
            assert torch.equal(O, V.repeat_interleave(H // Hk, 0)) and (dQ == 0).all() and (dK == 0).all()
            want = dO.double().view(Hk, H // Hk, n, d).sum(1)
            assert ((dV.double() - want).abs() <= HALF * want.abs() + 2.0 ** -20 * dO.double().abs().view(Hk, -1, n, d).sum(1)).all()
        # causal: the first of several rows
        one = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        O, lse2 = lf.lf_packed_attn_fwd(Q, K, V, one, one, causal=1)
        dQ, dK, dV = lf.lf_packed_attn_bwd(Q, K, V, O, dO, lse2, one, one, causal=1)
        assert (dQ[:, 0] == 0).all() and (n < 3 or (dQ[:, 2] != 0).any())


def test_short_sequences_keep_their_gradients_precision(gpu):
    """Sequences of two to four tokens with large keys: nearly all of a row's probability lies on one token.  The roundings are dS's (2^-9 of the value with the
    standard deviation of 2^-9 / sqrt 3 x 2), P's and the output's, independent: below 3.2e-3 in the 2-norm."""
    torch, lf = gpu
    starts = list(np.concatenate([[0], np.cumsum([2, 3, 4] * 8)]))
    n, H, d = int(starts[-1]), 8, 128
    for key_scale in (1.0, 3.0):
        g = torch.Generator().manual_seed(5)
        r = lambda s=1.0: (s * torch.randn((H, n, d), generator=g)).to(torch.bfloat16).cuda()
        Q, K, V, dO = r(), r(key_scale), r(), r()
        s = torch.tensor(starts, dtype=torch.int32, device="cuda")
        O, lse2 = lf.lf_packed_attn_fwd(Q, K, V, s, s, causal=1)
        got = lf.lf_packed_attn_bwd(Q, K, V, O, dO, lse2, s, s, causal=1)
        ref = R.packed_attention(_np(Q), _np(K), _np(V), [int(x) for x in starts], [int(x) for x in starts], 1, d ** -0.5, _np(dO))[3]
        for name, a, b in zip(("dQ", "dK", "dV"), got, ref):
            rel = np.linalg.norm(_np(a) - b) / np.linalg.norm(b)
            print(key_scale, name, rel)
            assert rel <= 3.2e-3, name


def test_few_rows_are_as_exact_as_their_output(gpu):
    """16 rows of a tile and fewer keep 16 bits of P: the output's rounding is what is left (2^-9 x 2 / sqrt 12 = 1.1e-3 at the least, 1.7e-3 over a binade)."""
    torch, lf = gpu
    O, _ = _run(gpu, 12, 12, 128, [0, 1], [0, 5000], 1, seed=2, train=False)
    g = torch.Generator().manual_seed(9)
    Q, K, V = ((torch.randn((h, n, 128), generator=g)).to(torch.bfloat16).cuda() for h, n in ((12, 1), (12, 5000), (12, 5000)))
    s = [torch.tensor([0, n], dtype=torch.int32, device="cuda") for n in (1, 5000)]
    ref = R.packed_attention(_np(Q), _np(K), _np(V), [0, 1], [0, 5000], 1, 128 ** -0.5)[0]
    got = _np(lf.lf_packed_attn(Q, K, V, *s, causal=1))
    assert np.linalg.norm(got - ref) / np.linalg.norm(ref) <= 1.9e-3


def test_gradient_against_differences(gpu):
    """The derivative of <O, dO> along a direction of V (O is linear in it: no curvature) and of Q.  bfloat16 leaves 2^-8 of O in each of two calls, and P's
    roundings half of that more, independent."""
    torch, lf = gpu
    H, n, d = 2, 96, 64
    g = torch.Generator().manual_seed(8)
    r = lambda: torch.randn((H, n, d), generator=g).to(torch.bfloat16).cuda()
    Q, K, V, dO = r(), r(), r(), r()
    s = torch.tensor([0, 40, n], dtype=torch.int32, device="cuda")
    O, lse2 = lf.lf_packed_attn_fwd(Q, K, V, s, s, causal=1)
    dQ, dK, dV = lf.lf_packed_attn_bwd(Q, K, V, O, dO, lse2, s, s, causal=1)
    for which, grad, h in ((2, dV, 0.5), (0, dQ, 0.125), (1, dK, 0.125)):
        dirn = torch.randint(-1, 2, (H, n, d), generator=g).cuda().float()
        args = [Q, K, V]
        up, down = (args[which].float() + h * dirn).to(torch.bfloat16), (args[which].float() - h * dirn).to(torch.bfloat16)
        step = (up.double() - down.double())              # what was really moved
        f = lambda x: lf.lf_packed_attn(*[x if i == which else t for i, t in enumerate(args)], s, s, causal=1).double() * dO.double()
        a, b = f(up), f(down)
        diff, exact = float((a - b).sum()), float((grad.double() * step).sum())
        noise = 5 * 1.2 * HALF * float((a.square() + b.square()).sum().sqrt()) + 5 * HALF * float((grad.double() * step).norm())
        curve = 0.0 if which == 2 else h * h * float((grad.double() * step).abs().sum())
        print(which, "difference", diff, "gradient", exact, "bars", noise, curve)
        assert abs(diff - exact) <= noise + curve


def test_no_rows_and_no_tokens(gpu):
    torch, lf = gpu
    H, d = 2, 64
    z = lambda n: torch.randn((H, n, d), device="cuda").to(torch.bfloat16)
    s = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    assert lf.lf_packed_attn(z(0), z(4), z(4), s(0, 0), s(0, 4)).shape == (H, 0, d)
    Q, dO = z(5), z(5)
    O, lse2 = lf.lf_packed_attn_fwd(Q, z(0), z(0), s(0, 5), s(0, 0))
    assert (O == 0).all() and torch.isposinf(lse2).all()
    dQ, dK, dV = lf.lf_packed_attn_bwd(Q, z(0), z(0), O, dO, lse2, s(0, 5), s(0, 0))
    assert (dQ == 0).all() and dK.shape == (H, 0, d)
    K = z(4)
    dQ, dK, dV = lf.lf_packed_attn_bwd(z(0), K, K, z(0), z(0), torch.empty((H, 0), device="cuda"), s(0, 0), s(0, 4))
    assert (dK == 0).all() and (dV == 0).all()


def test_starts_of_any_values_touch_nothing_outside(gpu):
    """Offsets out of range and out of order: what is written stays inside the tensors (results then mean nothing)."""
    torch, lf = gpu
    H, n, d = 2, 90, 64
    g = torch.Generator().manual_seed(1)
    for starts in ([-5, 200], [90, 0], [50, 10, 70, 3], [2 ** 31 - 1, -2 ** 31, 40], [0, 90, 0, 90]):
        (Q, _), (K, _), (V, _), (dO, _) = (_make(torch, H, n, d, g) for _ in range(4))
        O, buf = _make(torch, H, n, d, g, scale=0.0)
        s = torch.tensor(starts, dtype=torch.int64).to(torch.int32).cuda()
        lse2 = torch.zeros((H, n), device="cuda")
        lf.lf_packed_attn_fwd(Q, K, V, s, s, causal=1, O=O, lse2=lse2)
        grads = [_make(torch, H, n, d, g, scale=0.0) for _ in range(3)]
        lf.lf_packed_attn_bwd(Q, K, V, O, dO, lse2, s, s, causal=1, grads=[v for v, _ in grads])
        torch.cuda.synchronize()
        for b in [buf] + [b for _, b in grads]:
            assert (b[:, :3] == 7.0).all()


@pytest.mark.parametrize("H,Hk,d,q,kv,causal", [(4, 2, 64, [5, 38, 201], [3, 70, 180], 1), (4, 2, 128, [5, 38, 201], [3, 70, 180], 0), (8, 2, 128, [2, 3, 5], [70, 800, 3001], 1),
                                                (8, 2, 64, [2, 22, 49], [70, 800, 3001], 0), (14, 14, 128, [7, 70, 141], [5, 1000, 2060], 0), (30, 30, 128, [9, 1100], [2, 8300], 1), (30, 30, 128, [9, 1100], [2, 8300], 0)])
def test_nan_beside_the_sequences_stays_there(gpu, H, Hk, d, q, kv, causal):
    """Rows and tokens of no sequence hold NaN, in every kernel."""
    torch, lf = gpu
    L, T = q[-1] + 9, kv[-1] + 77
    print(f"nan beside H={H} Hk={Hk} d={d} q={q} kv={kv} causal={causal}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(0)
    make = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    Q, K, V, dO = make(H, L, d), make(Hk, T, d), make(Hk, T, d), make(H, L, d)
    qs, ks = (torch.tensor(s, dtype=torch.int32, device="cuda") for s in (q, kv))
    results = []
    for beside in (0.0, float("nan")):
        for t, s in ((Q, q), (dO, q), (K, kv), (V, kv)):
            t[:, :s[0]] = beside
            t[:, s[-1]:] = beside
        O, lse2 = torch.full_like(Q, beside), torch.full((H, L), beside, device="cuda")
        lf.lf_packed_attn_fwd(Q, K, V, qs, ks, causal=causal, O=O, lse2=lse2)
        grads = lf.lf_packed_attn_bwd(Q, K, V, O, dO, lse2, qs, ks, causal=causal)
        results.append([O[:, q[0]:q[-1]], lse2[:, q[0]:q[-1]], grads[0][:, q[0]:q[-1]]] + [x[:, kv[0]:kv[-1]] for x in grads[1:]])
    for a, b in zip(*results):
        assert torch.equal(a, b) and not torch.isnan(a).any()


def test_results_are_the_same_again_and_on_another_stream(gpu):
    torch, lf = gpu
    g = torch.Generator().manual_seed(4)
    H, Hk, n, d = 6, 2, 700, 128
    r = lambda h: torch.randn((h, n, d), generator=g).to(torch.bfloat16).cuda()
    Q, K, V, dO = r(H), r(Hk), r(Hk), r(H)
    s = torch.tensor([0, 333, 700], dtype=torch.int32, device="cuda")
    O, lse2 = lf.lf_packed_attn_fwd(Q, K, V, s, s, causal=1)
    a = lf.lf_packed_attn_bwd(Q, K, V, O, dO, lse2, s, s, causal=1)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    O2, l2 = lf.lf_packed_attn_fwd(Q, K, V, s, s, causal=1, stream=st)
    b = lf.lf_packed_attn_bwd(Q, K, V, O2, dO, l2, s, s, causal=1, stream=st)
    st.synchronize()
    assert torch.equal(O, O2) and torch.equal(lse2, l2) and all(torch.equal(x, y) for x, y in zip(a, b))


def test_captured_steps_replay_with_other_lengths(gpu):
    """Training over packed sequences, and single rows over a cache: the offsets are read on the device."""
    torch, lf = gpu
    g = torch.Generator().manual_seed(6)
    r = lambda h, n, d: torch.randn((h, n, d), generator=g).to(torch.bfloat16).cuda()
    H, Hk, n, d = 4, 2, 400, 64
    Q, K, V, dO = r(H, n, d), r(Hk, n, d), r(Hk, n, d), r(H, n, d)
    q1, k1, v1 = r(8, 3, 128), r(2, 6000, 128), r(2, 6000, 128)
    s = torch.tensor([0, 100, 400], dtype=torch.int32, device="cuda")
    sq, sk = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda"), torch.tensor([0, 10, 3000, 6000], dtype=torch.int32, device="cuda")
    O, O1 = torch.zeros_like(Q), torch.zeros_like(q1)
    lse2, grads = torch.zeros((H, n), device="cuda"), [torch.zeros_like(t) for t in (Q, K, V)]
    ws = torch.empty(max(lf.lf_packed_attn_workspace_bytes(H, Hk, d, 2, n, n, 1), 256), dtype=torch.uint8, device="cuda")
    wsb = torch.empty(lf.lf_packed_attn_bwd_workspace_bytes(H, Hk, d, 2, n, n, 1), dtype=torch.uint8, device="cuda")
    ws1 = torch.empty(lf.lf_packed_attn_workspace_bytes(8, 2, 128, 3, 3, 6000, 1), dtype=torch.uint8, device="cuda")

    def step():
        lf.lf_packed_attn_fwd(Q, K, V, s, s, causal=1, O=O, lse2=lse2, workspace=ws)
        lf.lf_packed_attn_bwd(Q, K, V, O, dO, lse2, s, s, causal=1, grads=grads, workspace=wsb)
        lf.lf_packed_attn(q1, k1, v1, sq, sk, causal=1, O=O1, workspace=ws1)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    outs = [O, O1, lse2] + grads
    for k in range(3):
        Q.copy_(torch.randn(Q.shape, device="cuda").to(torch.bfloat16))
        s.copy_(torch.tensor([0, 37 + 90 * k, 400], dtype=torch.int32))
        sk.copy_(torch.tensor([0, 2000 * k, 5000, 5900], dtype=torch.int32))
        step()
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs)), k


def test_offsets_beyond_32_bits(gpu):
    """A cache whose heads lie more than 2^32 bytes apart and whose last tokens lie behind 2^31 elements."""
    torch, lf = gpu
    n, d = 5_000_000, 128
    big = torch.zeros((2, 2 * n, d), dtype=torch.bfloat16, device="cuda")       # 5 GB: [K | V] of two heads
    K, V = big[:, :n], big[:, n:]
    g = torch.Generator().manual_seed(0)
    tail = 700
    for t in (K, V):
        t[:, n - tail:] = torch.randn((2, tail, d), generator=g).to(torch.bfloat16).cuda()
    Q = torch.randn((2, 3, d), generator=g).to(torch.bfloat16).cuda()
    qs, ks = torch.tensor([0, 0, 3], dtype=torch.int32, device="cuda"), torch.tensor([0, n - tail, n], dtype=torch.int32, device="cuda")
    got = _np(lf.lf_packed_attn(Q, K, V, qs, ks, causal=1))
    ref, _, size = R.packed_attention(_np(Q), _np(K[:, n - tail:]), _np(V[:, n - tail:]), [0, 0, 3], [0, 0, tail], 1, d ** -0.5)
    _ok("O", got, ref, size, 2 * HALF + 2.0 ** -11)


def test_binding_refuses(gpu):
    torch, lf = gpu
    r = lambda *s: torch.randn(s, device="cuda").to(torch.bfloat16)
    Q, K, V = r(4, 8, 64), r(2, 8, 64), r(2, 8, 64)
    s = torch.tensor([0, 8], dtype=torch.int32, device="cuda")
    ok = dict(Q=Q, K=K, V=V, q_start=s, kv_start=s)
    O, lse2 = lf.lf_packed_attn_fwd(**ok)
    for bad in (dict(Q=Q.float()), dict(Q=Q.cpu()), dict(K=K[:, :, :32]), dict(V=V[:1]), dict(q_start=s.long()), dict(q_start=s[:1]), dict(kv_start=torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda")),
                dict(kv_start=s.cpu()), dict(O=Q[:2]), dict(causal=1 << 40), dict(Q=Q.transpose(1, 2)), dict(workspace=torch.empty(4, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            lf.lf_packed_attn(**{**ok, **bad})
    for bad in (dict(causal=-1), dict(softmax_scale=-1.0), dict(softmax_scale=float("nan")), dict(Q=r(3, 8, 64)), dict(Q=r(4, 8, 32), K=r(2, 8, 32), V=r(2, 8, 32))):
        with pytest.raises(lf.LfError):
            lf.lf_packed_attn(**{**ok, **bad})
    with pytest.raises(lf.LfError):        # heads of the output that share elements
        lf.lf_packed_attn(**ok, O=torch.empty(4096, dtype=torch.bfloat16, device="cuda").as_strided((4, 8, 64), (0, 64, 1)))
    with pytest.raises(ValueError):
        lf.lf_packed_attn_fwd(**ok, lse2=torch.empty((4, 7), device="cuda"))
    for bad in (dict(dO=O[:2]), dict(dO=O.transpose(0, 1).contiguous().transpose(0, 1)), dict(lse2=lse2.double()), dict(grads=(Q, K, V[:1])), dict(grads=(Q.float(), K, V))):
        with pytest.raises(ValueError):
            lf.lf_packed_attn_bwd(**{**ok, **dict(O=O, dO=O.clone(), lse2=lse2), **bad})
    with pytest.raises(lf.LfError):
        lf.lf_packed_attn_bwd(**ok, O=O, dO=O.clone(), lse2=lse2, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
