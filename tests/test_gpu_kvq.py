"""The 4-bit cache (store, read back) and attention over it against their binary64 oracle, through the C ABI.

Bars.  Codes and scales are whole numbers: equal, byte for byte.  Attention: a probability is rounded to bfloat16 for its product (half a
step, 2^-8 of it) and so is the output; a score is a float32 sum of d products and meets two more roundings and exp2's, (d + 8) 2^-24 of the sum of
its terms' sizes, twice (also in the row's sum); and the float32 sums over T tokens add (T + 300) 2^-24 at the most, with A the mean of |v|:
    |error| <= 2^-8 |O| + (2^-8 + 2 (d + 8) 2^-24 max sum |q k| scale + (T + 300) 2^-24) A + 2^-26 max |v|.
The last term: the bfloat16 kernels, which calls with many tiles run on the cache's rows, let a row's sum grow to 1e30 = 2^99.7 against the row's
reference before they move that up and scale what was summed, by a factor that float32 flushes to zero below 2^-126.  What is lost then weighs less than
2^(99.7 - 126) < 2^-26 of the row's sum, which the new reference makes at least 1.  It shows where the v of the heavy tokens are zero, as many in
4 bits are, so that A says little."""
import numpy as np
import pytest

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


def _rand(torch, seed, *shape, scale=1.0):
    return (scale * torch.randn(shape, generator=torch.Generator().manual_seed(seed))).to(torch.bfloat16)


def _np(t):
    return t.double().cpu().numpy()


def _cache(gpu, H, cap, d, K, V, first=0):
    """A cache on the GPU and its bytes by the oracle; what nobody wrote holds noise (scale bytes of NaN among it)."""
    torch, lf = gpu
    noise = torch.randint(0, 256, (lf.lf_kvq_bytes(H, d, cap),), generator=torch.Generator().manual_seed(9), dtype=torch.uint8)
    dev, host = noise.cuda(), noise.numpy().copy()
    if K.shape[1]:
        lf.lf_kvq_append(K.cuda(), V.cuda(), dev, cap, first)
        R.cache_write(host, H, cap, d, first, _np(K), _np(V))
    return dev, host


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,L,first,room", [(1, 1, 0, 0), (1, 1, 3, 0), (3, 31, 5, 2), (2, 77, 0, 100), (12, 64, 63, 1), (5, 300, 4680, 7)])
def test_store_and_read_back(gpu, d, H, L, first, room):
    torch, lf = gpu
    print(f"store d={d} H={H} L={L} first={first}", flush=True)
    cap = first + L + room
    K, V = _rand(torch, L, H, L, d, scale=3.0), _rand(torch, L + 1, H, L, d)
    dev, host = _cache(gpu, H, cap, d, K, V, first)
    assert np.array_equal(dev.cpu().numpy(), host)
    k, v = lf.lf_kvq_read(dev, H, d, cap, first, L)
    rk, rv = R.cache_read(host, H, cap, d, first, first + L)
    assert np.array_equal(_np(k), rk) and np.array_equal(_np(v), rv)


@pytest.mark.parametrize("d", [64, 128])
def test_every_value_and_special_groups(gpu, d):
    """All bfloat16 bit patterns as the largest of their group, with zeros, small ones and ties beside them; groups with infinities and NaN."""
    torch, lf = gpu
    bits = torch.arange(1 << 16, dtype=torch.int32)
    bits = torch.where(bits >= 1 << 15, bits - (1 << 16), bits).to(torch.int16)
    x = torch.zeros((1 << 16, 32), dtype=torch.bfloat16)
    x[:, 5] = bits.view(torch.bfloat16)
    for i, f in enumerate((1 / 16, 1 / 8, 3 / 16, 1 / 4, 3 / 8, 1 / 2, 5 / 8, 3 / 4, 7 / 8, 15 / 16)):
        x[:, 8 + i] = (x[:, 5].double() * f * (-1) ** i).to(torch.bfloat16)
    big = x[:, 5].float().abs() > 2.9e38
    x[big & torch.isfinite(x[:, 5].float())] = 1.0          # (come back as infinity)
    K = x.reshape(1, -1, d)
    dev, host = _cache(gpu, 1, K.shape[1], d, K, -K)
    assert np.array_equal(dev.cpu().numpy(), host)
    k, v = lf.lf_kvq_read(dev, 1, d, K.shape[1], 0, K.shape[1])
    rk, _ = R.cache_read(host, 1, K.shape[1], d, 0, K.shape[1])
    assert np.array_equal(_np(k), rk, equal_nan=True) and np.array_equal(_np(v), -rk, equal_nan=True)
    assert np.isnan(rk).any()


def test_store_from_token_major_rows_and_into_views(gpu):
    """Strides of a projection's output (token-major), one head shared by all, and outputs inside larger tensors."""
    torch, lf = gpu
    H, L, d, cap = 3, 50, 64, 60
    rows = _rand(torch, 1, L, H * d + 16).cuda()
    K = rows[:, :H * d].view(L, H, d).transpose(0, 1)
    V = _rand(torch, 2, 1, L, d).cuda().expand(H, L, d)
    dev = torch.zeros(lf.lf_kvq_bytes(H, d, cap), dtype=torch.uint8, device="cuda")
    lf.lf_kvq_append(K, V, dev, cap, 7)
    host = np.zeros(dev.numel(), dtype=np.uint8)
    R.cache_write(host, H, cap, d, 7, _np(K), _np(V))
    assert np.array_equal(dev.cpu().numpy(), host)
    buf = torch.full((2, H, L + 4, d + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    lf.lf_kvq_read(dev, H, d, cap, 7, L, K=buf[0, :, 2:L + 2, :d], V=buf[1, :, 2:L + 2, :d])
    rk, rv = R.cache_read(host, H, cap, d, 7, 7 + L)
    assert np.array_equal(_np(buf[0, :, 2:L + 2, :d]), rk) and np.array_equal(_np(buf[1, :, 2:L + 2, :d]), rv)
    assert (buf[:, :, :2] == 7).all() and (buf[:, :, L + 2:] == 7).all() and (buf[..., d:] == 7).all()
    lf.lf_kvq_append(K[:, :0], V[:, :0], dev, cap, 60)          # nothing to do
    assert np.array_equal(dev.cpu().numpy(), host)


def _check(got, Q, K, V, scale):
    ref, size, terms = R.attention(Q, K, V, scale)
    T, d = len(K), Q.shape[1]
    bar = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2 * (d + 8) * 2.0 ** -24 * terms + (T + 300) * 2.0 ** -24) * size + 2.0 ** -26 * np.abs(V).max(initial=0) + 1e-37
    assert np.all(np.abs(got - ref) <= bar), (float((np.abs(got - ref) / bar).max()), T)


def _token(gpu, H, d, rows, cached, extra, seed=0, qscale=1.0, room=3, scale=0.0):
    torch, lf = gpu
    print(f"token H={H} d={d} rows={rows} cached={cached} extra={extra}", flush=True)
    Q = _rand(torch, seed, H, rows, d, scale=qscale)
    K, V = _rand(torch, seed + 1, H, cached, d), _rand(torch, seed + 2, H, cached, d)
    Kx, Vx = _rand(torch, seed + 3, H, extra, d), _rand(torch, seed + 4, H, extra, d)
    dev, host = _cache(gpu, H, cached + room, d, K, V)
    buf = torch.full((H, rows + 2, d + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    more = dict(K=Kx.cuda(), V=Vx.cuda()) if extra else {}
    O = lf.lf_token_attn_kvq(Q.cuda(), dev, cached + room, cached, O=buf[:, 1:rows + 1, :d], softmax_scale=scale, **more)
    torch.cuda.synchronize()
    rk, rv = R.cache_read(host, H, cached + room, d, 0, cached)
    for h in range(H):
        _check(_np(O[h]), _np(Q[h]), np.concatenate((rk[h], _np(Kx[h]))), np.concatenate((rv[h], _np(Vx[h]))), scale or d ** -0.5)
    assert (buf[:, 0] == 7).all() and (buf[:, rows + 1:] == 7).all() and (buf[..., d:] == 7).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [1, 16, 17, 33, 64])
def test_token_attention_rows_and_lengths(gpu, d, rows):
    for cached, extra in ((1, 0), (0, 1), (31, 1), (32, 32), (33, 0), (64, 65), (65, 0), (777, 33)):
        _token(gpu, 2, d, rows, cached, extra, seed=cached + rows)


@pytest.mark.parametrize("H,rows,cached,extra", [(1, 1, 9000, 1), (3, 5, 5001, 70), (12, 1, 2500, 0), (40, 3, 1300, 3), (1, 64, 4111, 64), (600, 1, 70, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_token_attention_divided_lists(gpu, d, H, rows, cached, extra):
    _token(gpu, H, d, rows, cached, extra, seed=H)


@pytest.mark.parametrize("d", [64, 128])
def test_token_attention_scores_far_apart(gpu, d):
    """Scores of hundreds, a scale given by the caller, references that have to move."""
    _token(gpu, 2, d, 7, 1500, 20, qscale=30.0)
    _token(gpu, 2, d, 40, 1500, 20, qscale=0.01, scale=0.5)


def test_token_attention_without_a_token(gpu):
    torch, lf = gpu
    cache = torch.full((lf.lf_kvq_bytes(2, 64, 8),), 255, dtype=torch.uint8, device="cuda")
    Q = torch.ones((2, 5, 64), dtype=torch.bfloat16, device="cuda")
    O = torch.full_like(Q, 7.0)
    assert (lf.lf_token_attn_kvq(Q, cache, 8, 0, O=O) == 0).all()
    empty = torch.empty((2, 0, 64), dtype=torch.bfloat16, device="cuda")
    assert (lf.lf_token_attn_kvq(Q, cache, 8, 0, K=empty, V=empty) == 0).all()


def test_query_heads_that_share_a_cached_head(gpu):
    """Four query heads of one token over each cached head, as rows."""
    torch, lf = gpu
    H, G, d, T = 3, 4, 128, 333
    Q = _rand(torch, 0, H * G, 1, d).cuda()
    dev, host = _cache(gpu, H, T, d, _rand(torch, 1, H, T, d), _rand(torch, 2, H, T, d))
    O = lf.lf_token_attn_kvq(Q.view(H, G, d), dev, T, T).view(H * G, 1, d)
    rk, rv = R.cache_read(host, H, T, d, 0, T)
    for h in range(H * G):
        _check(_np(O[h]), _np(Q[h]), rk[h // G], rv[h // G], d ** -0.5)


def test_a_cache_beyond_32_bit_offsets(gpu):
    """Codes of K alone take more than 4 GiB: the last head's last tokens are stored, read and seen where they belong."""
    torch, lf = gpu
    H, d, cap, L = 6, 128, 12_000_000, 200
    assert H * cap * d // 2 > 1 << 32
    cache = torch.zeros(lf.lf_kvq_bytes(H, d, cap), dtype=torch.uint8, device="cuda")
    K, V = _rand(torch, 1, H, L, d), _rand(torch, 2, H, L, d)
    lf.lf_kvq_append(K.cuda(), V.cuda(), cache, cap, cap - L)
    k, v = lf.lf_kvq_read(cache, H, d, cap, cap - L, L)
    for x, y in ((K, k), (V, v)):
        assert np.array_equal(_np(y), R.values(*R.quantise(_np(x))))
    assert sum(int(part.ne(0).sum()) for part in cache.split(1 << 30)) <= 2 * H * L * (d // 2 + d // 32)
    lf.lf_kvq_append(K.cuda(), V.cuda(), cache, cap, 0)
    Q = _rand(torch, 3, H, 2, d).cuda()
    O = lf.lf_token_attn_kvq(Q, cache, cap, L)
    for h in range(H):
        _check(_np(O[h]), _np(Q[h]), R.values(*R.quantise(_np(K[h]))), R.values(*R.quantise(_np(V[h]))), d ** -0.5)


def _lists(torch, kind, H, n_q, n_k, length, seed):
    g = torch.Generator().manual_seed(seed)
    idx = torch.rand((H, n_q, n_k), generator=g).argsort(-1)[..., :length].to(torch.int32)
    if idx.shape[-1] < length:
        idx = torch.cat((idx, torch.full((H, n_q, length - idx.shape[-1]), -1, dtype=torch.int32)), -1)
    if kind == "odd":            # ids that are none, and one twice
        idx[:, :, 0] = torch.tensor([-1, n_k, -(1 << 31), (1 << 31) - 1])[torch.arange(n_q) % 4].to(torch.int32)
        if length > 2:
            idx[:, :, 1] = idx[:, :, 2]
    if kind == "empty":          # every second list holds nothing
        idx[:, ::2] = -1
    return idx.contiguous()


def _sparse(gpu, H, d, n, f, F, length, kind="plain", own=True, seed=0, qscale=1.0):
    torch, lf = gpu
    print(f"sparse H={H} d={d} n={n} f={f} F={F} list={length} {kind} own={own}", flush=True)
    nb = -(-n // 64)
    q, kv, n_q, n_k = f * n, F * n, f * nb, F * nb
    Q, K, V = _rand(torch, seed, H, q, d, scale=qscale), _rand(torch, seed + 1, H, kv, d), _rand(torch, seed + 2, H, kv, d)
    held = kv - q if own else kv
    dev, host = _cache(gpu, H, max(1, held), d, K[:, :held], V[:, :held])
    idx = _lists(torch, kind, H, n_q, n_k, length, seed)
    buf = torch.full((H, q + 2, d + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    O = buf[:, 1:q + 1, :d]
    Kd, Vd = K.cuda(), V.cuda()
    more = dict(K=Kd[:, held:], V=Vd[:, held:]) if own else {}
    lf.lf_sparse_attn_kvq(Q.cuda(), dev, max(1, held), kv, idx.cuda(), n, 64, O=O, **more)
    torch.cuda.synchronize()
    rk, rv = R.cache_read(host, H, max(1, held), d, 0, held)
    rk, rv = np.concatenate((rk, _np(K[:, held:])), 1), np.concatenate((rv, _np(V[:, held:])), 1)
    got = _np(O)
    for h in range(H):
        for r in range(n_q):
            rows = R.block_tokens([r], n, nb, n_q)
            t = R.block_tokens(idx[h, r].tolist(), n, nb, n_k)
            _check(got[h, rows], _np(Q[h])[rows], rk[h, t], rv[h, t], d ** -0.5)
    assert (buf[:, 0] == 7).all() and (buf[:, q + 1:] == 7).all() and (buf[..., d:] == 7).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("own", [True, False])
@pytest.mark.parametrize("n", [1, 16, 20, 33, 64, 65, 97, 200])
def test_sparse_attention_frames_and_lists(gpu, d, own, n):
    nb = -(-n // 64)
    for kind, length in (("plain", 3 * nb), ("odd", 2 * nb + 1), ("empty", 2)):
        _sparse(gpu, 2, d, n, 2, 5, length, kind, own, seed=n)


@pytest.mark.parametrize("d", [64, 128])
def test_sparse_attention_without_a_history(gpu, d):
    _sparse(gpu, 2, d, 97, 3, 3, 5, own=True)
    _sparse(gpu, 2, d, 97, 3, 3, 6, own=False)


@pytest.mark.parametrize("H,d,n,f,F,length", [(1, 128, 64, 1, 80, 70), (2, 64, 130, 1, 40, 100), (12, 128, 64, 1, 12, 12), (5, 64, 64, 13, 20, 20),
                                              (7, 128, 200, 3, 9, 30), (12, 128, 320, 3, 9, 25), (12, 64, 320, 5, 10, 30)])
def test_sparse_attention_few_and_many_query_blocks(gpu, H, d, n, f, F, length):
    _sparse(gpu, H, d, n, f, F, length, seed=H)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("own", [True, False])
@pytest.mark.parametrize("kind", ["plain", "odd", "empty"])
@pytest.mark.parametrize("H,n,f,F,length,rows_first", [(3, 97, 2, 6, 5, False), (2, 33, 1, 70, 60, False), (24, 97, 3, 8, 14, True), (100, 20, 3, 9, 9, True)])
def test_sparse_attention_both_ways(gpu, H, d, n, f, F, length, rows_first, own, kind):
    """Calls that convert what they read and calls that write the cache's rows in bfloat16 first: the workspace says which."""
    torch, lf = gpu
    need = lf.lf_sparse_attn_kvq_workspace_bytes(H, d, n, 64, f * n, F * n, length)
    padded = (H * F * n * d * 2 + 255) // 256 * 256
    assert (need == 2 * padded) == rows_first
    _sparse(gpu, H, d, n, f, F, length, kind, own, seed=H)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,n,f,F,length", [(1, 64, 1, 70, 60), (24, 130, 2, 6, 12)])
def test_sparse_attention_scores_far_apart(gpu, d, H, n, f, F, length):
    _sparse(gpu, H, d, n, f, F, length, qscale=30.0)


def test_sparse_attention_strides_of_the_current_chunk(gpu):
    """Q, K, V as views of token-major rows, in both ways; rows of a workspace that held NaN."""
    torch, lf = gpu
    for H, d, n, f, F, length in ((2, 64, 70, 1, 5, 6), (40, 64, 70, 2, 5, 10)):
        nb, q, kv = -(-n // 64), f * n, F * n
        rows = _rand(torch, 3, q, 3 * H * d).cuda()
        Q, K, V = (rows[:, i * H * d:(i + 1) * H * d].view(q, H, d).transpose(0, 1) for i in range(3))
        dev, host = _cache(gpu, H, kv, d, _rand(torch, 4, H, kv - q, d), _rand(torch, 5, H, kv - q, d))
        idx = _lists(torch, "plain", H, f * nb, F * nb, length, 0)
        need = lf.lf_sparse_attn_kvq_workspace_bytes(H, d, n, 64, q, kv, length)
        ws = torch.full((max(need, 256),), 255, dtype=torch.uint8, device="cuda")
        O = _np(lf.lf_sparse_attn_kvq(Q, dev, kv, kv, idx.cuda(), n, 64, K=K, V=V, workspace=ws))
        rk, rv = R.cache_read(host, H, kv, d, 0, kv - q)
        rk, rv = np.concatenate((rk, _np(K)), 1), np.concatenate((rv, _np(V)), 1)
        for h in range(H):
            for r in range(f * nb):
                at, t = R.block_tokens([r], n, nb, f * nb), R.block_tokens(idx[h, r].tolist(), n, nb, F * nb)
                _check(O[h, at], _np(Q[h])[at], rk[h, t], rv[h, t], d ** -0.5)


def test_results_are_the_same_again_on_another_stream_and_in_a_graph(gpu):
    torch, lf = gpu
    H, d, n, f, F, T = 4, 128, 64, 1, 40, 40 * 64
    dev, _ = _cache(gpu, H, T, d, _rand(torch, 1, H, T, d), _rand(torch, 2, H, T, d))
    Q = _rand(torch, 0, H, n, d).cuda()
    idx = _lists(torch, "plain", H, 1, F, 33, 0).cuda()
    calls = (lambda **kw: lf.lf_sparse_attn_kvq(Q, dev, T, T, idx, n, 64, **kw), lambda **kw: lf.lf_token_attn_kvq(Q, dev, T, T - 3, **kw))
    for call in calls:
        want = call().clone()
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        a, b = call(stream=st), call()                 # two at once, each with a workspace of its own
        torch.cuda.synchronize()
        assert torch.equal(a, want) and torch.equal(b, want)
        O = torch.empty_like(Q)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(O=O)
        for k in range(3):
            Q.copy_(_rand(torch, 20 + k, *Q.shape).cuda())
            want = call().clone()
            O.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(O, want), k


def test_binding_refuses(gpu):
    torch, lf = gpu
    H, d, T = 2, 64, 128
    cache = torch.zeros(lf.lf_kvq_bytes(H, d, T), dtype=torch.uint8, device="cuda")
    Q = torch.zeros((H, 64, d), dtype=torch.bfloat16, device="cuda")
    idx = torch.zeros((H, 1, 2), dtype=torch.int32, device="cuda")
    bad = [lambda: lf.lf_kvq_append(Q, Q[:, :5], cache, T, 0), lambda: lf.lf_kvq_append(Q.float(), Q.float(), cache, T, 0),
           lambda: lf.lf_kvq_append(Q, Q, cache.float(), T, 0), lambda: lf.lf_kvq_append(Q, Q, cache.cpu(), T, 0),
           lambda: lf.lf_kvq_read(cache, H, d, T, 0, 5, K=Q), lambda: lf.lf_kvq_read(cache[::2], H, d, T, 0, 64, K=Q, V=Q),
           lambda: lf.lf_token_attn_kvq(Q, cache, T, T, K=Q), lambda: lf.lf_token_attn_kvq(Q, cache, T, T, K=Q, V=Q[:, :3]),
           lambda: lf.lf_token_attn_kvq(Q, cache, T, T, O=Q[:, :3]), lambda: lf.lf_token_attn_kvq(Q.transpose(1, 2), cache, T, T),
           lambda: lf.lf_sparse_attn_kvq(Q, cache, T, T, idx.long(), 64, 64), lambda: lf.lf_sparse_attn_kvq(Q, cache, T, T, idx[:1], 64, 64),
           lambda: lf.lf_sparse_attn_kvq(Q, cache, T, T, idx, 64, 64, K=Q[:, :32], V=Q[:, :32]),
           lambda: lf.lf_token_attn_kvq(Q, cache, T, T, workspace=cache[::2])]
    for k, call in enumerate(bad):
        print("refusal", k, flush=True)
        with pytest.raises(ValueError):
            call()
    for call in (lambda: lf.lf_kvq_append(Q, Q, cache, T, 65), lambda: lf.lf_kvq_append(Q, Q, cache[:-256], T, 0),
                 lambda: lf.lf_kvq_append(Q, Q, cache, T, -1), lambda: lf.lf_token_attn_kvq(Q, cache, T, T + 1),
                 lambda: lf.lf_sparse_attn_kvq(Q, cache, T, 3 * 64, idx, 64, 64), lambda: lf.lf_kvq_read(cache, H, d, T, 127, 2)):
        with pytest.raises(lf.LfError):
            call()


@pytest.mark.parametrize("H,n,f,F,length", [(2, 70, 1, 8, 6), (40, 70, 2, 6, 12)])
def test_what_no_list_keeps_may_be_anything(gpu, H, n, f, F, length):
    """NaN and infinities in the cache right behind the tokens of listed blocks, and in the blocks that no list holds, in both ways."""
    torch, lf = gpu
    d, nb, kv, q = 64, 2, F * n, f * n
    K, V = _rand(torch, 1, H, kv, d), _rand(torch, 2, H, kv, d)
    Q = _rand(torch, 3, H, q, d)
    keep = torch.tensor([c for c in range(F * nb) if c % 3 != 1])          # 0, 2, 3, 5, ...: whole blocks and short ones
    for c in range(F * nb):
        if c % 3 == 1:
            t = torch.from_numpy(R.block_tokens([c], n, nb, F * nb))
            K[:, t, 5], V[:, t, 7] = float("nan"), float("inf")
    dev, host = _cache(gpu, H, kv, d, K, V)
    g = torch.Generator().manual_seed(4)
    idx = torch.stack([keep[torch.randperm(len(keep), generator=g)[:length]] for _ in range(H * f * nb)]).to(torch.int32).view(H, f * nb, -1)
    O = _np(lf.lf_sparse_attn_kvq(Q.cuda(), dev, kv, kv, idx.cuda(), n, 64))
    rk, rv = R.cache_read(host, H, kv, d, 0, kv)
    for h in range(H):
        for r in range(f * nb):
            rows, t = R.block_tokens([r], n, nb, f * nb), R.block_tokens(idx[h, r].tolist(), n, nb, F * nb)
            _check(O[h, rows], _np(Q[h])[rows], rk[h, t], rv[h, t], d ** -0.5)


def test_a_value_that_is_not_finite_stays_in_its_heads_rows(gpu):
    """One NaN among the keys or the values: all rows of that head (its channels, for a value's) are NaN, other heads are as they were."""
    torch, lf = gpu
    H, d, T = 3, 128, 300
    K, V, Q = _rand(torch, 1, H, T, d), _rand(torch, 2, H, T, d), _rand(torch, 3, H, 4, d).cuda()
    dev, _ = _cache(gpu, H, T, d, K, V)
    want = lf.lf_token_attn_kvq(Q, dev, T, T).clone()
    K[1, 170, 3], V[2, 11, 40] = float("inf"), float("nan")
    dev, _ = _cache(gpu, H, T, d, K, V)
    got = lf.lf_token_attn_kvq(Q, dev, T, T)
    assert torch.equal(got[0], want[0]) and torch.isnan(got[1]).all() and torch.isnan(got[2, :, 32:64]).all()
    assert torch.equal(got[2, :, :32], want[2, :, :32]) and torch.equal(got[2, :, 64:], want[2, :, 64:])
