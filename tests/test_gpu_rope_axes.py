"""RMSNorm with rotary positions over three axes and its gradients against their binary64 oracle, through the C ABI.

Bars.  The kernels compute in float32 and round once to bfloat16: half a step of it, 2^-8 of the value, and what float32 adds up to.
  Y   a term of the rotated pair is |a| + |b| large; it goes through the sum of squares (at most 64 additions in a row per lane and
      through the lanes, halved by the root), the division, two products, the angle's cosine and sine (4 units) and two sums:
      fewer than 64 roundings of 2^-24 each, so 2^-18 (|a| + |b|).
  dX  two such sums and their products, fewer than 128 roundings of the terms' sizes: 2^-17.
  dg  every term is that exact to 64 roundings, and the tokens of a lane are added one after the other (at most tokens / 512 + 1 of them),
      then those of a workgroup (64 at the most) and 8 rows and 6 halvings of the last launch: (160 + tokens / 512) 2^-24."""
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


def _axes(d):
    side = 2 * (d // 6) // 2
    return (d // 2 - 2 * side, side, side)


def _inputs(torch, L, H, d, seed, far, pad=0):
    g = torch.Generator().manual_seed(seed)
    X = torch.randn((L, H * d + pad), generator=g).to(torch.bfloat16)
    w = 1.0 + 0.1 * torch.randn(H * d, generator=g)
    pos = torch.randint(-far, far + 1, (L, 3), generator=g, dtype=torch.int32)
    freq = torch.cat([10000.0 ** (-torch.arange(n, dtype=torch.float64) / max(n, 1)) for n in _axes(d)])
    dY = torch.randn((H, L, d), generator=g).to(torch.bfloat16)
    return X, w, pos, freq, dY


def _rel_ok(got, ref, size, unit):
    err = np.abs(got - ref)
    bar = 2.0 ** -8 * np.abs(ref) + unit * size + 1e-37
    assert np.all(err <= bar), (float((err / bar).max()), np.unravel_index((err / bar).argmax(), err.shape))


def _run(gpu, L, H, d, across, pairing, seed=0, far=40, pad=0, eps=1e-6, axes=None):
    torch, lf = gpu
    print(f"rope axes L={L} H={H} d={d} across={across} pairing={pairing} far={far} pad={pad}", flush=True)
    X, w, pos, freq, dY = _inputs(torch, L, H, d, seed, far, pad)
    axes = axes or _axes(d)
    Xg, wg, pg, fg = X.cuda(), w.cuda(), pos.cuda(), freq.cuda()
    # Y and dY are the last tokens of larger buffers
    buf = torch.full((H, L + 3, d + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    Y = buf[:, 3:, :d]
    dYg = torch.full_like(buf, float("nan"))
    dYg[:, 3:, :d] = dY.cuda()
    how = dict(eps=eps, across_heads=across, pairing=pairing)
    lf.lf_qk_norm_rope_axes(Xg, wg, pg, fg, axes, H, Y, **how)
    dX = torch.full_like(Xg, 7.0)
    dg = torch.full((H * d,), float("nan"), device="cuda")
    ws = torch.full((lf.lf_qk_norm_rope_axes_bwd_workspace_bytes(H, d, L),), 255, dtype=torch.uint8, device="cuda")
    lf.lf_qk_norm_rope_axes_bwd(Xg, wg, pg, fg, axes, H, dYg[:, 3:, :d], workspace=ws, grads=(dX, dg), **how)
    torch.cuda.synchronize()
    x = X.double().numpy()[:, :H * d]
    theta = R.angles(pos.numpy(), freq.numpy(), axes)
    ref = R.rope_axes(x, w.numpy(), theta, H, eps, across, pairing)
    n, _ = R._norm(x, H, eps, across)
    y = np.abs(n * w.double().numpy().reshape(H, d))
    a, b = R._split(y, pairing)
    size = R._join(a + b, a + b, pairing).transpose(1, 0, 2)
    _rel_ok(Y.double().cpu().numpy(), ref, size, 2.0 ** -18)
    assert torch.isnan(buf[:, :3].float()).all() and torch.isnan(buf[:, :, d:].float()).all()
    rX, rg, sX, sg = R.rope_axes_backward(x, w.numpy(), theta, H, eps, across, pairing, dY.double().numpy())
    _rel_ok(dX[:, :H * d].double().cpu().numpy(), rX, sX, 2.0 ** -17)
    assert (dX[:, H * d:] == 7.0).all()
    err = np.abs(dg.double().cpu().numpy() - rg)
    assert np.all(err <= (160 + L / 512) * 2.0 ** -24 * sg + 1e-37), float((err / sg).max())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("across", [False, True])
@pytest.mark.parametrize("pairing", [0, 1])
def test_forward_and_gradients(gpu, d, across, pairing):
    for L, H, pad in ((1, 1, 0), (1, 12, 0), (37, 3, 8), (130, 5, 0), (65, 2, 24)):
        _run(gpu, L, H, d, across, pairing, seed=L + H, pad=pad)


@pytest.mark.parametrize("H,d", [(4, 128), (7, 128), (9, 64), (40, 128), (33, 64), (65, 128), (128, 128), (129, 64), (256, 64)])
@pytest.mark.parametrize("across", [False, True])
def test_numbers_of_heads(gpu, H, d, across):
    """One to four heads of a thread, workgroups of one and of several tokens, up to the most channels of a token."""
    _run(gpu, 11, H, d, across, across, seed=H)


@pytest.mark.parametrize("L", [511, 4680])
def test_many_tokens(gpu, L):
    _run(gpu, L, 2, 64, True, 0, seed=L)
    _run(gpu, L, 3, 128, False, 1, seed=L + 1)


@pytest.mark.parametrize("far", [1 << 20, (1 << 31) - 1])
@pytest.mark.parametrize("pairing", [0, 1])
def test_far_positions_keep_their_phase(gpu, far, pairing):
    """Angles of up to 2^31 radians: the oracle's and the kernel's float64 products are each off by at most 2^31 2^-52 = 2^-21, the float32 bars'
    2^-18."""
    _run(gpu, 40, 2, 128, False, pairing, seed=5, far=far)


def test_one_axis_and_an_empty_one(gpu):
    _run(gpu, 20, 2, 64, False, 0, axes=(32, 0, 0))
    _run(gpu, 20, 2, 64, True, 1, axes=(0, 5, 27))


def test_rows_of_zeros_and_large_eps(gpu):
    """A token of zeros: the norm divides by the root of eps, the gradients are finite."""
    torch, lf = gpu
    X = torch.zeros((3, 128), dtype=torch.bfloat16, device="cuda")
    X[1] = 1.0
    w, pos, freq = torch.ones(128, device="cuda"), torch.zeros((3, 3), dtype=torch.int32, device="cuda"), torch.ones(32, dtype=torch.float64, device="cuda")
    Y = torch.empty((2, 3, 64), dtype=torch.bfloat16, device="cuda")
    lf.lf_qk_norm_rope_axes(X, w, pos, freq, (32, 0, 0), 2, Y)
    dX, dg = lf.lf_qk_norm_rope_axes_bwd(X, w, pos, freq, (32, 0, 0), 2, torch.ones_like(Y))
    assert (Y[:, 0] == 0).all() and (Y[:, 1] == 1).all()
    assert (dX[0] == 1000).all() and (dX[1].abs() <= 2.0 ** -16).all()
    # dg is token 1's 1 / sqrt(1 + eps) = 1 - 5e-7, which is not 1 in float32; four roundings of 2^-24
    assert ((dg.double() - (1.0 + 1e-6) ** -0.5).abs() <= 2.0 ** -22).all()
    _run(gpu, 9, 2, 64, True, 0, eps=3.0)


def test_gradient_against_differences(gpu):
    """The derivative of <Y, dY> along a direction, from two forward calls: bfloat16 inputs allow a step of 1/16 (values of one binade keep
    it exactly), the outputs' rounding leaves 2^-9 of the sizes, and the third derivative h^2 / 6 of about the sum's size."""
    torch, lf = gpu
    L, H, d = 16, 2, 64
    X, w, pos, freq, dY = (t.cuda() for t in _inputs(torch, L, H, d, 3, 20))
    X = (X.float().sign() * (1.0 + X.float().abs().clamp(max=3).mul(8).round() / 32)).to(torch.bfloat16)     # 1 .. 1.75, steps of 1/32
    dirn = torch.randint(-1, 2, X.shape, generator=torch.Generator().manual_seed(1)).cuda().float()
    up, down = (X.float() + dirn / 16).to(torch.bfloat16), (X.float() - dirn / 16).to(torch.bfloat16)
    assert torch.equal(up.float() - down.float(), dirn / 8)
    f = lambda x: (lf.lf_qk_norm_rope_axes(x, w, pos, freq, _axes(d), H, torch.empty_like(dY)).double() * dY.double())
    a, b = f(up), f(down)
    diff = float((a - b).sum()) * 8
    dX, dg = lf.lf_qk_norm_rope_axes_bwd(X, w, pos, freq, _axes(d), H, dY)
    exact = float((dX.double() * dirn.double()).sum())
    # rounding of Y: independent, half a step each (standard deviation 2^-8 / sqrt(3) of a value at the most), five of them; dX's likewise
    noise = 5 * 8 * 2.0 ** -8 / 3 ** 0.5 * float((a.square() + b.square()).sum().sqrt()) + 5 * 2.0 ** -8 * float((dX.double() * dirn).norm())
    curve = float((dX.double() * dirn).abs().sum()) / 16 ** 2
    print("difference", diff, "gradient", exact, "bars", noise, curve)
    assert abs(diff - exact) <= noise + curve


def test_results_are_the_same_again_and_on_another_stream(gpu):
    torch, lf = gpu
    L, H, d = 700, 12, 128
    X, w, pos, freq, dY = (t.cuda() for t in _inputs(torch, L, H, d, 3, 20))
    args = (X, w, pos, freq, _axes(d), H)
    Y = lf.lf_qk_norm_rope_axes(*args, torch.empty_like(dY), across_heads=True)
    dX, dg = lf.lf_qk_norm_rope_axes_bwd(*args, dY, across_heads=True)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    Y2 = lf.lf_qk_norm_rope_axes(*args, torch.empty_like(dY), across_heads=True, stream=st)
    dX2, dg2 = lf.lf_qk_norm_rope_axes_bwd(*args, dY, across_heads=True, stream=st)
    st.synchronize()
    assert torch.equal(Y, Y2) and torch.equal(dX, dX2) and torch.equal(dg, dg2)


def test_a_captured_step_replays(gpu):
    torch, lf = gpu
    L, H, d = 300, 3, 64
    X, w, pos, freq, dY = (t.cuda() for t in _inputs(torch, L, H, d, 8, 20))
    args = (X, w, pos, freq, _axes(d), H)
    Y, dX, dg = torch.empty_like(dY), torch.empty_like(X), torch.empty_like(w)
    ws = torch.empty(lf.lf_qk_norm_rope_axes_bwd_workspace_bytes(H, d, L), dtype=torch.uint8, device="cuda")

    def step():
        lf.lf_qk_norm_rope_axes(*args, Y)
        lf.lf_qk_norm_rope_axes_bwd(*args, dY, workspace=ws, grads=(dX, dg))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        X.copy_(torch.randn(X.shape, device="cuda").to(torch.bfloat16))
        step()
        want = [t.clone() for t in (Y, dX, dg)]
        for t in (Y, dX, dg):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (Y, dX, dg))), k


def test_binding_refuses(gpu):
    torch, lf = gpu
    X, w, pos, freq, dY = (t.cuda() for t in _inputs(torch, 8, 2, 64, 0, 9))
    Y, axes = torch.empty_like(dY), _axes(64)
    for bad in (dict(g=w.double()), dict(pos=pos.long()), dict(freq=freq.float()), dict(pos=pos[:7]), dict(freq=freq[:16]), dict(g=w[:64]),
                dict(pos=pos.T.contiguous().T), dict(X=X.float()), dict(X=X[:, :64]), dict(axes=(16, 16)), dict(Y=Y[:1]), dict(Y=Y.float()), dict(X=X.cpu())):
        a = dict(X=X, g=w, pos=pos, freq=freq, axes=axes, Y=Y)
        a.update(bad)
        for call in (lf.lf_qk_norm_rope_axes, lf.lf_qk_norm_rope_axes_bwd):
            with pytest.raises(ValueError):
                call(a["X"], a["g"], a["pos"], a["freq"], a["axes"], 2, a["Y"])
    with pytest.raises(lf.LfError):
        lf.lf_qk_norm_rope_axes(X, w, pos, freq, (16, 16, 1), 2, Y)
    with pytest.raises(lf.LfError):
        lf.lf_qk_norm_rope_axes_bwd(X, w, pos, freq, axes, 2, dY, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        lf.lf_qk_norm_rope_axes_bwd(X, w, pos, freq, axes, 2, dY, grads=(X[:, :64], w))
