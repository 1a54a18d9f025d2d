"""The norm between two blocks and its gradients against their binary64 oracle, through the C ABI.

Bars, with u = 2^-24 (a rounding of float32) and half a step of bfloat16, 2^-8 of the value.
  Xout   gate and residual_scale once, one fma: 3 u of |gate p|; p's norm adds up squares in at most 24 additions of a thread, 6 of a wavefront and 4
         of a workgroup, halved by the root, and 6 more roundings: fewer than 32 in all, so 2^-18 of |X| + |gate p|.
  Y      from the stream as the kernel wrote it.  The mean is off by at most 36 u of the mean of |x|, a difference by that and its rounding, 1 / root by
         as many: each below 2^-18 of (|x| + |mean| + mean |x|) / root + |n|, two products and a sum behind them: 2^-17 of that times the factor.
  dX, dB sums of products of such terms: the oracle returns the sum of their sizes; another 64 roundings: 2^-16.  dB with post_weight twice: 2^-15.
  tables' gradients   sums over N tokens in any order, (N + 128) u of the sum of sizes, and the terms' own 2^-15."""
import numpy as np
import pytest

from oracle import blocks_oracle as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2602_04789_amd import lf
    lf.load()
    return torch, lf


def _ok(name, got, ref, size, unit, step):
    err, bar = np.abs(got - ref), step * np.abs(ref) + unit * size + 1e-30
    assert np.all(err <= bar), (name, float((err / bar).max()), np.unravel_index((err / bar).argmax(), err.shape))


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _inputs(torch, L, C, G, f32, seed, pad):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g)
    tall = 1.0 + 12.0 * (torch.rand((1, C), generator=g) < 0.02).float()
    dt = torch.float32 if f32 else torch.bfloat16
    wide = torch.full((L, C + pad), 7.0)
    t = dict(X=(r(L, C) * tall + 0.3).to(dt), B=r(L, C).to(torch.bfloat16), dY=r(L, C).to(torch.bfloat16), dXout=r(L, C).to(dt))
    for k, v in t.items():          # rows of a larger buffer
        w = wide.to(v.dtype).cuda()
        w[:, :C] = v.cuda()
        t[k] = w[:, :C]
    tables = (0.3 * r(G, 4, C)).cuda()
    t.update(gate=tables[:, 0], scale=tables[:, 1], shift=tables[:, 3], weight=(1.0 + 0.2 * r(C)).cuda(), post=(1.0 + 0.2 * r(C)).cuda())
    return t


def _run(gpu, L, C, starts=None, group_len=0, f32=False, layer=True, post=False, block=True, gate=True, weight=True, scale=True, shift=True, pad=0, eps=1e-6,
         rs=1.0, seed=0, dXout=True, dY=True):
    torch, lf = gpu
    print(f"gate norm L={L} C={C} starts={starts} group_len={group_len} f32={f32} layer={layer} post={post} block={block} pad={pad}", flush=True)
    G = len(starts) - 1 if starts else -(-L // group_len)
    t = _inputs(torch, L, C, G, f32, seed, pad)
    have = lambda k, on: t[k] if on else None
    gate_, post_, weight_ = have("gate", block and gate), have("post", block and post), have("weight", weight)
    scale_, shift_ = have("scale", scale), have("shift", shift)
    how = dict(B=have("B", block), gate=gate_, post_weight=post_, weight=weight_, scale=scale_, group_len=group_len, kind=lf.LF_NORM_LAYER if layer else lf.LF_NORM_RMS,
               starts=torch.tensor(starts, dtype=torch.int32, device="cuda") if starts else None, eps=eps, residual_scale=rs)
    step = 2.0 ** -24 if f32 else 2.0 ** -8
    g = R.groups_of(L, group_len, starts)
    keep = np.nonzero(g >= 0)[0]
    out = lambda: torch.full((L, C + pad), 7.0, device="cuda")
    Xo = out().to(t["X"].dtype)[:, :C] if block else None
    Yb = out().to(torch.bfloat16)
    X1, Y = lf.lf_gate_norm(t["X"], shift=shift_, Xout=Xo, Y=Yb[:, :C], **how)
    torch.cuda.synchronize()
    X, B = _np(t["X"]), _np(t["B"])
    if block:
        a = _np(gate_)
        ref = R.gate(X[keep], B[keep], g[keep], a, _np(post_), eps, rs)
        p = np.abs(R.gate(0 * X[keep], B[keep], g[keep], a, _np(post_), eps, rs))
        _ok("Xout", _np(X1)[keep], ref, np.abs(X[keep]) + p, 2.0 ** -18, step)
    xo, gk = _np(X1)[keep], g[keep]
    ref = R.norm(xo, gk, _np(weight_), _np(scale_), _np(shift_), eps, layer)
    n, mean, inv = R._norm(xo, eps, layer)
    sn = (np.abs(xo) + np.abs(mean) + np.abs(xo).mean(1, keepdims=True)) * inv + np.abs(n)
    sY = sn * np.abs(R._factor(C, G, _np(weight_), _np(scale_), gk)) + (np.abs(_np(shift_))[gk] if shift else 0.0)
    _ok("Y", _np(Y)[keep], ref, sY, 2.0 ** -17, 2.0 ** -8)
    rest = np.setdiff1d(np.arange(L), keep)
    for o in ([Xo] if block else []) + [Yb[:, :C]]:
        assert np.all(_np(o)[rest] == 7.0)
    assert (Yb[:, C:] == 7.0).all()
    # gradients
    dX, dB = (out().to(t["X"].dtype)[:, :C], out().to(torch.bfloat16)[:, :C] if block else None)
    ws = torch.full((lf.lf_gate_norm_bwd_workspace_bytes(L, C, G, group_len),), 255, dtype=torch.uint8, device="cuda")
    got = lf.lf_gate_norm_bwd(X1, t["dY"] if dY else None, dXout=t["dXout"] if dXout else None, dX=dX, dB=dB, workspace=ws, **how)
    torch.cuda.synchronize()
    zero = np.zeros((len(keep), C))
    ref, size = R.gate_norm_backward(xo, B[keep] if block else None, gk, G, _np(gate_), _np(post_), _np(weight_), _np(scale_), eps, rs, layer,
                                     _np(t["dY"])[keep] if dY else zero, _np(t["dXout"])[keep] if dXout else zero)
    names = ("dX", "dB", "dgate", "dpost_weight", "dweight", "dscale", "dshift")
    assert [k for k, v in zip(names, got) if v is None] == [k for k, on in (("dB", block), ("dgate", gate_ is not None), ("dpost_weight", post_ is not None),
                                                                            ("dweight", weight)) if not on]
    most = max(np.bincount(gk, minlength=1)) if len(gk) else 0
    for k, v in zip(names, got):
        if v is None:
            continue
        v = _np(v)
        if k in ("dX", "dB"):
            assert np.all(v[rest] == 7.0)
            _ok(k, v[keep], ref[k], size[k], 2.0 ** -16 if k == "dX" or not post else 2.0 ** -15, step if k == "dX" else 2.0 ** -8)
        else:
            N = len(gk) + G if k in ("dweight", "dpost_weight") else most
            _ok(k, v, ref[k], size[k], 2.0 ** -15 + (N + 128) * 2.0 ** -24, 2.0 ** -24)
    return X1, Y, got


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("post", [False, True])
def test_forward_and_gradients(gpu, f32, layer, post):
    for L, C, kw in ((1, 8, dict(group_len=1)), (1, 1536, dict(group_len=5)), (37, 320, dict(group_len=10)), (13, 64, dict(starts=[0, 4, 13])),
                     (70, 1536, dict(starts=[0, 0, 33, 64, 64, 70]))):
        _run(gpu, L, C, f32=f32, layer=layer, post=post, seed=L + C, pad=16, **kw)


@pytest.mark.parametrize("C", [8, 72, 512, 520, 1000, 1024, 1536, 1544, 2048, 2056, 4096, 5120, 6144, 6152, 8192, 8200, 16384])
@pytest.mark.parametrize("f32", [False, True])
def test_widths(gpu, C, f32):
    """Both sides of every line between layouts: chunks of a thread, wavefronts of a row, forms of the backward kernel."""
    _run(gpu, 19, C, group_len=7, f32=f32, post=C % 3 == 0, seed=C)
    _run(gpu, 6, C, starts=[0, 2, 6], f32=f32, layer=False, seed=C)


@pytest.mark.parametrize("starts", [[2, 5, 9], [0, 0, 0, 12], [3, 3], [0, 12, 12], [11, 12], [12, 12], [0, 0], [1, 2, 3, 4, 5, 6, 7, 8, 9]])
def test_tokens_of_no_group_and_empty_groups(gpu, starts):
    _run(gpu, 12, 264, starts=starts, seed=3, pad=8)


@pytest.mark.parametrize("G", [1, 63, 64, 65, 400])
def test_many_groups(gpu, G):
    rng = np.random.default_rng(G)
    starts = np.sort(rng.integers(0, 501, G + 1))
    _run(gpu, 500, 72, starts=[int(x) for x in starts], layer=False, seed=G)
    _run(gpu, 500, 72, group_len=-(-500 // G), seed=G)


def test_many_tokens(gpu):
    """Slots of many rows, groups of many slots."""
    _run(gpu, 5003, 72, group_len=5003, seed=1)
    _run(gpu, 9001, 16, starts=[5, 9000], f32=True, post=True, seed=2)
    _run(gpu, 3001, 1600, group_len=1500, seed=3)


@pytest.mark.parametrize("off", ["block", "gate", "weight", "scale", "shift", "dXout", "dY"])
def test_what_may_be_left_out(gpu, off):
    for layer in (True, False):
        _run(gpu, 21, 328, group_len=8, layer=layer, post=off in ("gate", "shift"), seed=4, **{off: False})


@pytest.mark.parametrize("off", ["gate", "weight", "scale", "block"])
@pytest.mark.parametrize("kw", [dict(group_len=23), dict(starts=[0, 23]), dict(starts=[4, 4])])
def test_one_group(gpu, off, kw):
    """Its sums are those of the weights too."""
    _run(gpu, 23, 200, post=off != "block", seed=5, **{off: False}, **kw)


@pytest.mark.parametrize("C", [72, 1536, 2048, 8200])
@pytest.mark.parametrize("starts", [[2, 9, 30], [3, 3, 31]])
def test_nan_beside_the_groups_stays_there(gpu, C, starts):
    torch, lf = gpu
    L, G = 37, len(starts) - 1
    t = _inputs(torch, L, C, G, False, 6, 0)
    st = torch.tensor(starts, dtype=torch.int32, device="cuda")
    how = dict(B=t["B"], gate=t["gate"], post_weight=t["post"], weight=t["weight"], scale=t["scale"], starts=st)
    results = []
    for beside in (0.0, float("nan")):
        for k in ("X", "B", "dY", "dXout"):
            t[k][:starts[0]] = beside
            t[k][starts[-1]:] = beside
        X1, Y = lf.lf_gate_norm(t["X"], shift=t["shift"], Xout=torch.full_like(t["X"], beside), **how)
        dX, dB, *tables = lf.lf_gate_norm_bwd(X1, t["dY"], dXout=t["dXout"], **how)
        results.append([x[starts[0]:starts[-1]] for x in (X1, Y, dX, dB)] + tables)
    for a, b in zip(*results):
        assert torch.equal(a, b) and not torch.isnan(a).any()


def test_nothing_but_the_norm(gpu):
    _run(gpu, 9, 128, group_len=9, block=False, weight=False, scale=False, shift=False)


def test_residual_scale_and_eps(gpu):
    _run(gpu, 10, 192, group_len=4, rs=-0.25, post=True, eps=0.5)
    _run(gpu, 10, 192, group_len=4, rs=0.0)


def test_a_large_mean(gpu):
    """A row whose mean is a thousand times its deviation: the variance is taken of the differences."""
    torch, lf = gpu
    X = (1000.0 + torch.randn((5, 640), generator=torch.Generator().manual_seed(0))).cuda()
    _, Y = lf.lf_gate_norm(X, group_len=5)
    x = X.double()
    want = (x - x.mean(1, keepdim=True)) / (x.var(1, unbiased=False, keepdim=True) + 1e-6).sqrt()
    # the mean's rounding, 36 u of 1000, and a difference's: 2^-18 of 2000
    assert ((Y.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2000 * 2.0 ** -18).all()


def test_in_place(gpu):
    """Xout may be X, and dX may be dXout."""
    torch, lf = gpu
    t = _inputs(torch, 300, 1536, 3, False, 5, 0)
    how = dict(B=t["B"], gate=t["gate"], scale=t["scale"], group_len=100)
    X1, Y1 = lf.lf_gate_norm(t["X"], shift=t["shift"], **how)
    X2 = t["X"].clone()
    got = lf.lf_gate_norm(X2, shift=t["shift"], Xout=X2, **how)
    assert got[0] is X2 and torch.equal(X1, X2) and torch.equal(Y1, got[1])
    a = lf.lf_gate_norm_bwd(X1, t["dY"], dXout=t["dXout"], **how)
    d = t["dXout"].clone()
    b = lf.lf_gate_norm_bwd(X1, t["dY"], dXout=d, dX=d, **how)
    assert b[0] is d and all(x is None if y is None else torch.equal(x, y) for x, y in zip(a, b))


def test_gradient_against_differences(gpu):
    """The derivative of <Y, dY> + <Xout, dXout> along a direction of a float32 stream, from two forward calls a step of 2 h apart: bfloat16 leaves 2^-8 of
    every Y, independent (standard deviation 1 / sqrt 3 of it), and the third derivative h^2 / 6 of about the sum's size."""
    torch, lf = gpu
    t = _inputs(torch, 24, 256, 3, True, 6, 0)
    how = dict(B=t["B"], gate=t["gate"], post_weight=t["post"], weight=t["weight"], scale=t["scale"], group_len=8)
    h = 1.0 / 16
    dirn = torch.randn(t["X"].shape, generator=torch.Generator().manual_seed(2)).cuda()

    def f(x):
        Xo, Y = lf.lf_gate_norm(x, shift=t["shift"], **how)
        return Y.double() * t["dY"].double(), Xo.double() * t["dXout"].double()
    (ya, xa), (yb, xb) = f(t["X"] + h * dirn), f(t["X"] - h * dirn)
    diff = float(((ya - yb).sum() + (xa - xb).sum()) / (2 * h))
    Xo, _ = lf.lf_gate_norm(t["X"], shift=t["shift"], **how)
    dX = lf.lf_gate_norm_bwd(Xo, t["dY"], dXout=t["dXout"], **how)[0].double()
    exact = float((dX * dirn).sum())
    noise = 5 / (2 * h) * 2.0 ** -8 / 3 ** 0.5 * float((ya.square() + yb.square()).sum().sqrt())
    curve = h * h * float((dX * dirn).abs().sum())
    print("difference", diff, "gradient", exact, "bars", noise, curve)
    assert abs(diff - exact) <= noise + curve


def test_results_are_the_same_again_and_on_another_stream(gpu):
    torch, lf = gpu
    t = _inputs(torch, 777, 1536, 3, False, 7, 0)
    how = dict(B=t["B"], gate=t["gate"], post_weight=t["post"], scale=t["scale"], group_len=259)
    X1, Y1 = lf.lf_gate_norm(t["X"], shift=t["shift"], **how)
    a = lf.lf_gate_norm_bwd(X1, t["dY"], dXout=t["dXout"], **how)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    X2, Y2 = lf.lf_gate_norm(t["X"], shift=t["shift"], stream=st, **how)
    b = lf.lf_gate_norm_bwd(X2, t["dY"], dXout=t["dXout"], stream=st, **how)
    st.synchronize()
    assert torch.equal(X1, X2) and torch.equal(Y1, Y2) and all(x is None if y is None else torch.equal(x, y) for x, y in zip(a, b))


def test_a_captured_step_replays(gpu):
    torch, lf = gpu
    t = _inputs(torch, 300, 320, 4, True, 8, 0)
    starts = torch.tensor([0, 90, 100, 250, 300], dtype=torch.int32, device="cuda")
    how = dict(B=t["B"], gate=t["gate"], weight=t["weight"], scale=t["scale"], starts=starts)
    Xo, Y, dX, dB = torch.empty_like(t["X"]), torch.empty_like(t["B"]), torch.empty_like(t["X"]), torch.empty_like(t["B"])
    ws = torch.empty(lf.lf_gate_norm_bwd_workspace_bytes(300, 320, 4), dtype=torch.uint8, device="cuda")
    kept = []

    def step():
        lf.lf_gate_norm(t["X"], shift=t["shift"], Xout=Xo, Y=Y, **how)
        kept[:] = lf.lf_gate_norm_bwd(Xo, t["dY"], dXout=t["dXout"], dX=dX, dB=dB, workspace=ws, **how)
        return [Xo, Y] + [x for x in kept if x is not None]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for k in range(3):
        t["X"].copy_(torch.randn(t["X"].shape, device="cuda"))
        starts.copy_(torch.tensor([0, 10 + k, 100, 200, 290], dtype=torch.int32))
        want = [x.clone() for x in step()]
        for x in outs:
            x.zero_()
        Xo.copy_(want[0]); Y.copy_(want[1])     # (rows of no group are left alone)
        dX.copy_(want[2]); dB.copy_(want[3])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs)), k


def test_binding_refuses(gpu):
    torch, lf = gpu
    t = _inputs(torch, 8, 64, 2, False, 0, 0)
    ok = dict(X=t["X"], B=t["B"], gate=t["gate"], post_weight=t["post"], weight=t["weight"], scale=t["scale"], shift=t["shift"], group_len=4)
    lf.lf_gate_norm(**ok)
    starts = torch.tensor([0, 8, 8], dtype=torch.int32, device="cuda")
    for bad in (dict(X=t["X"].half()), dict(X=t["X"].cpu()), dict(X=t["X"][0]), dict(X=t["X"].T.contiguous().T), dict(B=t["B"].float()), dict(B=t["B"][:7]), dict(B=None),
                dict(gate=t["gate"][:1]), dict(scale=t["scale"].half()), dict(shift=t["shift"][:, :32]), dict(weight=t["weight"][:8]), dict(weight=t["weight"].double()),
                dict(group_len=0), dict(group_len=-4), dict(starts=starts), dict(group_len=0, starts=starts.long()), dict(group_len=0, starts=starts[:1]),
                dict(Y=t["X"].float()), dict(Xout=t["X"][:4]), dict(group_len=1 << 40)):
        with pytest.raises(ValueError):
            lf.lf_gate_norm(**{**ok, **bad})
    for bad in (dict(eps=-1.0), dict(eps=float("nan")), dict(kind=2), dict(residual_scale=float("inf"))):
        with pytest.raises(lf.LfError):
            lf.lf_gate_norm(**{**ok, **bad})
    with pytest.raises(lf.LfError):
        lf.lf_gate_norm(torch.zeros((4, 60), device="cuda"), group_len=4)
    how = dict(B=t["B"], gate=t["gate"], scale=t["scale"], group_len=4)
    for bad in (dict(dXout=t["dXout"].float()), dict(dX=t["X"][:4]), dict(dB=t["B"].float()), dict(B=None), dict(workspace=torch.empty(256, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            lf.lf_gate_norm_bwd(t["X"], t["dY"], **{**how, **bad})
    with pytest.raises(lf.LfError):
        lf.lf_gate_norm_bwd(t["X"], t["dY"], workspace=torch.empty(256, dtype=torch.uint8, device="cuda"), **how)
