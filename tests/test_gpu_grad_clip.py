"""Clipping to a largest norm against its binary64 oracle.  The norm is a sum of exact squares in binary64, rounded once to float32 (2^-24); the factor is
rounded once (2^-24, and 2^-50 of the norm's), an output's product (2^-24) and its own type once: 2^-22 of the value beside half a step."""
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


def _tensors(torch, sizes, kinds, seed=0, scale=0.05):
    """Tensors that begin at odd places of one buffer, 7.0 around them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out, flat = [], []
    for i, n in enumerate(sizes):
        dt = torch.bfloat16 if kinds[i % len(kinds)] == "b" else torch.float32
        buf = torch.full((n + 9,), 7.0, dtype=dt, device="cuda")
        x = buf[1 + i % 5:1 + i % 5 + n]
        x.copy_(torch.randn(n, generator=g, device="cuda") * scale)
        out.append(x)
        flat.append(buf)
    return out, flat


def _check(torch, got, x, f):
    ref = x.double().cpu().numpy() * f
    step = 2.0 ** -8 if got.dtype is torch.bfloat16 else 2.0 ** -24
    err = np.abs(got.double().cpu().numpy() - ref)
    assert np.all(err <= (step + 2.0 ** -22) * np.abs(ref) + 1e-38)


CASES = [[1], [7], [8], [9], [1, 1, 1], [4095, 4096, 4097], [0, 5, 0], [65536 * 3 + 5], [3, 100000, 17, 2048, 8, 1], list(range(1, 260)), [1 << 21, 3, 1 << 20]]


@pytest.mark.parametrize("sizes", CASES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("kinds", ["b", "f", "bf"])
def test_in_place_and_apart(gpu, sizes, kinds):
    torch, lf = gpu
    for max_norm in (0.01, 1e9):
        xs, flat = _tensors(torch, sizes, kinds)
        n, f = R.clip([x.double().cpu().numpy() for x in xs], max_norm, 1e-6)
        for out_kind in (None, "b", "f"):
            keep = [x.clone() for x in xs]
            out, oflat = (None, None) if out_kind is None else _tensors(torch, sizes, out_kind, seed=9)
            norm = lf.lf_grad_clip(xs, max_norm, out=out)
            torch.cuda.synchronize()
            assert norm.shape == (1,) and abs(float(norm) - n) <= 2.0 ** -23 * n
            for x, y, k in zip(xs, xs if out is None else out, keep):
                _check(torch, y, k, f)
                if out is not None or f == 1.0:
                    assert torch.equal(x, k)
            for bufs in (flat, oflat):
                for i, (b, s) in enumerate(zip(bufs or [], sizes)):
                    assert (b[:1 + i % 5] == 7.0).all() and (b[1 + i % 5 + s:] == 7.0).all()
            for x, k in zip(xs, keep):
                x.copy_(k)


def test_many_tensors_and_shares(gpu):
    """More tensors than a launch describes, and more shares than a workgroup adds by itself."""
    torch, lf = gpu
    sizes = [5000 + 13 * i for i in range(500)]
    xs, _ = _tensors(torch, sizes, "bf", seed=3)
    keep = [x.clone() for x in xs]
    n, f = R.clip([x.double().cpu().numpy() for x in xs], 0.5, 1e-6)
    norm = lf.lf_grad_clip(xs, 0.5)
    assert f < 1 and abs(float(norm) - n) <= 2.0 ** -23 * n
    for x, k in zip(xs, keep):
        _check(torch, x, k, f)


@pytest.mark.parametrize("count", [1024, 1025, 2000])
def test_more_shares_than_a_workgroup_adds(gpu, count):
    torch, lf = gpu
    sizes = [1 + i % 7 for i in range(count)]
    xs, _ = _tensors(torch, sizes, "bf", seed=4)
    keep = [x.clone() for x in xs]
    n, f = R.clip([x.double().cpu().numpy() for x in xs], 0.5, 1e-6)
    norm = lf.lf_grad_clip(xs, 0.5)
    assert f < 1 and abs(float(norm) - n) <= 2.0 ** -23 * n
    for x, k in zip(xs, keep):
        _check(torch, x, k, f)


def test_norm_alone(gpu):
    torch, lf = gpu
    xs, _ = _tensors(torch, [1000, 0, 77], "bf")
    keep = [x.clone() for x in xs]
    norm = torch.full((1,), -1.0, device="cuda")
    assert lf.lf_grad_clip(xs, float("inf"), norm=norm) is norm
    n, _ = R.clip([x.double().cpu().numpy() for x in xs], 1.0, 0.0)
    assert abs(float(norm) - n) <= 2.0 ** -23 * n and all(torch.equal(a, b) for a, b in zip(xs, keep))
    out, _ = _tensors(torch, [1000, 0, 77], "f")
    lf.lf_grad_clip(xs, float("inf"), out=out)
    assert all(torch.equal(a.float(), b) for a, b in zip(xs, out))
    assert float(lf.lf_grad_clip([], 1.0)) == 0.0 and float(lf.lf_grad_clip([xs[1]], 1.0)) == 0.0


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("many", [False, True])
def test_not_finite(gpu, bad, many):
    """The norm says so, and nothing is scaled: in place all stays, apart it is copied."""
    torch, lf = gpu
    xs, _ = _tensors(torch, [5000] * (1500 if many else 3), "f")
    xs[1][77] = bad
    keep = [x.clone() for x in xs]
    norm = float(lf.lf_grad_clip(xs, 0.1))
    assert not np.isfinite(norm) and (np.isnan(norm) == np.isnan(bad))
    out = [torch.zeros_like(x) for x in xs]
    lf.lf_grad_clip(xs, 0.1, out=out)
    for x, k, o in zip(xs, keep, out):
        assert torch.equal(x.view(torch.int32), k.view(torch.int32)) and torch.equal(o.nan_to_num(1.0, 2.0, 3.0), k.nan_to_num(1.0, 2.0, 3.0))


def test_squares_that_float32_cannot_hold(gpu):
    torch, lf = gpu
    x = torch.tensor([3e30, -4e30, 1e-30], device="cuda")
    norm = lf.lf_grad_clip([x], 1.0, eps=0.0)
    assert abs(float(norm) - 5e30) <= 1e24
    assert torch.allclose(x, torch.tensor([0.6, -0.8, 2e-61], device="cuda"), rtol=1e-6, atol=0)
    y = torch.full((4,), 3.0e38, device="cuda")                 # the norm is above float32: infinity is told, the factor is right
    norm = lf.lf_grad_clip([y], 2.0)
    assert float(norm) == float("inf") and torch.allclose(y, torch.ones(4, device="cuda"), rtol=1e-6)
    z = torch.full((1000,), 1e-30, device="cuda")
    assert abs(float(lf.lf_grad_clip([z], 1.0)) - 1000 ** 0.5 * 1e-30) <= 1e-36


def test_dense_tensors_in_any_order(gpu):
    torch, lf = gpu
    x = torch.randn((6, 5, 4), device="cuda").permute(2, 0, 1)
    keep = x.clone()
    lf.lf_grad_clip([x], 0.5)
    assert torch.allclose(x, keep * (0.5 / (keep.double().norm() + 1e-6)).float(), rtol=1e-6)
    for bad in (torch.randn((4, 6), device="cuda")[:, :3], torch.randn((3, 1), device="cuda").expand(3, 4)):
        with pytest.raises(ValueError):
            lf.lf_grad_clip([bad], 0.5)


def test_results_are_the_same_again_captured_and_on_another_stream(gpu):
    torch, lf = gpu
    xs, _ = _tensors(torch, [100000 + 3 * i for i in range(150)], "bf")
    out = [torch.empty_like(x) for x in xs]
    ws = torch.empty(lf.lf_grad_workspace_bytes(150, sum(x.numel() for x in xs)), dtype=torch.uint8, device="cuda")
    norm = lf.lf_grad_clip(xs, 0.3, out=out, workspace=ws).clone()
    want = [o.clone() for o in out]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    n2 = lf.lf_grad_clip(xs, 0.3, out=out, workspace=ws, stream=st)
    st.synchronize()
    assert torch.equal(norm, n2) and all(torch.equal(a, b) for a, b in zip(want, out))
    graph, nb = torch.cuda.CUDAGraph(), torch.empty(1, device="cuda")
    with torch.cuda.graph(graph):
        lf.lf_grad_clip(xs, 0.3, out=out, workspace=ws, norm=nb)
    for k in range(3):
        for x in xs:
            x.mul_(1.5)
        n3 = lf.lf_grad_clip(xs, 0.3, out=out, workspace=ws).clone()
        want = [o.clone() for o in out]
        for o in out:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(n3, nb) and all(torch.equal(a, b) for a, b in zip(want, out)), k


def test_binding_refuses(gpu):
    torch, lf = gpu
    x = torch.randn(10, device="cuda")
    for bad in (dict(grads=[x.half()]), dict(grads=[x.cpu()]), dict(out=[]), dict(out=[x[:5].clone()]), dict(out=[x.double()]), dict(norm=torch.zeros(2, device="cuda")),
                dict(norm=torch.zeros(1)), dict(out=[torch.randn((5, 4), device="cuda")[:, :2]])):
        with pytest.raises(ValueError):
            lf.lf_grad_clip(**{**dict(grads=[x], max_norm=1.0), **bad})
    with pytest.raises(lf.LfError):        # scaled twice
        lf.lf_grad_clip([x, x], 1.0)
    assert float(lf.lf_grad_clip([x, x], float("inf"))) > 0.0
    for bad in (dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(eps=-1.0), dict(eps=float("inf")), dict(workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(lf.LfError):
            lf.lf_grad_clip(**{**dict(grads=[x], max_norm=1.0), **bad})
