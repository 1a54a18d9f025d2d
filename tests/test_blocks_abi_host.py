"""Argument checks and sizes of the calls around the attention: every refusal is reported before anything is enqueued (no GPU)."""
import ctypes as C
import os
import re

import pytest

from paper_2602_04789_amd import lf

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000  # a non-NULL, 256-byte aligned address that is never dereferenced on error paths


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(lf.library_path()):
        from paper_2602_04789_amd import build
        build.build()
    return lf.load()


def test_symbols_and_struct_sizes(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "lf.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(lf_[a-z_]+)\s*\(", text))
    assert {"lf_gate_norm", "lf_gate_norm_bwd", "lf_gate_norm_bwd_workspace_bytes", "lf_packed_attn", "lf_packed_attn_workspace_bytes", "lf_packed_attn_bwd",
            "lf_packed_attn_bwd_workspace_bytes", "lf_grad_clip", "lf_grad_workspace_bytes"} <= names
    assert C.sizeof(lf.lf_norm_shape) == 32 + 7 * 8 and C.sizeof(lf.lf_packed_shape) == 32 + 8 * 8 and C.sizeof(lf.lf_grad_tensor) == 32


def _norm(**kw):
    p = lf.lf_norm_shape(4680, 1536, 3, 1560, 0, 0, 1e-6, 1.0, *[1536] * 4, *[6 * 1536] * 3)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


BAD_NORM = [(dict(tokens=0), -2), (dict(tokens=(1 << 30) + 1), -2), (dict(channels=4), -2), (dict(channels=1540), -2), (dict(channels=16392), -2), (dict(groups=0), -2),
            (dict(groups=2), -2), (dict(group_len=-1), -2), (dict(groups=(1 << 24) + 1), -2), (dict(kind=2), -2), (dict(eps=-1e-9), -2), (dict(eps=float("inf")), -2),
            (dict(residual_scale=float("nan")), -2), (dict(stream_dtype=2), -4), (dict(xo_stride=1528), -2), (dict(b_stride=1535), -2),
            (dict(y_stride=1540), -5), (dict(scale_stride=1000), -2), (dict(gate_stride=1538), -5), (dict(xo_stride=(1 << 40) + 8), -2)]


def test_gate_norm_refuses_bad_arguments(lib):
    def call(X=FAKE, B=FAKE, gate=FAKE, post=FAKE, w=FAKE, sc=FAKE, sh=FAKE, st=None, p=None, Xo=FAKE, Y=FAKE):
        return lib.lf_gate_norm(X, B, gate, post, w, sc, sh, st, C.byref(p if p is not None else _norm()), Xo, Y, None)
    assert lib.lf_gate_norm(FAKE, None, None, None, None, None, None, None, None, None, FAKE, None) == -1
    assert call(X=None) == call(Y=None) == call(Xo=None) == call(B=None) == call(B=None, gate=None) == call(B=None, post=None) == -1
    assert call(p=_norm(group_len=0)) == -1        # no starts
    for kw, code in BAD_NORM + [(dict(x_stride=1000), -2), (dict(shift_stride=1538), -5), (dict(x_stride=1540), -5)]:
        assert call(p=_norm(**kw)) == code, kw
    for k in ("X", "B", "gate", "post", "w", "sc", "sh", "Xo", "Y"):
        assert call(**{k: FAKE + 8}) == -5, k
    assert call(st=FAKE + 2, p=_norm(group_len=0)) == -5


def test_gate_norm_backward_refuses_bad_arguments(lib):
    need = lf.lf_gate_norm_bwd_workspace_bytes(4680, 1536, 3, 1560)
    assert need > 0 and need % (1536 * 4) == 0 and lf.lf_gate_norm_bwd_workspace_bytes(4680, 1540, 3, 1560) == 0
    assert lf.lf_gate_norm_bwd_workspace_bytes(1, 8, 1, 1) == (3 + 2) * 8 * 4 and lf.lf_gate_norm_bwd_workspace_bytes(1 << 40, 8, 1, 1) == 0

    def call(Xo=FAKE, B=FAKE, gate=FAKE, post=FAKE, w=FAKE, sc=FAKE, st=None, p=None, dY=FAKE, dXo=FAKE, dX=FAKE, dB=FAKE, dg=FAKE, dp=FAKE, dw=FAKE, ds=FAKE, dh=FAKE,
             ws=FAKE, n=need):
        return lib.lf_gate_norm_bwd(Xo, B, gate, post, w, sc, st, C.byref(p if p is not None else _norm()), dY, dXo, dX, dB, dg, dp, dw, ds, dh, ws, n, None)
    for kw in (dict(Xo=None), dict(dX=None), dict(B=None), dict(dB=None), dict(post=None), dict(w=None), dict(B=None, dB=None, gate=None, post=None, dp=None),
               dict(p=_norm(group_len=0))):
        assert call(**kw) == -1, kw
    for kw, code in BAD_NORM:
        assert call(p=_norm(**kw)) == code, kw
    assert call(ws=None) == -6 and call(n=need - 1) == -6 and call(ws=FAKE + 16) == -5
    for k in ("Xo", "B", "gate", "post", "w", "sc", "dY", "dXo", "dX", "dB", "dg", "dp", "dw", "ds", "dh"):
        assert call(**{k: FAKE + 4}) == -5, k
    # more slots than a grid has workgroups for
    assert call(p=_norm(tokens=1 << 30, channels=8, groups=1 << 24, group_len=64, x_stride=8, xo_stride=8, b_stride=8, y_stride=8), n=1 << 60) in (-2,)


def _packed(**kw):
    s = lf.lf_packed_shape(40, 8, 128, 7, 16384, 16384, 1, 0, 128, 128 * 16384, 128, 128 * 16384, 128, 128 * 16384, 128, 128 * 16384)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


BAD_PACKED = [(dict(head_dim=96), -2), (dict(kv_heads=0), -2), (dict(kv_heads=4097, heads=4097), -2), (dict(heads=41), -2), (dict(heads=0), -2), (dict(heads=257, kv_heads=1), -2),
              (dict(seqs=0), -2), (dict(seqs=(1 << 20) + 1), -2), (dict(q_len=-1), -2), (dict(kv_len=-1), -2), (dict(q_len=(1 << 30) + 1), -2), (dict(causal=-1), -2),
              (dict(causal=(1 << 30) + 1), -2), (dict(q_len=1 << 30), -2), (dict(kv_len=1 << 30, kv_heads=40), -2), (dict(dtype=1), -4), (dict(q_stride_tok=120), -2),
              (dict(k_stride_tok=(1 << 20) + 8), -2), (dict(v_stride_head=-8), -2), (dict(o_stride_tok=132), -5), (dict(k_stride_head=128 * 16384 + 4), -5)]


def test_packed_attention_refuses_bad_arguments(lib):
    need = lf.lf_packed_attn_workspace_bytes(40, 8, 128, 16, 16, 120003, 1)
    few = dict(seqs=16, q_len=16, kv_len=120003)

    def call(Q=FAKE, K=FAKE, V=FAKE, s=None, a=FAKE, b=FAKE, scale=0.0, O=FAKE, l=FAKE, ws=FAKE, n=0):
        return lib.lf_packed_attn(Q, K, V, C.byref(s if s is not None else _packed()), a, b, scale, O, l, ws, n, None)
    assert call(Q=None) == call(K=None) == call(V=None) == call(O=None) == call(a=None) == call(b=None) == -1
    assert lib.lf_packed_attn(FAKE, FAKE, FAKE, None, FAKE, FAKE, 0.0, FAKE, None, None, 0, None) == -1
    for kw, code in BAD_PACKED + [(dict(o_stride_head=64), -2)]:
        assert call(s=_packed(**kw)) == code, kw
    for scale in (-1.0, float("nan"), float("inf"), 1e-40, 0.99e-30, 1.01e20, 3e38):
        assert call(scale=scale) == -2
    assert all(call(s=_packed(**few), scale=scale, n=need - 1) == -6 for scale in (0.0, 1e-30, 1e20))
    assert need > 0 and call(s=_packed(**few), n=need - 1) == -6 and call(s=_packed(**few), ws=None, n=need) == -6 and call(s=_packed(**few), ws=FAKE + 16, n=need) == -5
    for k in ("Q", "K", "V", "O"):
        assert call(**{k: FAKE + 8}) == -5
    assert call(a=FAKE + 2) == call(b=FAKE + 2) == call(l=FAKE + 2) == -5
    assert call(Q=None, O=None, s=_packed(q_len=0)) == 0           # nothing to do


def test_packed_backward_refuses_bad_arguments(lib):
    need = lf.lf_packed_attn_bwd_workspace_bytes(40, 8, 128, 7, 16384, 16384, 1)
    assert need == 40 * 16384 * 8

    def call(Q=FAKE, K=FAKE, V=FAKE, O=FAKE, dO=FAKE, l=FAKE, s=None, a=FAKE, b=FAKE, scale=0.0, dQ=FAKE, dK=FAKE, dV=FAKE, ws=FAKE, n=need):
        return lib.lf_packed_attn_bwd(Q, K, V, O, dO, l, C.byref(s if s is not None else _packed()), a, b, scale, dQ, dK, dV, ws, n, None)
    for k in ("Q", "K", "V", "O", "dO", "l", "a", "b", "dQ", "dK", "dV"):
        assert call(**{k: None}) == -1, k
    for kw, code in BAD_PACKED + [(dict(q_stride_head=64), -2), (dict(k_stride_head=0), -2), (dict(v_stride_head=128), -2)]:
        assert call(s=_packed(**kw), n=1 << 60) == code, kw
    assert call(scale=-1.0) == call(scale=1e-31) == call(scale=1e21) == -2 and call(scale=1e-30, n=need - 1) == -6 and call(ws=None) == call(n=need - 1) == -6
    for k in ("Q", "K", "V", "O", "dO", "dQ", "dK", "dV"):
        assert call(**{k: FAKE + 8}) == -5, k
    assert call(ws=FAKE + 16) == call(l=FAKE + 2) == call(a=FAKE + 1) == -5


def test_which_kernels_a_packed_call_takes(lib):
    """From the scratch that divided calls ask for: tiles of 16 and 32 rows and head, or of 128 rows."""
    def states(H, Hk, d, seqs, q, kv):
        return lf.lf_packed_attn_workspace_bytes(H, Hk, d, seqs, q, kv, 1) // ((d + 2) * 4)
    assert states(12, 12, 128, 1, 1, 512) == 0 and states(12, 12, 128, 1, 1, 513) > 0       # short axes stay whole
    assert states(12, 12, 128, 1, 1, 130000) == 12 * 21 * 16                                  # one tile of 16 rows a head, 21 parts: 252 workgroups
    assert states(3, 3, 128, 1, 1, 130000) == 3 * 64 * 16                                    # 64 parts at the most
    assert states(40, 8, 128, 16, 16, 120003) % (17 * 8 * 0 + 8 * 16) == 0
    assert states(40, 8, 128, 1, 4, 130000) % (8 * 32) == 0                                    # 20 rows and heads: tiles of 32
    assert states(1, 1, 64, 1, 33, 130000) % 128 == 0                                          # more than 32 rows
    assert states(12, 12, 128, 1, 32760, 32760) == 0                                           # enough tiles
    assert states(6, 2, 64, 9, 1352, 1352) == 0                                                # short sequences


def _grads(lib, entries, count=None, max_norm=1.0, eps=1e-6, norm=FAKE, ws=FAKE, n=1 << 40):
    t = (lf.lf_grad_tensor * max(len(entries), 1))(*[lf.lf_grad_tensor(*e) for e in entries])
    return lib.lf_grad_clip(t, len(entries) if count is None else count, max_norm, eps, norm, ws, n, None)


def test_clipping_refuses_bad_arguments(lib):
    ok = (FAKE, None, 10, 0, 0)
    assert lib.lf_grad_clip(None, 1, 1.0, 0.0, FAKE, FAKE, 1 << 40, None) == -1 and _grads(lib, [ok], norm=None) == -1 and _grads(lib, [(None, None, 10, 0, 0)]) == -1
    for kw in (dict(count=-1), dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))):
        assert _grads(lib, [ok], **kw) == -2, kw
    assert _grads(lib, [(FAKE, None, -1, 0, 0)]) == -2 and _grads(lib, [(FAKE, None, (1 << 40) + 1, 0, 0)]) == -2
    assert _grads(lib, [(FAKE, None, 1 << 40, 0, 0), ok]) == -2
    assert _grads(lib, [(FAKE, None, 10, 2, 0)]) == -4 and _grads(lib, [(FAKE, 2 * FAKE, 10, 0, 7)]) == -4 and _grads(lib, [(FAKE, FAKE, 10, 0, 1)]) == -4
    assert _grads(lib, [(FAKE + 1, None, 10, 0, 0)]) == -5 and _grads(lib, [(FAKE + 2, None, 10, 1, 0)]) == -5 and _grads(lib, [(FAKE, FAKE + 2, 10, 0, 1)]) == -5
    need = lf.lf_grad_workspace_bytes(1, 10)
    assert need == (0 + 1 + 1) * 8 and _grads(lib, [ok], n=need - 1) == -6 and _grads(lib, [ok], ws=None) == -6
    assert _grads(lib, [ok], ws=FAKE + 8) == _grads(lib, [ok], norm=FAKE + 2) == -5
    assert lf.lf_grad_workspace_bytes(-1, 5) == lf.lf_grad_workspace_bytes(1, -5) == lf.lf_grad_workspace_bytes(1 << 40, 5) == lf.lf_grad_workspace_bytes(1, 1 << 41) == 0


def test_clipping_refuses_a_tensor_that_is_scaled_twice(lib):
    """Judged from addresses; calls that are let through miss their workspace."""
    let = lambda *e, **kw: _grads(lib, list(e), n=0, **kw) == -6
    a, b, c = FAKE, 2 * FAKE, 3 * FAKE
    assert let((a, None, 10, 0, 0), (b, None, 10, 0, 0)) and let((b, None, 10, 0, 0), (a, None, FAKE // 2, 0, 0)) and let((b, None, 1, 0, 0), (a, None, FAKE // 4, 1, 0))
    assert not let((b, None, 10, 0, 0), (a, None, FAKE // 2 + 1, 0, 0)) and not let((b, None, 1, 0, 0), (a, None, FAKE // 4 + 1, 1, 0))
    for twice in ([(a, None, 10, 0, 0)] * 2, [(a, None, 10, 0, 0), (a + 18, None, 10, 0, 0)], [(a, b, 10, 0, 0), (c, b, 10, 0, 0)], [(a, b, 10, 0, 0), (b, None, 10, 0, 0)],
                  [(a, b, 10, 0, 0), (b, c, 10, 0, 0)], [(a, a, 10, 0, 0), (a, b, 10, 0, 0)], [(a, a + 2, 10, 0, 0)], [(a, b, FAKE // 2, 0, 1), (c - 2, None, 5, 0, 0)]):
        assert _grads(lib, twice, n=0) == -2, twice
        rest = [(a + (i << 32), None, 9, 0, 0) for i in range(1, 100)]
        assert _grads(lib, rest + twice, n=0) == -2 and let(*rest)
    assert let((a, b, 10, 0, 0), (a, c, 10, 0, 1))                                              # read twice: counted twice
    assert let((a, None, 10, 0, 0), (a, None, 10, 0, 0), max_norm=float("inf"))                 # nothing is written
    assert not let((a, b, 10, 0, 0), (b, None, 10, 0, 0), max_norm=float("inf"))
    assert let((a, None, 0, 0, 0), (a, None, 10, 0, 0), (a, a, 0, 0, 0))


def test_host_side_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    """lf_host_blocks.cpp on the CPU with -fsanitize=address,undefined: sizes at and past every limit; what reaches a launcher fits its grid, its threads
    and the workspace that was asked for."""
    import subprocess
    from paper_2602_04789_amd import build
    exe = build.build_sanitized_host(str(tmp_path), ("lf_host_blocks.cpp",), "host_blocks_sanitize_driver.cpp", "lf_host_blocks_sanitized")
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1")
    res = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=120)
    assert res.returncode == 0 and "ALL OK" in res.stdout, res.stdout[-3000:]
