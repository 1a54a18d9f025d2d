"""Argument checks and sizes of the three-axis producer and of the 4-bit cache's calls: every refusal is reported before
anything is enqueued (no GPU)."""
import ctypes as C
import os
import re

import pytest

from oracle import rollout_oracle as R
from paper_2602_04789_amd import lf, synth

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
    assert {"lf_qk_norm_rope_axes", "lf_qk_norm_rope_axes_bwd", "lf_qk_norm_rope_axes_bwd_workspace_bytes", "lf_kvq_bytes",
            "lf_kvq_append", "lf_kvq_read", "lf_sparse_attn_kvq", "lf_sparse_attn_kvq_workspace_bytes", "lf_token_attn_kvq",
            "lf_token_attn_kvq_workspace_bytes"} <= names
    assert C.sizeof(lf.lf_axes_shape) == 10 * 4 + 3 * 8 and C.sizeof(lf.lf_kvq_shape) == 16
    assert C.sizeof(lf.lf_kvq_rows) == 8 + 4 * 8 and C.sizeof(lf.lf_token_shape) == 24 + 8 * 8


def _axes(**kw):
    p = lf.lf_axes_shape(12, 128, 4680, 0, 0, (C.c_int32 * 3)(22, 21, 21), 1e-6, 0, 1536, 128, 128 * 4680)
    for k, v in kw.items():
        setattr(p, k, (C.c_int32 * 3)(*v) if k == "pairs" else v)
    return p


BAD_AXES = [(dict(head_dim=96), -2), (dict(heads=0), -2), (dict(heads=129), -2), (dict(tokens=0), -2), (dict(tokens=(1 << 30) + 1), -2),
            (dict(across_heads=2), -2), (dict(pairing=-1), -2), (dict(pairs=(22, 21, 20)), -2), (dict(pairs=(-1, 44, 21)), -2),
            (dict(pairs=(2 ** 31 - 1, 2 ** 31 - 1, 66)), -2), (dict(eps=-1.0), -2), (dict(eps=float("nan")), -2),
            (dict(x_stride_tok=1528), -2), (dict(y_stride_tok=64), -2), (dict(x_stride_tok=1540), -5), (dict(y_stride_head=128 * 4680 + 4), -5)]


def test_axes_producer_refuses_bad_arguments(lib):
    call = lambda X=FAKE, g=FAKE, pos=FAKE, f=FAKE, p=None, Y=FAKE: lib.lf_qk_norm_rope_axes(
        X, g, pos, f, C.byref(p if p is not None else _axes()), Y, None)
    assert lib.lf_qk_norm_rope_axes(FAKE, FAKE, FAKE, FAKE, None, FAKE, None) == -1
    assert call(X=None) == call(g=None) == call(pos=None) == call(f=None) == call(Y=None) == -1
    for kw, code in BAD_AXES + [(dict(y_stride_head=64), -2)]:        # (heads that overlap where they are written)
        assert call(p=_axes(**kw)) == code, kw
    assert call(X=FAKE + 8) == call(g=FAKE + 4) == call(pos=FAKE + 2) == call(f=FAKE + 4) == call(Y=FAKE + 2) == -5


def test_axes_backward_refuses_bad_arguments(lib):
    need = lf.lf_qk_norm_rope_axes_bwd_workspace_bytes(12, 128, 4680)
    assert need > 0 and need % (1536 * 4) == 0 and lf.lf_qk_norm_rope_axes_bwd_workspace_bytes(12, 96, 4680) == 0
    assert lf.lf_qk_norm_rope_axes_bwd_workspace_bytes(12, 128, 1) == 1536 * 4
    call = lambda X=FAKE, g=FAKE, pos=FAKE, f=FAKE, p=None, dY=FAKE, dX=FAKE, dg=FAKE, ws=FAKE, n=need: lib.lf_qk_norm_rope_axes_bwd(
        X, g, pos, f, C.byref(p if p is not None else _axes()), dY, dX, dg, ws, n, None)
    for kw in (dict(X=None), dict(g=None), dict(pos=None), dict(f=None), dict(dY=None), dict(dX=None), dict(dg=None)):
        assert call(**kw) == -1, kw
    for kw, code in BAD_AXES:
        assert call(p=_axes(**kw)) == code, kw
    assert call(ws=None) == -6 and call(n=need - 1) == -6
    assert call(ws=FAKE + 16) == call(dY=FAKE + 8) == call(dX=FAKE + 8) == call(dg=FAKE + 2) == -5


def _kvq(**kw):
    s = lf.lf_kvq_shape(12, 128, 32760, 0)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


BAD_CACHE = [dict(heads=0), dict(heads=32768), dict(head_dim=96), dict(capacity=0), dict(capacity=(1 << 24) + 1)]


def test_cache_size_and_store_refusals(lib):
    for H, d, cap in ((12, 128, 32760), (1, 64, 1), (3, 64, 77), (40, 128, 1 << 24)):
        assert lf.lf_kvq_bytes(H, d, cap) == R.cache_parts(H, cap, d)[1]
    for kw in BAD_CACHE:
        assert lib.lf_kvq_bytes(C.byref(_kvq(**kw))) == 0
    assert lib.lf_kvq_bytes(None) == 0
    need = lf.lf_kvq_bytes(12, 128, 32760)

    def rows(**kw):
        r = lf.lf_kvq_rows(28080, 4680, 128, 128 * 4680, 128, 128 * 4680)
        for k, v in kw.items():
            setattr(r, k, v)
        return r
    app = lambda K=FAKE, V=FAKE, s=None, r=None, c=FAKE, n=need: lib.lf_kvq_append(
        K, V, C.byref(s or _kvq()), C.byref(r or rows()), c, n, None)
    read = lambda K=FAKE, V=FAKE, s=None, r=None, c=FAKE, n=need: lib.lf_kvq_read(
        c, n, C.byref(s or _kvq()), C.byref(r or rows()), K, V, None)
    for call in (app, read):
        assert call(K=None) == call(V=None) == -1
        for kw in BAD_CACHE:
            assert call(s=_kvq(**kw)) == -2, kw
        for kw in (dict(first=-1), dict(first=28081), dict(tokens=-1), dict(first=2 ** 31 - 1), dict(k_stride_tok=64), dict(v_stride_tok=0)):
            assert call(r=rows(**kw)) == -2, kw
        for kw in (dict(k_stride_tok=132), dict(v_stride_head=128 * 4680 + 4)):
            assert call(r=rows(**kw)) == -5, kw
        assert call(c=None) == -6 and call(n=need - 1) == -6
        assert call(K=FAKE + 8) == call(V=FAKE + 2) == call(c=FAKE + 128) == -5
        assert call(K=None, V=None, r=rows(tokens=0)) == 0        # nothing to do, nothing enqueued
    assert read(r=rows(k_stride_head=0)) == -2 and read(r=rows(v_stride_head=64)) == -2      # written: heads must lie apart
    assert lib.lf_kvq_append(FAKE, FAKE, None, C.byref(rows()), FAKE, need, None) == -1
    assert lib.lf_kvq_read(FAKE, need, C.byref(_kvq()), None, FAKE, FAKE, None) == -1


def _shape(**kw):
    w = synth.cfg_last_chunk()
    sh = lf.lf_shape()
    sh.heads, sh.head_dim, sh.frame_len, sh.block = w.heads, w.head_dim, w.frame_len, 64
    sh.q_len, sh.kv_len, sh.dtype = w.q_len, w.kv_len, 0
    for t in "qkvo":
        setattr(sh, f"{t}_stride_tok", w.head_dim)
        setattr(sh, f"{t}_stride_head", w.head_dim * w.q_len)
    for k, v in kw.items():
        setattr(sh, k, v)
    return sh


def test_sparse_attention_over_the_cache_refuses_bad_arguments(lib):
    nbytes = lf.lf_kvq_bytes(12, 128, 32760)
    need = lib.lf_sparse_attn_kvq_workspace_bytes(C.byref(_shape()), 188)
    call = lambda Q=FAKE, c=FAKE, n=nbytes, cs=None, K=FAKE, V=FAKE, s=None, idx=FAKE, ll=188, sc=0.0, O=FAKE, ws=FAKE, wn=need: \
        lib.lf_sparse_attn_kvq(Q, c, n, C.byref(cs or _kvq()), K, V, C.byref(s or _shape()), idx, ll, sc, O, ws, wn, None)
    assert call(Q=None) == call(idx=None) == call(O=None) == call(K=None) == call(V=None) == -1
    assert lib.lf_sparse_attn_kvq(FAKE, FAKE, nbytes, None, None, None, C.byref(_shape()), FAKE, 8, 0.0, FAKE, FAKE, need, None) == -1
    assert lib.lf_sparse_attn_kvq(FAKE, FAKE, nbytes, C.byref(_kvq()), None, None, None, FAKE, 8, 0.0, FAKE, FAKE, need, None) == -1
    assert call(ll=0) == call(ll=(1 << 30) + 1) == -3 and call(sc=-1.0) == call(sc=float("nan")) == call(sc=float("inf")) == -2
    for kw, code in ((dict(block=32), -2), (dict(head_dim=96), -2), (dict(dtype=1), -4), (dict(heads=11), -2), (dict(q_len=4681), -2),
                     (dict(kv_len=1560), -2), (dict(kv_len=1560 * 25), -2), (dict(k_stride_tok=64), -2), (dict(v_stride_tok=132), -5),
                     (dict(o_stride_head=0), -2), (dict(q_stride_head=4), -5)):
        assert call(s=_shape(**kw)) == code, kw
    # without K and V all kv_len tokens lie in the cache, and their strides are not looked at
    assert call(K=None, V=None, cs=_kvq(capacity=32759)) == -2 and call(cs=_kvq(capacity=28079)) == -2
    assert call(K=None, V=None, s=_shape(k_stride_tok=4), idx=FAKE + 2) == -5
    for kw in BAD_CACHE:
        assert call(cs=_kvq(**kw)) == -2, kw
    assert call(c=None) == -6 and call(n=nbytes - 1) == -6
    for kw in (dict(Q=FAKE + 8), dict(c=FAKE + 64), dict(K=FAKE + 8), dict(V=FAKE + 8), dict(O=FAKE + 8), dict(idx=FAKE + 2)):
        assert call(**kw) == -5, kw
    few = _shape(heads=12, frame_len=64, q_len=64, kv_len=64 * 200)       # 12 query blocks: their lists are divided
    need = lib.lf_sparse_attn_kvq_workspace_bytes(C.byref(few), 200)
    assert need > 0
    assert call(s=few, ll=200, ws=None) == -6 and call(s=few, ll=200, wn=need - 1) == -6 and call(s=few, ll=200, ws=FAKE + 64, wn=need) == -5
    assert lib.lf_sparse_attn_kvq_workspace_bytes(None, 8) == 0 and lib.lf_sparse_attn_kvq_workspace_bytes(C.byref(few), 0) == 0


def test_token_attention_refuses_bad_arguments(lib):
    def shape(**kw):
        s = lf.lf_token_shape(12, 128, 1, 32760, 1, 0, 128, 128, 128, 128, 128, 128, 128, 128)
        for k, v in kw.items():
            setattr(s, k, v)
        return s
    nbytes = lf.lf_kvq_bytes(12, 128, 32760)
    need = lib.lf_token_attn_kvq_workspace_bytes(C.byref(shape()))
    assert need > 0 and lib.lf_token_attn_kvq_workspace_bytes(C.byref(shape(cached_len=5))) == 0
    assert lf.lf_token_attn_kvq_workspace_bytes(12, 128, 1, 32760, 1) == need and lib.lf_token_attn_kvq_workspace_bytes(None) == 0
    call = lambda Q=FAKE, c=FAKE, n=nbytes, cs=None, K=FAKE, V=FAKE, s=None, sc=0.0, O=FAKE, ws=FAKE, wn=need: \
        lib.lf_token_attn_kvq(Q, c, n, C.byref(cs or _kvq()), K, V, C.byref(s or shape()), sc, O, ws, wn, None)
    assert call(Q=None) == call(O=None) == call(K=None) == call(V=None) == -1
    assert lib.lf_token_attn_kvq(FAKE, FAKE, nbytes, None, FAKE, FAKE, C.byref(shape()), 0.0, FAKE, FAKE, need, None) == -1
    assert lib.lf_token_attn_kvq(FAKE, FAKE, nbytes, C.byref(_kvq()), FAKE, FAKE, None, 0.0, FAKE, FAKE, need, None) == -1
    for kw, code in ((dict(heads=0), -2), (dict(heads=11), -2), (dict(head_dim=64), -2), (dict(head_dim=32), -2), (dict(q_len=0), -2),
                     (dict(q_len=65), -2), (dict(cached_len=-1), -2), (dict(cached_len=32761), -2), (dict(extra_len=-1), -2),
                     (dict(extra_len=(1 << 24) + 1), -2), (dict(q_stride_tok=64), -2), (dict(k_stride_tok=0), -2), (dict(o_stride_head=0), -2),
                     (dict(v_stride_head=4), -5), (dict(o_stride_tok=132), -5)):
        assert call(s=shape(**kw)) == code, kw
    assert call(sc=-0.5) == call(sc=float("inf")) == -2
    assert call(c=None) == -6 and call(n=nbytes - 1) == -6 and call(ws=None) == -6 and call(wn=need - 1) == -6
    for kw in (dict(Q=FAKE + 8), dict(c=FAKE + 64), dict(K=FAKE + 8), dict(V=FAKE + 8), dict(O=FAKE + 8), dict(ws=FAKE + 64)):
        assert call(**kw) == -5, kw


def test_binding_refuses_wrong_tensors():
    """What the binding checks before it asks for the library (CPU tensors are refused)."""
    import torch
    X, Y = torch.zeros(4, 128, dtype=torch.bfloat16), torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    g, pos, freq = torch.ones(128), torch.zeros(4, 3, dtype=torch.int32), torch.ones(32, dtype=torch.float64)
    cache = torch.zeros(4096, dtype=torch.uint8)
    for call in (lambda: lf.lf_qk_norm_rope_axes(X, g, pos, freq, (12, 10, 10), 2, Y),
                 lambda: lf.lf_qk_norm_rope_axes_bwd(X, g, pos, freq, (12, 10, 10), 2, Y),
                 lambda: lf.lf_kvq_append(Y, Y, cache, 8, 0), lambda: lf.lf_kvq_read(cache, 2, 64, 8, 0, 4, Y, Y),
                 lambda: lf.lf_token_attn_kvq(Y, cache, 8, 4), lambda: lf.lf_token_attn_kvq(Y, cache, 8, 4, K=Y),
                 lambda: lf.lf_sparse_attn_kvq(Y, cache, 8, 8, pos, 4, 64)):
        with pytest.raises(ValueError):
            call()


def _parts(H, d, rows, cached, extra=0):
    """Workgroups that share a head's tokens, from the size of their states."""
    need = lf.lf_token_attn_kvq_workspace_bytes(H, d, rows, cached, extra)
    tiles = 1 if rows <= 16 else 2 if rows <= 32 else 4
    assert need % (H * 16 * tiles * (d + 2) * 4) == 0
    return need // (H * 16 * tiles * (d + 2) * 4) or 1


def test_how_token_attention_is_divided(lib):
    for rows, cached, extra, H, want in ((1, 1024, 0, 12, 1), (1, 1025, 0, 12, 4), (1, 960, 64, 12, 1), (1, 1024, 1, 12, 4), (32, 1024, 0, 12, 1),
                                         (33, 512, 0, 12, 1), (33, 513, 0, 12, 2), (64, 131072, 0, 12, 42), (1, 131072, 0, 1, 64),
                                         (1, 131072, 0, 256, 2), (1, 131072, 0, 257, 1), (1, 0, 1, 600, 1), (1, 0, 0, 3, 1)):
        assert _parts(H, 128, rows, cached, extra) == want, (rows, cached, extra, H)


def test_which_way_list_calls_go(lib):
    """Few query blocks over a long cache convert what they read; many tiles are worth the cache's rows in bfloat16."""
    for H, d, n, f, F, length, rows_first in ((12, 128, 1560, 3, 21, 188, True), (12, 64, 1560, 3, 21, 188, True), (12, 128, 64, 1, 400, 40, False),
                                              (40, 64, 256, 1, 100, 40, False), (1, 128, 256, 2, 260, 1000, False), (12, 128, 1560, 1, 20, 73, False),
                                              (12, 128, 1560, 1, 20, 180, True), (24, 64, 97, 3, 8, 14, True), (2, 64, 256, 1, 5, 12, False)):
        need = lf.lf_sparse_attn_kvq_workspace_bytes(H, d, n, 64, f * n, F * n, length)
        rows = 2 * ((H * F * n * d * 2 + 255) // 256 * 256)
        assert (need == rows) == rows_first, (H, d, n, f, F, length)


def test_host_side_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    """lf_host_rollout.cpp (with lf_host.cpp) on the CPU with -fsanitize=address,undefined: sizes at and past every limit; what
    reaches a launcher fits its grid, its LDS and the workspace that was asked for."""
    import subprocess
    from paper_2602_04789_amd import build
    exe = build.build_sanitized_host(str(tmp_path), ("lf_host.cpp", "lf_host_rollout.cpp"), "host_rollout_sanitize_driver.cpp",
                                     "lf_host_rollout_sanitized")
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1")
    res = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=120)
    assert res.returncode == 0 and "ALL OK" in res.stdout, res.stdout[-3000:]
