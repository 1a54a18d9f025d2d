"""Sizes that do not fit the int32 fields of the C structures: refused by the binding of the calls around the attention (ctypes would drop their upper bits, and
the call would run on other tokens, channels, heads or sequences).  No GPU: a stand-in for the library sees what would reach it."""
import pytest
import torch

from paper_2602_04789_amd import lf

BIG = (2 ** 31, 2 ** 32, 2 ** 32 + 8)


class Library:
    """Lets everything through."""

    def __getattr__(self, name):
        return lambda *a: 0


@pytest.fixture(autouse=True)
def on_the_cpu(monkeypatch):
    monkeypatch.setattr(lf, "_lib", Library())
    monkeypatch.setattr(lf, "_here", lambda stream: (-1, 0))
    monkeypatch.setattr(lf, "_rows", lambda t, name: (t.shape, t.stride(1), t.stride(0)))


def _wide(*shape, dtype=torch.bfloat16):
    """A tensor of any size that holds one element."""
    return torch.zeros((1,) * len(shape), dtype=dtype).expand(shape)


def _rows_of(L, n, dtype=torch.bfloat16):
    """[L, n] with contiguous channels, without their memory (only sizes and strides are looked at)."""
    return torch.empty((L, n), dtype=dtype, device="meta").as_strided((L, n), (n, 1))


def _refused(call, what):
    with pytest.raises(ValueError, match="32 bits"):
        call()
        print("taken:", what)


@pytest.mark.parametrize("big", BIG)
def test_norms_refuse_what_does_not_fit(big):
    for L, n in ((big, 8), (1, big)):
        X = _rows_of(L, n)
        for group_len in (1, L if L < 2 ** 31 else 1 << 30):
            _refused(lambda: lf.lf_gate_norm(X, group_len=group_len, Y=X), (L, n))
            _refused(lambda: lf.lf_gate_norm_bwd(X, X, dX=X, group_len=group_len, workspace=X), (L, n))
    X, starts = torch.zeros((4, 8), dtype=torch.bfloat16), _wide(big + 1, dtype=torch.int32)
    _refused(lambda: lf.lf_gate_norm(X, starts=starts), "groups")
    _refused(lambda: lf.lf_gate_norm_bwd(X, X, starts=starts), "groups")
    _refused(lambda: lf.lf_gate_norm(X, group_len=4, kind=big), "kind")


@pytest.mark.parametrize("big", BIG)
@pytest.mark.parametrize("which", ["heads", "kv_heads", "head_dim", "q_len", "kv_len", "causal"])
def test_packed_attention_refuses_what_does_not_fit(big, which):
    size = dict(heads=2, kv_heads=2, head_dim=64, q_len=4, kv_len=4, causal=0)
    size[which] = big
    Q, K = _wide(size["heads"], size["q_len"], size["head_dim"]), _wide(size["kv_heads"], size["kv_len"], size["head_dim"])
    s, lse2 = torch.zeros(2, dtype=torch.int32), torch.zeros((2, 4))
    _refused(lambda: lf.lf_packed_attn(Q, K, K, s, s, causal=size["causal"], O=Q), which)
    _refused(lambda: lf.lf_packed_attn_fwd(Q, K, K, s, s, causal=size["causal"], O=Q, lse2=lse2), which)
    _refused(lambda: lf.lf_packed_attn_bwd(Q, K, K, Q, Q, lse2, s, s, causal=size["causal"], grads=(Q, K, K)), which)


@pytest.mark.parametrize("big", BIG)
def test_packed_attention_refuses_more_sequences_than_fit(big):
    Q, lse2 = torch.zeros((2, 4, 64), dtype=torch.bfloat16), torch.zeros((2, 4))
    s = torch.empty(big + 1, dtype=torch.int32, device="meta")
    _refused(lambda: lf.lf_packed_attn(Q, Q, Q, s, s), "seqs")
    _refused(lambda: lf.lf_packed_attn_bwd(Q, Q, Q, Q, Q, lse2, s, s, grads=(Q, Q, Q)), "seqs")


def test_what_fits_is_let_through():
    X, starts = torch.zeros((4, 8), dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    assert lf.lf_gate_norm(X, group_len=2)[0] is X and lf.lf_gate_norm(X, starts=starts)[0] is X
    assert lf.lf_gate_norm_bwd(X, X, starts=starts)[0].shape == X.shape
    Q, s = torch.zeros((2, 4, 64), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    assert lf.lf_packed_attn(Q, Q, Q, s, s).shape == Q.shape


@pytest.mark.parametrize("big", BIG)
def test_sizes_of_what_does_not_fit_are_zero(big, monkeypatch):
    monkeypatch.setattr(lf, "_lib", None)
    for f, args in ((lf.lf_gate_norm_bwd_workspace_bytes, (40, 64, 4, 10)), (lf.lf_packed_attn_workspace_bytes, (2, 1, 64, 1, 5, 130000, 1)),
                    (lf.lf_packed_attn_bwd_workspace_bytes, (2, 1, 64, 1, 5, 5, 1)), (lf.lf_grad_workspace_bytes, (4, 100))):
        assert f(*args) > 0
        for at in range(len(args)):
            if f is not lf.lf_grad_workspace_bytes or at == 0:
                assert f(*args[:at], big, *args[at + 1:]) == 0, (f.__name__, at)
