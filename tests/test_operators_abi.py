"""The stand-alone operators reject invalid arguments on the host, before any
device work (CPU only: no address handed over here is real)."""
import ctypes
import math

import pytest
import torch

from paper_2608_22646_amd import binding as B

A = 0x10000  # a made-up, aligned address


def view(data=A, b=0, l=512, h=128):
    return B.View(data, b, l, h)


def rotary_rc(cfg=None, dtype=B.DLLM_BF16, Bn=1, L=2, q=None, q_out=None, n_q=2, k=None, k_out=None, n_k=0):
    c = dict(head_dim=128, rot_dim=128, interleaved=0, scaling=0, base=1e4, factor=1, orig_len=0, low=1, high=32, gain=1)
    c.update(cfg or {})
    return B.lib().dllm_rotary(B.RotaryCfg(**c), dtype, Bn, L, None, 0, q or view(), q_out or view(), n_q, k, k_out, n_k, 0,
                               None)


@pytest.mark.parametrize("kw,code", [
    (dict(cfg=dict(head_dim=1)), -2), (dict(cfg=dict(head_dim=513)), -2), (dict(cfg=dict(rot_dim=127)), -2),
    (dict(cfg=dict(rot_dim=0)), -2), (dict(cfg=dict(rot_dim=130)), -2), (dict(cfg=dict(head_dim=512, rot_dim=258)), -2),
    (dict(cfg=dict(base=0.0)), -1), (dict(cfg=dict(base=math.nan)), -1), (dict(cfg=dict(gain=math.inf)), -1),
    (dict(cfg=dict(scaling=3)), -1), (dict(cfg=dict(scaling=1, factor=0.0)), -1),
    (dict(cfg=dict(scaling=2, orig_len=0.0)), -1), (dict(cfg=dict(scaling=2, orig_len=10.0, low=2.0, high=2.0)), -1),
    (dict(dtype=2), -1), (dict(Bn=-1), -2), (dict(L=-1), -2), (dict(n_q=-1), -2), (dict(n_q=4097), -2),
    (dict(Bn=1 << 16, L=1 << 15), -2), (dict(q=view(0)), -1), (dict(q_out=view(0)), -1), (dict(q=view(l=-1)), -2),
    (dict(k=view(), n_k=1), -1), (dict(k=view(), k_out=view(0), n_k=1), -1), (dict(k=view(), k_out=view(), n_k=-1), -2),
])
def test_rotary_refuses(kw, code):
    assert rotary_rc(**kw) == code, B.lib().dllm_last_error()
    assert B.lib().dllm_last_error().decode() != ""


def test_rotary_of_nothing_is_nothing():
    for kw in (dict(Bn=0), dict(L=0), dict(n_q=0)):
        assert rotary_rc(**kw) == 0
    assert B.lib().dllm_rotary(None, 0, 1, 1, None, 0, None, None, 0, None, None, 0, 0, None) == -1


def attn_args(**kw):
    a = dict(dtype=B.DLLM_BF16, n_heads=4, n_kv_heads=2, head_dim=128, q=view(), k=view(l=256), v=view(l=256), out=view(),
             docs=1, q_tokens=8, kv_tokens=8, max_q=8, max_kv=8, scale=0.1, cap=0.0, block=0)
    a.update(kw)
    return B.AttnArgs(**a)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=5), -1), (dict(head_dim=96), -5), (dict(n_heads=3), -2), (dict(n_kv_heads=0), -2), (dict(n_heads=0), -2),
    (dict(docs=-1), -2), (dict(docs=65536), -2), (dict(max_q=9), -2), (dict(max_kv=9), -2), (dict(max_q=-1), -2),
    (dict(scale=math.nan), -1), (dict(scale=math.inf), -1), (dict(cap=-1.0), -1), (dict(cap=math.inf), -1), (dict(block=-1), -1),
    (dict(q=view(0)), -1), (dict(k=view(0)), -1), (dict(v=view(0)), -1), (dict(out=view(0)), -1),
    (dict(q=view(A + 8)), -5), (dict(k=view(l=260)), -5), (dict(v=view(h=132)), -5), (dict(out=view(l=64)), -2),
    (dict(docs=2, q=view(b=4)), -5), (dict(k=view(l=-128)), -2), (dict(v=view(l=1 << 24)), -2),
    (dict(n_heads=4096, n_kv_heads=1, max_q=1 << 20, q_tokens=1 << 20), -2),
])
def test_attention_refuses(kw, code):
    assert B.lib().dllm_attention(attn_args(**kw), None, 0, None) == code, B.lib().dllm_last_error()
    assert B.lib().dllm_last_error().decode() != ""


def test_attention_of_nothing_is_nothing():
    n = ctypes.c_size_t(7)
    for kw in (dict(docs=0), dict(max_q=0)):
        assert B.lib().dllm_attention(attn_args(**kw), None, 0, None) == 0
        assert B.lib().dllm_attention_workspace_size(attn_args(**kw), n) == 0 and n.value == 0
    assert B.lib().dllm_attention_workspace_size(attn_args(), None) == -1
    assert B.lib().dllm_attention_workspace_size(None, n) == -1
    assert B.lib().dllm_attention(None, None, 0, None) == -1


def test_attention_checks_its_workspace():
    """One query over a long cache splits its keys; the partial states need room."""
    a = attn_args(q_tokens=1, max_q=1, kv_tokens=100000, max_kv=100000)
    n = ctypes.c_size_t()
    assert B.lib().dllm_attention_workspace_size(a, n) == 0
    if n.value:
        assert B.lib().dllm_attention(a, None, 0, None) == -1
        assert B.lib().dllm_attention(a, ctypes.c_void_p(A + 16), n.value, None) == -1
        assert B.lib().dllm_attention(a, ctypes.c_void_p(A), n.value - 1, None) == -4


def sample_args(**kw):
    a = dict(logits=A, row_stride=100, dtype=B.DLLM_F32, rows=2, vocab=100, mask_id=-1, u=A, temperature=None, top_k=None,
             top_p=None, min_p=None, token=A, conf=None, prob=None)
    a.update(kw)
    return B.SampleArgs(**a)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=9), -1), (dict(rows=-1), -2), (dict(vocab=0), -2), (dict(vocab=(1 << 22) + 1), -2), (dict(row_stride=99), -2),
    (dict(logits=None), -1), (dict(u=None), -1), (dict(token=None), -1),
])
def test_sample_refuses(kw, code):
    assert B.lib().dllm_sample(sample_args(**kw), ctypes.c_void_p(A), 1 << 40, None) == code, B.lib().dllm_last_error()


def test_sample_checks_its_workspace_and_takes_no_rows():
    n = ctypes.c_size_t()
    assert B.lib().dllm_sample(sample_args(rows=0), None, 0, None) == 0
    assert B.lib().dllm_sample(None, None, 0, None) == -1
    assert B.lib().dllm_sample_workspace_size(1, 100, None) == -1
    assert B.lib().dllm_sample_workspace_size(-1, 100, n) == -2
    assert B.lib().dllm_sample_workspace_size(2, 100, n) == 0
    if n.value:
        assert B.lib().dllm_sample(sample_args(), None, 0, None) == -1
        assert B.lib().dllm_sample(sample_args(), ctypes.c_void_p(A), n.value - 1, None) == -4


def test_binding_refuses_tensors_that_are_not_on_the_gpu():
    x = torch.zeros((1, 2, 3, 64))
    for call in (lambda: B.rotary(B.Rotary(64), x), lambda: B.attention(x, x, x),
                 lambda: B.sample(torch.zeros((2, 10)), torch.zeros(2)),
                 lambda: B.rotary(B.Rotary(64), x.double()), lambda: B.rotary(B.Rotary(32), x),
                 lambda: B.attention(x[0, 0], x, x)):
        with pytest.raises(B.DllmError):
            call()
    with pytest.raises(KeyError):
        B.Rotary(64, scaling="cubic").to_c()


def test_struct_sizes_match_the_c_layout():
    assert ctypes.sizeof(B.RotaryCfg) == 64 and ctypes.sizeof(B.View) == 32
    assert ctypes.sizeof(B.AttnArgs) == 16 + 4 * 32 + 5 * 4 + 4 + 7 * 8 + 16
    assert ctypes.sizeof(B.SampleArgs) == 16 + 16 + 8 * 8
