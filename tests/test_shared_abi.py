"""dllm_shared_attention rejects invalid arguments on the host, before any device work (CPU only: no address handed over
here is real), and its binding refuses operands that do not belong together."""
import ctypes
import math

import pytest
import torch

from paper_2608_22646_amd import binding as B

A = 0x10000  # a made-up, aligned address


def view(data=A, b=0, l=512, h=128):
    return B.View(data, b, l, h)


def args(own=None, **kw):
    o = dict(dtype=B.DLLM_BF16, n_heads=4, n_kv_heads=2, head_dim=128, q=view(), k=view(l=256), v=view(l=256), out=view(),
             docs=2, q_tokens=8, kv_tokens=8, max_q=4, max_kv=8, scale=0.1, cap=0.0, block=0)
    o.update(own or {})
    a = dict(pk=view(l=256), pv=view(l=256), prompts=1, p_tokens=64, max_p=64)
    a.update(kw)
    return B.SharedAttnArgs(B.AttnArgs(**o), **a)


def call(a, ws=A, n=1 << 40):
    return B.lib().dllm_shared_attention(a, ws, n, None)


SIZES = [
    (dict(own=dict(dtype=5)), -1), (dict(own=dict(head_dim=96)), -5), (dict(own=dict(n_heads=3)), -2), (dict(own=dict(docs=-1)), -2),
    (dict(own=dict(docs=65536)), -2), (dict(own=dict(max_q=9)), -2), (dict(own=dict(max_kv=9)), -2), (dict(own=dict(scale=math.nan)), -1),
    (dict(own=dict(cap=-1.0)), -1), (dict(own=dict(block=-1)), -1), (dict(prompts=-1), -2), (dict(prompts=65536), -2), (dict(max_p=-1), -2),
    (dict(max_p=65), -2), (dict(p_tokens=(1 << 29) + 1), -2), (dict(own=dict(kv_tokens=(1 << 29) + 1)), -2),
    (dict(own=dict(docs=65535, q_tokens=1 << 30, max_q=1 << 14, n_heads=4, n_kv_heads=4, q=view(b=1 << 20))), -2),
    (dict(own=dict(docs=65535, q_tokens=1 << 30, max_q=1, n_heads=4096, n_kv_heads=4096, q=view(b=1 << 20), out=view(b=1 << 20))), -2),
]


@pytest.mark.parametrize("kw,code", SIZES + [
    (dict(own=dict(q=view(0))), -1), (dict(own=dict(k=view(0))), -1), (dict(own=dict(out=view(0))), -1), (dict(own=dict(q=view(A + 8))), -5),
    (dict(pk=view(0)), -1), (dict(pv=view(0)), -1), (dict(pk=view(A + 8)), -5), (dict(pv=view(l=260)), -5), (dict(pk=view(l=-256)), -2),
    (dict(pk=view(l=64)), -2), (dict(pv=view(l=1 << 24)), -2), (dict(pk=view(b=4), prompts=2), -5),
])
def test_refuses(kw, code):
    assert call(args(**kw)) == code, B.lib().dllm_last_error()
    assert B.lib().dllm_last_error().decode() != ""


@pytest.mark.parametrize("kw,code", SIZES)
def test_workspace_size_refuses_the_same_sizes(kw, code):
    assert B.lib().dllm_shared_attention_workspace_size(args(**kw), ctypes.c_size_t(7)) == code


def test_workspace():
    n, m = ctypes.c_size_t(), ctypes.c_size_t()
    size = B.lib().dllm_shared_attention_workspace_size
    assert size(None, n) == -1 and size(args(), None) == -1 and call(None) == -1
    for own in (dict(docs=0), dict(max_q=0)):
        assert size(args(own), n) == 0 and n.value == 0 and call(args(own), None, 0) == 0
    split = args(p_tokens=20000, max_p=20000)  # few rows behind many keys
    assert size(split, n) == 0 and n.value > 0
    assert call(split, A, n.value - 1) == -4
    assert call(split, None, n.value) == -1
    assert call(split, A + 128, n.value) == -1
    # without a prompt's key: the workspace of attention of documents
    long = dict(kv_tokens=8192, max_kv=8192)
    for kw in (dict(prompts=0), dict(max_p=0)):
        a = args(long, **kw)
        assert size(a, n) == 0 and B.lib().dllm_attention_workspace_size(a.own, m) == 0 and n.value == m.value > 0
    # row tiles that take prompt and own keys in one go, of few keys or of rows that fill the CUs: none
    assert size(args(), n) == 0 and n.value == 0
    many = dict(docs=256, q_tokens=256, max_q=256, q=view(b=1 << 17), n_heads=4, n_kv_heads=2)
    assert size(args(many), n) == 0 and n.value == 0


def test_binding_refuses_the_wrong_tensors():
    q, k, p = torch.zeros(4, 4, 64), torch.zeros(8, 2, 64), torch.zeros(16, 2, 64)
    for bad in (dict(q=q[0]), dict(k=k[None]), dict(pk=p[0]), dict(pk=p[None]), dict()):  # the last: not on the GPU
        with pytest.raises(B.DllmError):
            B.shared_attention(**{**dict(q=q, k=k, v=k, pk=p, pv=p), **bad})


@pytest.mark.parametrize("kw,code", [
    (dict(pk=torch.zeros(16, 3, 64)), -2), (dict(pv=torch.zeros(15, 2, 64)), -2), (dict(pk=torch.zeros(16, 2, 64).bfloat16()), -1),
    (dict(prompts=B.Prompts(start=torch.zeros(1, dtype=torch.int64))), -1), (dict(prompts=B.Prompts(of=torch.zeros(2, dtype=torch.int32))), -2),
    (dict(prompts=B.Prompts(start=torch.zeros(2, dtype=torch.int32), len=torch.zeros(3, dtype=torch.int32))), -2),
    (dict(prompts=B.Prompts(max=1 << 31)), -2), (dict(pk=torch.zeros(2, 8, 2, 64), pv=torch.zeros(2, 8, 2, 64), prompts=B.Prompts(count=1)), -2),
])
def test_marshalling_refuses(kw, code):
    p = torch.zeros(16, 2, 64)
    a = dict(dt=B.DLLM_F32, q=torch.zeros(4, 4, 64), k=torch.zeros(8, 2, 64), v=torch.zeros(8, 2, 64), pk=p, pv=p, out=torch.zeros(4, 4, 64),
             docs=B.Docs(), prompts=B.Prompts(), block=0, scale=None, cap=0.0, slopes=None)
    with pytest.raises(B.DllmError) as e:
        B._shared_args(**{**a, **kw})
    assert e.value.code == code


def test_packed_prompts():
    p = B.Prompts.packed([3, 0, 5], [2, -1], device="cpu")
    assert p.start.tolist() == [0, 3, 3] and p.len.tolist() == [3, 0, 5] and p.max == 5 and p.of.tolist() == [2, -1]
    e = B.Prompts.packed([], device="cpu")
    assert e.start.numel() == 0 and e.max == 0 and e.of is None


@pytest.mark.parametrize("docs,q,p", [(1, 700, 100), (2, 2000, 300), (3, 294, 64), (1, 405, 357), (8, 40, 200), (16, 64, 60), (4, 700, 2000)])
@pytest.mark.parametrize("dtype", [B.DLLM_F32, B.DLLM_BF16])
def test_workspace_of_any_block_mask(docs, q, p, dtype):
    """The size does not depend on the block mask, which the binding's query is not told of."""
    size = 0x100 * 4
    own = dict(dtype=dtype, n_heads=28, n_kv_heads=4, docs=docs, q_tokens=docs * q, kv_tokens=docs * q, max_q=q, max_kv=q,
               q=view(l=28 * 128), k=view(l=size), v=view(l=size), out=view(l=28 * 128))
    got = []
    for block in (0, 1, 32):
        n = ctypes.c_size_t()
        assert B.lib().dllm_shared_attention_workspace_size(args(dict(own, block=block), p_tokens=p, max_p=p), n) == 0
        got.append(n.value)
    assert got[0] == got[1] == got[2]
