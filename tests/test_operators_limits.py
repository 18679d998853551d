"""Limits of the stand-alone operators that the host checks, on both sides of each (CPU only: no address
handed over here is real, and what is accepted is only asked for its workspace)."""
import ctypes
import math

import pytest

from paper_2608_22646_amd import binding as B
from test_operators_abi import attn_args, rotary_rc

# documents, query heads, key/value heads, head_dim, most queries, type; a few documents and a head more do not fit
LARGEST = [
    (8191, 32, 8, 128, 8192, B.DLLM_BF16),      # 65528 units of 256 tiles, 256 threads each
    (32760, 256, 256, 64, 33, B.DLLM_BF16),     # a tile of 64 rows, 512 threads
    (65520, 256, 256, 64, 1, B.DLLM_F32),       # one query of each head
]


@pytest.mark.parametrize("docs,n_heads,n_kv,hd,max_q,dtype", LARGEST)
def test_attention_refuses_what_one_launch_cannot_hold(docs, n_heads, n_kv, hd, max_q, dtype):
    n = ctypes.c_size_t()
    sizes = dict(n_heads=n_heads, n_kv_heads=n_kv, head_dim=hd, dtype=dtype, q_tokens=1 << 20, kv_tokens=1 << 20, max_q=max_q,
                 max_kv=8192)
    assert B.lib().dllm_attention_workspace_size(attn_args(docs=docs, **sizes), n) == 0
    more = attn_args(**dict(sizes, docs=docs + 8, n_heads=n_heads + n_heads // n_kv, n_kv_heads=n_kv + 1))
    assert B.lib().dllm_attention_workspace_size(more, n) == -2
    assert B.lib().dllm_attention(more, None, 0, None) == -2
    assert B.lib().dllm_last_error().decode() != ""


def test_attention_always_takes_what_the_header_says():
    """docs * n_kv_heads * ceil(max_q * group / 32) of 2^23."""
    n = ctypes.c_size_t()
    for dtype in (B.DLLM_F32, B.DLLM_BF16):
        for hd in (64, 128):
            for docs, n_kv, group, max_q in ((1, 1, 1, 1 << 28), (32768, 256, 1, 1), (32768, 128, 1, 33), (1, 64, 4096 // 64, 1 << 16),
                                             (3, 3, 2, 14913056), (65, 1, 1, 4129760), (8192, 8, 4, 1024), (511, 1, 1, 525312)):
                a = attn_args(dtype=dtype, head_dim=hd, docs=docs, n_heads=n_kv * group, n_kv_heads=n_kv, q_tokens=1 << 30, kv_tokens=4096,
                              max_q=max_q, max_kv=4096)
                assert docs * n_kv * -(-max_q * group // 32) <= 1 << 23
                assert B.lib().dllm_attention_workspace_size(a, n) == 0, (docs, n_kv, group, max_q, B.lib().dllm_last_error())


@pytest.mark.parametrize("gain,code", [(1e39, -1), (-1e300, -1), (math.nan, -1), (3e38, 0), (0.0, 0)])
def test_rotary_refuses_a_gain_that_float32_cannot_hold(gain, code):
    """The sines are multiplied by it in float32: infinity times a sine of 0 is no number."""
    assert rotary_rc(cfg=dict(gain=gain), Bn=1 if code else 0) == code
