"""dllm_adapters rejects invalid arguments on the host, before any device work (CPU only: no address handed over here
is real), and its binding refuses operands that do not belong together."""
import ctypes

import pytest
import torch

from paper_2608_22646_amd import binding as B

A = 0x10000  # a made-up, aligned address


def view(data=A, b=0, l=64, h=0):
    return B.View(data, b, l, h)


def args(**kw):
    a = dict(dtype=B.DLLM_BF16, out_dtype=B.DLLM_BF16, rows=4, d_in=64, d_out=64, adapters=2, rank=8, slices=1,
             slice_end=(64, 0, 0, 0), x=view(), a=view(b=512), b=view(b=512, l=8), base=view(), out=view(), which=A)
    a.update(kw)
    a["slice_end"] = (ctypes.c_int32 * 4)(*a["slice_end"])
    return B.AdapterArgs(**a)


def call(a, ws=A, n=1 << 40):
    return B.lib().dllm_adapters(a, ws, n, None)


REFUSED = [
    (dict(dtype=2), -1), (dict(out_dtype=2), -1), (dict(dtype=B.DLLM_F32, out_dtype=B.DLLM_BF16), -1), (dict(rows=-1), -2),
    (dict(rows=(1 << 22) + 1), -2), (dict(d_in=0), -2), (dict(d_in=(1 << 20) + 1), -2), (dict(d_out=0), -2),
    (dict(d_out=(1 << 20) + 1), -2), (dict(adapters=-1), -2), (dict(adapters=4096), -2), (dict(rank=0), -2), (dict(rank=257), -2),
    (dict(slices=0), -2), (dict(slices=5), -2), (dict(slice_end=(63, 0, 0, 0)), -2), (dict(slices=2, slice_end=(64, 64, 0, 0)), -2),
    (dict(slices=2, slice_end=(0, 64, 0, 0)), -2), (dict(slices=3, slice_end=(40, 30, 64, 0)), -2), (dict(slices=2, slice_end=(32, 65, 0, 0)), -2),
]


@pytest.mark.parametrize("kw,code", REFUSED + [
    (dict(x=view(0)), -1), (dict(a=view(0)), -1), (dict(b=view(0)), -1), (dict(out=view(0)), -1), (dict(which=None), -1),
    (dict(x=view(l=-64)), -2), (dict(a=view(b=-1)), -2), (dict(base=view(l=-64)), -2), (dict(out=view(l=63)), -2),
    (dict(base=view(l=128)), -2),
])
def test_refuses(kw, code):
    assert call(args(**kw)) == code, B.lib().dllm_last_error()
    assert B.lib().dllm_last_error().decode() != ""


@pytest.mark.parametrize("kw,code", REFUSED)
def test_workspace_size_refuses_the_same_sizes(kw, code):
    n = ctypes.c_size_t(7)
    assert B.lib().dllm_adapters_workspace_size(args(**kw), n) == code


def test_workspace():
    n = ctypes.c_size_t()
    assert B.lib().dllm_adapters_workspace_size(None, n) == -1
    assert B.lib().dllm_adapters_workspace_size(args(), None) == -1
    assert B.lib().dllm_adapters_workspace_size(args(rows=0), n) == 0 and n.value == 0
    assert call(args(rows=0), None, 0) == 0
    assert call(None) == -1
    for kw in (dict(), dict(rows=100)):
        assert B.lib().dllm_adapters_workspace_size(args(**kw), n) == 0 and n.value > 0
        assert call(args(**kw), A, n.value - 1) == -4
        assert call(args(**kw), None, n.value) == -1
        assert call(args(**kw), A + 128, n.value) == -1


def test_binding_refuses_the_wrong_tensors():
    x, y, a, b, w = torch.zeros(4, 64), torch.zeros(4, 32), torch.zeros(2, 8, 64), torch.zeros(2, 32, 8), torch.zeros(4, dtype=torch.int32)
    for bad in (dict(x=x[0]), dict(A=a[0]), dict(B=b[0]), dict()):  # the last: tensors that are not on the GPU
        with pytest.raises(B.DllmError):
            B.adapters(**{**dict(x=x, base=y, A=a, B=b, which=w), **bad})


@pytest.mark.parametrize("kw,code", [
    (dict(x=torch.zeros(4, 64).half()), -1), (dict(base=torch.zeros(4, 31)), -2), (dict(base=torch.zeros(4, 32).half()), -1),
    (dict(A=torch.zeros(2, 8, 63)), -2), (dict(A=torch.zeros(3, 8, 64)), -2), (dict(A=torch.zeros(2, 2, 8, 64)), -2),
    (dict(B=torch.zeros(2, 32, 8).bfloat16()), -1), (dict(slices=(16, 16)), -2), (dict(slices=()), -2),
    (dict(A=torch.zeros(2, 5, 8, 64), slices=(8, 8, 8, 4, 4)), -2), (dict(which=torch.zeros(4, dtype=torch.int64)), -1),
    (dict(which=torch.zeros(5, dtype=torch.int32)), -2), (dict(ranks=torch.zeros(2)), -1), (dict(scales=torch.zeros(3)), -2),
    (dict(x=torch.zeros(64, 4).t()), -2), (dict(out=torch.zeros(4, 32).bfloat16()), -1),
])
def test_marshalling_refuses(kw, code):
    a = dict(x=torch.zeros(4, 64), base=torch.zeros(4, 32), A=torch.zeros(2, 8, 64), B=torch.zeros(2, 32, 8),
             which=torch.zeros(4, dtype=torch.int32), ranks=None, scales=None, slices=None, out=None)
    with pytest.raises(B.DllmError) as e:
        B._adapter_args(**{**a, **kw})
    assert e.value.code == code


@pytest.mark.parametrize("rows,code", [(1 << 22, -2), ((1 << 22) - 32 * 7, -2), ((1 << 22) - 32 * 11, 0), (1 << 10, 0)])
def test_refuses_more_workgroups_than_a_launch_has(rows, code):
    """4 x 16 blocks of ranks of rows / 32 + 3 tiles, those in eights: below 2^23 workgroups of 512 threads, or refused
    (2^17 - 7 + 3 tiles are 2^17 in eights, 2^17 - 11 + 3 are 2^17 - 8)."""
    n = ctypes.c_size_t()
    a = args(rows=rows, d_in=1, slices=4, slice_end=(16, 32, 48, 64), rank=256, x=view(l=1), a=view(b=1024, l=1, h=256), b=view(b=1 << 14, l=256))
    assert B.lib().dllm_adapters_workspace_size(a, n) == code
    if code:
        assert call(a) == code


def test_refuses_more_columns_than_a_launch_has():
    n = ctypes.c_size_t()
    wide = dict(d_out=1 << 20, slice_end=(1 << 20, 0, 0, 0), out=view(l=1 << 20), base=view(l=1 << 20), b=view(b=1 << 23, l=8))
    assert B.lib().dllm_adapters_workspace_size(args(rows=1 << 19, **wide), n) == -2 and call(args(rows=1 << 19, **wide)) == -2
    assert B.lib().dllm_adapters_workspace_size(args(rows=1 << 18, **wide), n) == 0
