"""The size of workspace that the binding tells for a call of adapters() is the one that the call needs, for each type of
its output, with a base and without (CPU only)."""
import ctypes

import pytest
import torch

from paper_2608_22646_amd import binding as B

F32, BF16 = torch.float32, torch.bfloat16


def needed(x, base, A, Bm, out):
    """What dllm_adapters asks for: the query of the call's own arguments."""
    n = ctypes.c_size_t()
    a, _ = B._adapter_args(x, base, A, Bm, None, None, None, None, out)
    assert B.lib().dllm_adapters_workspace_size(a, n) == 0
    return n.value


@pytest.mark.parametrize("M", [1, 40, 100, 5000])
@pytest.mark.parametrize("R", [8, 40, 200])
def test_size_by_the_type_of_out(M, R):
    x, A, Bm = torch.zeros(M, 64, dtype=BF16), torch.zeros(2, R, 64, dtype=BF16), torch.zeros(2, 72, R, dtype=BF16)
    size = {}
    for kind in (BF16, F32):
        out = torch.zeros(M, 72, dtype=kind)
        size[kind] = B.adapters_workspace_size(x, None, A, Bm, out=out)
        assert size[kind] == needed(x, None, A, Bm, out) == B.adapters_workspace_size(x, out, A, Bm) == B.adapters_workspace_size(x, out, A, Bm, out=out)
    assert B.adapters_workspace_size(x, None, A, Bm) == size[BF16] == needed(x, None, A, Bm, None)
    # ranks of more than a step: three pieces of 16 bits of an inner product are kept for a float32 output, else two
    assert size[F32] > size[BF16] if R > 32 else size[F32] == size[BF16]


def test_refuses_an_out_of_another_type_than_base():
    x, A, Bm = torch.zeros(4, 64, dtype=BF16), torch.zeros(2, 8, 64, dtype=BF16), torch.zeros(2, 72, 8, dtype=BF16)
    with pytest.raises(B.DllmError):
        B.adapters_workspace_size(x, torch.zeros(4, 72, dtype=BF16), A, Bm, out=torch.zeros(4, 72))
    with pytest.raises(B.DllmError):
        B.adapters_workspace_size(x, None, A, Bm, out=torch.zeros(4, 72, dtype=torch.float16))
    with pytest.raises(B.DllmError):
        B.adapters_workspace_size(x, None, A, Bm, out=torch.zeros(4, 71))
