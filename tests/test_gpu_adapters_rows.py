"""dllm_adapters: workspaces of the size that the binding tells, every count of rows of two groups of neighbours, and what a
row's result owes to the rows beside it.  Tolerances are test_gpu_adapters'."""
import pytest
import torch

from helpers import say
from paper_2608_22646_amd import binding as B
from test_gpu_adapters import BF16, F32, inputs, ints, run, verify

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [20, 300])
@pytest.mark.parametrize("kind", [BF16, F32])
def test_a_workspace_of_the_size_that_is_told(gpu_lib, M, kind):
    """bf16 operands, no base, an output of either type; ranks of more than one step."""
    say(f"{M} rows to {kind}")
    x, out, A, Bm = inputs(M, 64, (80,), 3, 40, BF16, kind)
    which = [m % 4 - 1 for m in range(M)]
    need = B.adapters_workspace_size(x, None, A, Bm, out=out)
    got = B.adapters(x, None, A, Bm, ints(which), out=out, ws=B.device_buffer(need))
    verify(got, x, None, A, Bm, which, None, None, (80,))
    with pytest.raises(B.DllmError):
        B.adapters(x, None, A, Bm, ints(which), out=out, ws=B.device_buffer(need)[:need - 256])
