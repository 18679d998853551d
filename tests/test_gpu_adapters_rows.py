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


@pytest.mark.parametrize("M", [33, 40, 47, 63, 64])
def test_groups_of_neighbours_that_are_not_full(gpu_lib, M):
    """Two groups of 32 rows, the second short: rows that are not there take no part, whatever the adapters."""
    for which in ([0] * M, [m % 6 - 1 for m in range(M)], [-1] * (M - 1) + [2]):
        run(M, 256, (136, 24), 5, 16, BF16, BF16, which, seed=M)


@pytest.mark.parametrize("kind", [BF16, F32])
@pytest.mark.parametrize("M", [30, 64, 100, 1500])
def test_other_rows_of_as_many(gpu_lib, M, kind):
    """Calls of the same sizes: a row's bits stay, whatever the others hold, wherever it stands, whoever shares its adapter."""
    x, base, A, Bm = inputs(M, 2048, (264,), 6, 40, BF16, kind)
    which = [(m * 5) % 7 - 1 for m in range(M)]
    one = B.adapters(x, base, A, Bm, ints(which))
    mine, a = 8, which[8]
    assert a >= 0
    for to, others in ((0, a), (M - 1, (a + 1) % 6), (M // 2, -1)):
        x2, base2, _, _ = inputs(M, 2048, (264,), 6, 40, BF16, kind, seed=50)
        x2[to], base2[to] = x[mine], base[mine]
        w2 = [others] * M
        w2[to] = a
        assert torch.equal(B.adapters(x2, base2, A, Bm, ints(w2))[to], one[mine])


@pytest.mark.parametrize("dtype,kind", [(F32, F32), (BF16, BF16), (BF16, F32)])
def test_a_row_alone_and_among_others(gpu_lib, dtype, kind):
    """d_in in as many shares as there are, and in fewer as rows grow: each within the bounds of one float32 sum."""
    n, R, K = 5, 40, 4096
    x, base, A, Bm = inputs(8448, K, (136,), n, R, dtype, kind)
    which = [(m * 3) % n for m in range(8448)]
    for M in (1, 64, 300, 2000, 8448):
        got = B.adapters(x[:M], base[:M], A, Bm, ints(which[:M]))
        verify(got[:3], x[:min(M, 3)], base[:min(M, 3)], A, Bm, which[:min(M, 3)], None, None, (136,))
