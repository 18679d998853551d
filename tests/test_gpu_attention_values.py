"""dllm_attention where values are no numbers, scores are far from zero, and caps meet their two forms;
tolerances as in test_gpu_attention."""
import math

import pytest
import torch

from helpers import say
from paper_2608_22646_amd import binding as B
from test_gpu_attention import randn, run_and_check, verify

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads", [(4, 4, 64), (4, 2, 128)])
@pytest.mark.parametrize("n,kv,q_pos", [(3, 80, 40), (60, 200, 100), (200, 400, 150)])
def test_broken_values_reach_their_own_dimension(gpu_lib, n, kv, q_pos, heads, dtype):
    """Every dimension, even and odd, in a key that some queries see, beside keys that none sees and are all broken;
    one, two and four row groups a workgroup."""
    say(f"attention broken values {heads} {n} {kv} {dtype}")
    hd = heads[2]

    def at(key, dims, bad):
        def mutate(q, k, v):
            k[q_pos + n:kv], v[q_pos + n:kv] = bad, bad
            v[key, :, dims] = bad
        return mutate
    for key in (q_pos + 1, q_pos + n // 2, q_pos + n - 1):
        for dims, bad in ((slice(0, hd, 2), math.nan), (slice(1, hd, 2), math.inf), (slice(2, hd, 4), -math.inf), (slice(hd - 1, hd), math.nan)):
            got = run_and_check(*heads, dtype, [n], [kv], block=1, q_pos=[q_pos], seed=key, mutate=at(key, dims, bad))
            assert torch.isfinite(got[:key - q_pos].float()).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("share", [0.2, 0.27, 0.285, 0.39, 0.41, 0.59, 0.61, 2.0])
def test_caps_on_both_sides_of_their_forms(gpu_lib, share, dtype):
    """Caps of which the largest score is a given share: small ones go by a series, large ones by exponentials."""
    say(f"attention cap forms {share} {dtype}")
    top = []

    def measure(q, k, v):
        s = torch.einsum("thd,shd->hts", q.cpu().double(), k.cpu().double().repeat_interleave(2, 1)) / 8
        top.append(float(s.abs().max()))
    for n, kv in ((3, 90), (300, 300)):
        run_and_check(4, 2, 64, dtype, [n], [kv], seed=kv, mutate=measure, cap=1e30, acts_as=0.0)
        run_and_check(4, 2, 64, dtype, [n], [kv], seed=kv, cap=top[-1] / share)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,kv", [(1, 70), (3, 5000), (150, 300)])
def test_biases_far_from_every_key(gpu_lib, n, kv, dtype):
    """Distances beyond what float32 counts: a query at or behind the last key it sees (or before the first) gives
    what one at that key does, since all its scores differ from that one's by the same amount."""
    say(f"attention far biases {n} {kv} {dtype}")
    slopes = [0.5, 0.25, 2.0 ** -8, -0.125]
    q, k, v = randn((n, 4, 64), dtype, 1, 1.3), randn((kv, 2, 64), dtype, 2, 1.3), randn((kv, 2, 64), dtype, 3, 1.3)
    sl = torch.tensor(slopes, dtype=F32, device="cuda")
    for pos in (kv + 3, 1 << 20, (1 << 24) + 1, (1 << 31) - 1, -n, -(1 << 22), -(1 << 31)):
        for block in (0, 1):
            got = B.attention(q, k, v, B.Docs.packed([n], [kv], [pos]), block=block, slopes=sl)
            if block and pos < 0:
                assert torch.count_nonzero(got) == 0
                continue
            for t in range(0, n, 37):
                verify(got[t:t + 1], q[t:t + 1], k, v, [1], [kv], 0, [kv - 1 if pos > 0 else 0], None, 0.0, sl.cpu().numpy(), 0.125, dtype)


def test_infinite_slopes(gpu_lib):
    """An infinite slope leaves a query no score above -inf, or at its own position none that is a number."""
    q, k, v = randn((2, 2, 64), F32, 1), randn((9, 2, 64), F32, 2), randn((9, 2, 64), F32, 3)
    sl = torch.tensor([math.inf, 1.0], device="cuda")
    for pos, nan in ((9, False), (100, False), (-2, False), (3, True)):
        got = B.attention(q, k, v, B.Docs.packed([2], [9], [pos]), slopes=sl)
        assert torch.isfinite(got[:, 1]).all() and torch.isnan(got[:, 0]).all() == nan and (nan or torch.count_nonzero(got[:, 0]) == 0)
