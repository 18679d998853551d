"""dllm_attention where values are no numbers, scores are far from zero, and caps meet their two forms;
tolerances as in test_gpu_attention."""
import math

import pytest
import torch

from helpers import say
from test_gpu_attention import run_and_check

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
