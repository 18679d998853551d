"""The sum behind dllm_sample's conf: many weights that are small beside the first.

One logit in sixteen is 0, the others x, whose weight e^x is a little less than half a step above a multiple of
2^-23: a float32 sum beside 1 loses that part of each.  A float32 weight is off by at most 2^-19 of itself (the difference
to the largest logit, its product with log2 e, below 25, and the exponential), all small ones together make less than 2^-12
of the sum, and conf is rounded once: 2^-31 + 2^-24, within 2^-23."""
import math

import numpy as np
import pytest
import torch

from helpers import say
from oracle import operators as oo
from paper_2608_22646_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [3000, 8192, 20000])
@pytest.mark.parametrize("which", ["plain", "greedy", "top_p"])
def test_many_small_weights(gpu_lib, V, which):
    say(f"sample conf {V} {which}")
    v = torch.arange(V)
    rows = [0.49, 5.49, 40.47, 100.45]
    x = torch.stack([torch.where((v % 8192 < 2048) & (v % 4 == 0), 0.0, math.log(m * 2.0 ** -23)) for m in rows])
    x = torch.cat([x, x.roll(5, 1), x + 3.0])
    R = len(x)
    c = {"plain": {}, "greedy": dict(temperature=torch.zeros(R)), "top_p": dict(top_p=torch.full((R,), 0.9))}[which]
    token, conf, _ = (t.cpu() for t in B.sample(x.cuda(), torch.full((R,), 0.3, device="cuda"), **{k: v.cuda() for k, v in c.items()}))
    for r in range(R):
        z = x[r].numpy().astype(np.float64)
        e = np.exp(z - z.max())
        want = e[token[r]] / math.fsum(e)
        assert abs(float(conf[r]) / want - 1) <= 2.0 ** -23, f"row {r}: {float(conf[r])} and not {want}"
        assert oo.sample(z, 0.3, 0.0 if which == "greedy" else 1.0, 0, 0.9 if which == "top_p" else 1.0)[0] == token[r]
