"""dllm_sample where a share of the mass falls exactly between two candidates.

Distinct logits give weights without a rational relation, so such a share lies between candidates that tie, in equal
parts of every level of ties.  What is expected follows from the counts alone: candidate i of n that tie stays while
i < top_p n, and a sum that equals u times the whole has not passed it."""
import math

import pytest
import torch

from helpers import say
from paper_2608_22646_amd import binding as B
from test_gpu_sample import check

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
SHARES = (0.25, 0.5, 0.75)


def column(v, n, dtype=F32):
    return torch.full((n,), v, dtype=dtype)


def tied(V, n, logits, dtype, others=-math.inf):
    """A row per logit: n candidates of it, spread over the vocabulary; their indices."""
    at = torch.arange(n) * V // n + V // (2 * n)
    x = torch.full((len(logits), V), others)
    x[:, at] = torch.tensor(logits)[:, None]
    return x.to(dtype), at


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V,n", [(700, 2), (700, 4), (3001, 10), (5000, 1000), (20000, 2), (40000, 64), (40000, 1000), (30000, 24000), (152064, 120000)])
def test_top_p_of_tied_candidates(gpu_lib, V, n, dtype):
    """The first ceil(top_p n) of n tied stay, at every logit (a constant added changes nothing), alone or by top-k."""
    say(f"sample shares {V} {n} {dtype}")
    logits = [-7.75, -3.0, -0.5, 0.0, 1.0, 1.5, 2.0, 3.0, 5.125, 8.0, 100.0] + [i / 64 for i in range(-500, 500, 61)]
    x, at = tied(V, n, logits, dtype)
    R = len(x)
    last = 1 - 2.0 ** -24
    cuda = x.cuda()
    for t in (1.0, 0.7):
        for p in SHARES:
            for k in (None, n, n + 5, max(1, n // 2)):
                kept = math.ceil(p * (n if k is None else min(k, n)))
                for u in (0.0, last):
                    token, _, prob = B.sample(cuda, column(u, R).cuda(), column(t, R).cuda(),
                                              None if k is None else column(k, R, torch.int32).cuda(), column(p, R).cuda())
                    want = int(at[kept - 1 if u else 0])
                    assert (token == want).all(), f"T {t} top_p {p} top_k {k} u {u}: {token.tolist()} and not {want}"
                    assert (prob.double() * kept - 1).abs().max() <= 2.0 ** -23


@pytest.mark.parametrize("t", [math.inf, 1e30])
def test_top_p_where_all_weigh_the_same(gpu_lib, t):
    """A temperature at which unlike logits weigh the same to 64 bits."""
    say(f"sample shares at temperature {t}")
    for V in (64, 20000):
        x = torch.randn((3, V), generator=torch.Generator().manual_seed(V))
        rank = torch.argsort(x, descending=True, stable=True)
        for p in SHARES:
            kept = math.ceil(p * V)
            token, _, prob = (c.cpu() for c in B.sample(x.cuda(), column(1.0, 3).cuda(), column(t, 3).cuda(), None, column(p, 3).cuda()))
            want = rank[:, :kept].amax(1)
            assert torch.equal(token.long(), want)
            assert (prob.double() * kept - 1).abs().max() <= 2.0 ** -23


@pytest.mark.parametrize("V", [700, 20000])
@pytest.mark.parametrize("below", [20.0, 30.0, 38.0])
def test_little_mass_beside_tied_candidates_counts(gpu_lib, V, below):
    """Two tie; others, with as little as 1e-14 of the mass in all, make half of the whole more than one of the two."""
    say(f"sample shares with little beside them {V} {below}")
    logits = [-7.75, 1.0, 1.5, 2.0, 3.0]
    x, at = tied(V, 2, logits, F32)
    x[:, V // 2 - 100:V // 2 + 100] = torch.tensor(logits)[:, None] - below
    u = column(1 - 2.0 ** -24, len(x))
    token, _, _ = check(x, u, top_p=column(0.5, len(x)))
    assert (token == int(at[1])).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V,n", [(700, 4), (5000, 1000), (40000, 64), (30000, 24000)])
def test_u_between_tied_candidates(gpu_lib, V, n, dtype):
    """u = i / n: i of the n tied have not passed it."""
    say(f"sample u between ties {V} {n} {dtype}")
    logits = [-7.75, 1.0, 1.5, 2.0, 3.0, 0.6]
    x, at = tied(V, n, logits, dtype)
    i = [i for i in range(n) if (i / n) == float(torch.tensor(i / n, dtype=F32))][:40]
    cuda = x.repeat_interleave(len(i), 0).contiguous().cuda()
    R = len(cuda)
    u = torch.tensor([a / n for a in i]).repeat(len(x)).cuda()
    want = at[torch.tensor(i).repeat(len(x))]
    for c in ({}, dict(temperature=column(0.7, R).cuda()), dict(min_p=column(0.5, R).cuda()), dict(top_p=column(1 - 2.0 ** -20, R).cuda()),
              dict(top_k=column(n, R, torch.int32).cuda()), dict(top_k=column(n + 1, R, torch.int32).cuda(), min_p=column(1.0, R).cuda())):
        token = B.sample(cuda, u, **c)[0].cpu().long()
        assert torch.equal(token, want), f"{list(c)}: {(token != want).sum()} of {R} rows"


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [512, 8192, 65536, 131072])
def test_u_between_repeated_levels(gpu_lib, V, dtype):
    """The same eight logits over and over: the first u V of them weigh u times the whole exactly."""
    say(f"sample u between levels {V} {dtype}")
    g = torch.Generator().manual_seed(V)
    levels = (torch.randn((6, 8), generator=g) * 2.0).to(dtype)
    x = levels.repeat(1, V // 8)
    u = torch.arange(0, 64) / 64
    cuda = x.repeat_interleave(len(u), 0).contiguous().cuda()
    R = len(cuda)
    want = (u * V).long().repeat(6)
    for c in ({}, dict(temperature=column(0.7, R).cuda()), dict(min_p=column(1e-9, R).cuda()),
              dict(min_p=column(1e-9, R).cuda(), temperature=column(1.3, R).cuda())):
        token = B.sample(cuda, u.repeat(6).cuda(), **c)[0].cpu().long()
        assert torch.equal(token, want), f"{list(c)}: {(token != want).sum()} of {R} rows"


@pytest.mark.parametrize("V", [512, 8192, 65536])
@pytest.mark.parametrize("kept", [1, 3, 4, 7])
def test_u_between_repeated_levels_that_top_k_keeps(gpu_lib, V, kept):
    """The same, of which top-k keeps the highest levels whole: in classes of their own, or with one that goes in theirs."""
    say(f"sample u between kept levels {V} {kept}")
    levels = torch.tensor([[0.5, -1.25, 2.0, 1.99, -3.0, 0.49, 1.0, -1.26], [3.0, -4.0, 5.0, 1.0, 7.0, 2.0, -9.0, 0.0]])
    u = torch.arange(0, 64) / 64
    for row in levels:
        rank = torch.argsort(torch.argsort(row, descending=True))
        R = len(u)
        members = (rank.repeat(V // 8) < kept).nonzero()[:, 0]
        want = members[(u * len(members)).long()]
        cuda = row.repeat(V // 8).expand(R, V).contiguous().cuda()
        k = column(V // 8 * kept, R, torch.int32).cuda()
        for t in (1.0, 0.7):
            token = B.sample(cuda, u.cuda(), column(t, R).cuda(), k)[0].cpu().long()
            assert torch.equal(token, want), f"T {t}: {(token != want).sum()} of {R} rows"
