"""One layer's attention half of a batch of requests, as a serving program runs it: a shared projection with each
request's adapter on queries, keys and values, rotary positions behind the request's prompt, attention behind prompts
held once, the output projection with its adapters into the float32 residual.  Each operator is checked against the
oracle on what the one before it left; the products of the shared projections, which the program computes itself, are
torch's."""
import numpy as np
import pytest
import torch

from helpers import say, to_np
from oracle import operators as oo
from paper_2608_22646_amd import binding as B
from test_gpu_adapters import ints, randn, verify as verify_adapters
from test_gpu_rotary import check as check_rotary
from test_gpu_shared import starts, verify as verify_shared

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
D, HQ, HKV, HD, R = 512, 4, 2, 128, 16
WIDTHS = (HQ * HD, HKV * HD, HKV * HD)
PROMPTS = [300, 77]                    # keys of each prompt
OF = [0, 0, 0, 1, 1, -1]               # the prompt that a request continues
ADAPTER = [2, 0, -1, 2, 1, 0]          # the adapter that it brings


class Batch:
    """Requests whose keys grow step by step, each in its slab, behind prompts packed in one."""

    def __init__(self, dtype, seed=0):
        self.dtype, self.n = dtype, len(OF)
        self.w_qkv, self.w_o = randn((sum(WIDTHS), D), dtype, seed, D ** -0.5), randn((D, HQ * HD), dtype, seed + 1, D ** -0.5)
        self.a_qkv, self.b_qkv = randn((3, 3, R, D), dtype, seed + 2, D ** -0.5), randn((3, sum(WIDTHS), R), dtype, seed + 3, 0.2)
        self.a_o, self.b_o = randn((3, R, HQ * HD), dtype, seed + 4, D ** -0.5), randn((3, D, R), dtype, seed + 5, 0.2)
        self.ranks, self.scales = ints([R, 5, 11]), torch.tensor([1.0, 2.0, 0.5], device="cuda")
        self.pk, self.pv = randn((sum(PROMPTS), HKV, HD), dtype, seed + 6), randn((sum(PROMPTS), HKV, HD), dtype, seed + 7)
        self.k, self.v = (torch.full((self.n, 64, HKV, HD), float("nan"), dtype=dtype, device="cuda") for _ in "kv")
        self.rope = B.Rotary(HD, base=1e4)
        self.prompts = B.Prompts.packed(PROMPTS, OF)
        self.before = [PROMPTS[p] if p >= 0 else 0 for p in OF]
        self.at = 0

    def step(self, x, h, check=True):
        """x [n, T, D] the normed rows of T new tokens of each request, h [n, T, D] the float32 residual, updated."""
        n, T, _ = x.shape
        rows, which = x.reshape(n * T, D), ints(np.repeat(ADAPTER, T))
        base = rows @ self.w_qkv.T
        qkv = B.adapters(rows, base, self.a_qkv, self.b_qkv, which, ranks=self.ranks, scales=self.scales, slices=WIDTHS)
        qkv = qkv.view(n, T, HQ + 2 * HKV, HD)
        new = slice(self.at, self.at + T)
        pos = torch.tensor(self.before, dtype=torch.int32, device="cuda")[:, None] + torch.arange(self.at, self.at + T, dtype=torch.int32, device="cuda")
        q, k = B.rotary(self.rope, qkv[:, :, :HQ], qkv[:, :, HQ:HQ + HKV], pos=pos.contiguous(), k_out=self.k[:, new])
        self.v[:, new] = qkv[:, :, HQ + HKV:]
        docs = B.Docs(kv_len=ints([self.at + T] * n))
        out = B.shared_attention(q, self.k, self.v, self.pk, self.pv, docs, self.prompts, block=1)
        flat = out.reshape(n * T, HQ * HD)
        o_base = (flat.float() @ self.w_o.float().T).add_(h.view(n * T, D))
        B.adapters(flat, o_base, self.a_o, self.b_o, which, ranks=self.ranks, scales=self.scales, out=h.view(n * T, D))
        self.at += T
        if check:
            adapter, ranks, scales = np.repeat(ADAPTER, T).tolist(), self.ranks.tolist(), self.scales.tolist()
            verify_adapters(qkv.view(n * T, -1), rows, base, self.a_qkv, self.b_qkv, adapter, ranks, scales, WIDTHS)
            for got, x_ in ((q, qkv[:, :, :HQ]), (self.k[:, new], qkv[:, :, HQ:HQ + HKV])):
                check_rotary(got, x_, pos.cpu().numpy(), dict(rot_dim=HD), self.dtype, False)
            p0 = starts(PROMPTS)
            for d in range(n):
                mine = slice(p0[OF[d]], p0[OF[d]] + PROMPTS[OF[d]]) if OF[d] >= 0 else slice(0, 0)
                verify_shared(out[d], q[d], self.k[d, :self.at], self.v[d, :self.at], self.pk[mine], self.pv[mine], [T], [self.at],
                              [mine.stop - mine.start], [0 if OF[d] >= 0 else -1], 1, None, None, 0.0, None, None, self.dtype)
            verify_adapters(h.view(n * T, D), flat, o_base, self.a_o[:, None], self.b_o, adapter, ranks, scales, (D,))
        return out


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_requests_behind_prompts_with_adapters(gpu_lib, dtype):
    b = Batch(dtype)
    for i, T in enumerate((7, 1, 1, 3, 33, 1)):
        say(f"requests: {T} tokens at {b.at}")
        b.step(randn((b.n, T, D), dtype, 50 + i), randn((b.n, T, D), F32, 80 + i))


def test_a_captured_step(gpu_lib):
    """A step of single tokens in a graph: replays on other rows give what eager calls give, with adapters of the
    requests changed in between."""
    b = Batch(BF16, seed=10)
    b.step(randn((b.n, 9, D), BF16, 1), randn((b.n, 9, D), F32, 2), check=False)
    x, h = randn((b.n, 1, D), BF16, 3), randn((b.n, 1, D), F32, 4)
    which, docs = ints(ADAPTER), B.Docs(kv_len=ints([10] * b.n))
    pos = (torch.tensor(b.before, dtype=torch.int32, device="cuda") + 9)[:, None].contiguous()

    def step():
        rows = x.view(b.n, D)
        qkv = B.adapters(rows, rows @ b.w_qkv.T, b.a_qkv, b.b_qkv, which, ranks=b.ranks, scales=b.scales, slices=WIDTHS).view(b.n, 1, -1, HD)
        q, _ = B.rotary(b.rope, qkv[:, :, :HQ], qkv[:, :, HQ:HQ + HKV], pos=pos, k_out=b.k[:, 9:10])
        b.v[:, 9:10] = qkv[:, :, HQ + HKV:]
        out = B.shared_attention(q, b.k, b.v, b.pk, b.pv, docs, b.prompts, block=1).view(b.n, HQ * HD)
        return B.adapters(out, h.view(b.n, D), b.a_o, b.b_o, which, ranks=b.ranks, scales=b.scales)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            got = step()
    for i in range(4):
        x.copy_(randn(x.shape, BF16, 30 + i))
        which.copy_(ints(np.roll(ADAPTER, i)))
        torch.cuda.synchronize()
        g.replay()
        side.synchronize()
        torch.cuda.synchronize()
        mine = got.clone()
        assert torch.equal(mine, step())
