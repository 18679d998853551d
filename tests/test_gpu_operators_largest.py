"""The stand-alone operators at sizes near the ends of what the header allows."""
import numpy as np
import pytest
import torch

from helpers import say, to_np
from oracle import operators as oo
from paper_2608_22646_amd import binding as B
from test_gpu_attention import randn, verify
from test_gpu_sample import check, controls, uniform

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_the_largest_vocabulary(gpu_lib, dtype):
    """2^22 logits a row: 512 chunks, indices of 22 bits; also one less."""
    for V in (1 << 22, (1 << 22) - 1):
        for which in ("t", "tkpm"):
            say(f"sample vocabulary {V} {which} {dtype}")
            g = torch.Generator().manual_seed(V)
            x = (torch.randn((2, V), generator=g) * 1.2).to(dtype)
            x[1, -1] = 30.0
            check(x, uniform(2, V + 1), mask_id=7, **controls(2, V, V, which))


def test_very_many_rows(gpu_lib):
    """400000 rows of three logits: the row sampled is the row given."""
    say("sample 400000 rows")
    R = 400_000
    g = torch.Generator().manual_seed(1)
    x, u = torch.randn((R, 3), generator=g), torch.rand(R, generator=g)
    p = torch.softmax(x.double(), 1)
    for c in ({}, dict(top_k=torch.full((R,), 2, dtype=torch.int32))):
        q = p if not c else torch.where(p > p.amin(1, keepdim=True), p, 0.0)
        s = torch.cumsum(q, 1)
        want = (s <= u.double()[:, None] * s[:, -1:]).sum(1)
        near = ((s - u.double()[:, None] * s[:, -1:]).abs() < 1e-11).any(1)
        token, conf, _ = (t.cpu() for t in B.sample(x.cuda(), u.cuda(), **{k: v.cuda() for k, v in c.items()}))
        wrong = (token != want) & ~near
        assert not wrong.any(), int(wrong.sum())
        assert (conf.double() / p.gather(1, token.long()[:, None])[:, 0] - 1).abs().max() <= 2.0 ** -19


def test_very_many_documents(gpu_lib):
    """65535 documents, the most of a call, of one query and up to two keys."""
    say("attention 65535 documents")
    n = 65535
    g = torch.Generator().manual_seed(2)
    kv = torch.randint(0, 3, (n,), generator=g).tolist()
    q, k, v = randn((n, 2, 64), BF16, 1), randn((sum(kv), 1, 64), BF16, 2), randn((sum(kv), 1, 64), BF16, 3)
    docs = B.Docs.packed([1] * n, kv)
    got = B.attention(q, k, v, docs)
    starts = docs.kv_start.tolist()
    empty = torch.tensor([m == 0 for m in kv])
    assert torch.count_nonzero(got.cpu()[empty]) == 0
    for d in (0, 1, 2, 255, 256, 257, 32767, 32768, 65533, 65534):
        verify(got[d:d + 1], q[d:d + 1], k[starts[d]:starts[d] + kv[d]], v[starts[d]:starts[d] + kv[d]], [1], [kv[d]], 0, None, None, 0.0,
               None, None, BF16)
    one = [d for d in range(n) if kv[d] == 1]
    assert torch.equal(got[one], v[[starts[d] for d in one]].expand(-1, 2, -1))     # one key: its value


def test_many_tokens_of_one_head(gpu_lib):
    """Two million tokens, more than there are workgroups to launch."""
    say("rotary two million tokens")
    n = 2_200_000
    x = torch.randn((1, n, 1, 8), generator=torch.Generator().manual_seed(3)).cuda()
    got, _ = B.rotary(B.Rotary(8), x, pos0=11)
    for a in (0, 1 << 20, n - 5):
        ref = oo.rotary(to_np(x[:, a:a + 5], np.float64), np.arange(a + 11, a + 16)[None], oo.rotary_rates(8))
        assert np.abs(to_np(got[:, a:a + 5], np.float64) - ref).max() <= 12 * 2.0 ** -24 * 2 * float(x.abs().max())
