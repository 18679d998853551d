"""dllm_shared_attention against the float64 oracle, document by document; the tolerance is that of dllm_attention
(test_gpu_attention.tolerance) over the prompt's keys and the document's own together."""
import math

import numpy as np
import pytest
import torch

from helpers import say, to_np
from oracle import operators as oo
from paper_2608_22646_amd import binding as B
from test_gpu_attention import randn, tolerance

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
HEADS = [(4, 4, 64), (4, 2, 128), (7, 1, 128), (28, 4, 128), (16, 2, 64)]


def starts(lens):
    return np.concatenate([[0], np.cumsum(lens)[:-1]]).astype(int) if len(lens) else np.zeros(0, int)


def run_and_check(Hq, Hkv, hd, dtype, q_lens, kv_lens, p_lens, of=None, block=0, q_pos=None, prefix=None, cap=0.0, slopes=None,
                  scale=None, seed=0, std=1.3, pad=3, mutate=None, check=True):
    """Packed documents and prompts (pad rows behind the last one); mutate(q, k, v, pk, pv) changes the inputs first."""
    T, S, P = sum(q_lens), sum(kv_lens), sum(p_lens)
    say(f"shared {Hq}/{Hkv}x{hd} {dtype} q{q_lens[:40]} kv{kv_lens[:40]} prompts {p_lens} of {of if of is None else of[:40]} block {block} pos "
        f"{q_pos} prefix {prefix} cap {cap} slopes {slopes is not None}")
    q, k, v, pk, pv = (randn((n + pad, H, hd), dtype, seed + i, std)
                       for i, (n, H) in enumerate([(T, Hq), (S, Hkv), (S, Hkv), (P, Hkv), (P, Hkv)]))
    if mutate:
        mutate(q, k, v, pk, pv)
    out = randn((T + pad, Hq, hd), dtype, seed + 5)
    behind = out[T:].clone()
    docs, prompts = B.Docs.packed(q_lens, kv_lens, q_pos, prefix), B.Prompts.packed(p_lens, of)
    sl = None if slopes is None else torch.tensor(slopes, dtype=F32, device="cuda")
    got = B.shared_attention(q, k, v, pk, pv, docs, prompts, block=block, cap=cap, slopes=sl, scale=scale, out=out)
    torch.cuda.synchronize()
    assert got is out and torch.equal(out[T:], behind)
    if check:
        verify(got, q, k, v, pk, pv, q_lens, kv_lens, p_lens, of, block, q_pos, prefix, cap, None if slopes is None else np.float32(slopes),
               scale, dtype)
    return got, (q, k, v, pk, pv, docs, prompts, sl)


def verify(got, q, k, v, pk, pv, q_lens, kv_lens, p_lens, of, block, q_pos, prefix, cap, slopes, scale, dtype):
    hd = q.shape[2]
    sc = float(np.float32(1 / math.sqrt(hd) if scale is None else scale))
    q0, k0, p0 = starts(q_lens), starts(kv_lens), starts(p_lens)
    f = lambda t: to_np(t, np.float64)  # noqa: E731
    for d, (a, b) in enumerate(zip(q_lens, kv_lens)):
        p = 0 if of is None else of[d]
        mine = slice(p0[p], p0[p] + p_lens[p]) if 0 <= p < len(p_lens) else slice(0, 0)
        with np.errstate(all="ignore"):
            ref, mass, top, dot = oo.shared_attention(
                f(q[q0[d]:q0[d] + a]), f(k[k0[d]:k0[d] + b]), f(v[k0[d]:k0[d] + b]), f(pk[mine]), f(pv[mine]),
                (b - a) if q_pos is None else q_pos[d], block, 0 if prefix is None else prefix[d], sc, cap, slopes)
            tol = tolerance(ref, mass, top, dot, b + mine.stop - mine.start, hd, dtype, sc, cap)
        g = f(got[q0[d]:q0[d] + a])
        fine = np.isfinite(ref)
        assert (np.isfinite(g) == fine).all(), f"document {d}: {(np.isfinite(g) != fine).sum()} elements finite on one side only"
        err = np.where(fine, np.abs(np.where(fine, g, 0) - np.where(fine, ref, 0)), 0)
        tol = np.where(fine, tol, 1)
        assert (err <= tol).all(), f"document {d}: {(err > tol).sum()} off, worst {(err / tol).max():.3g} tolerances"


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("q_lens,kv_lens,p_lens,of", [
    ([1], [1], [1], None), ([1, 1, 1], [5, 64, 65], [300], None), ([3, 0, 40, 1], [3, 7, 40, 33], [31, 129], [0, 0, 1, 1]),
    ([33, 64], [129, 64], [513], [0, -1]), ([5, 2, 1], [0, 2, 0], [64, 0], [0, 0, 1]), ([2, 2, 2, 2], [9, 9, 9, 9], [40, 50], [1, 0, 1, 0]),
])
def test_lengths(gpu_lib, heads, q_lens, kv_lens, p_lens, of, dtype):
    run_and_check(*heads, dtype, q_lens, kv_lens, p_lens, of, seed=sum(q_lens))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads", [(4, 4, 64), (6, 2, 128)])
@pytest.mark.parametrize("block,prefix", [(1, None), (1, [70, 0, 3]), (32, None), (5, [3, 100, 0])])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (20.0, False), (0.0, True), (5.0, True)])
def test_masks_caps_and_biases(gpu_lib, heads, block, prefix, cap, bias, dtype):
    slopes = [2.0 ** -(1 + h) for h in range(heads[0])] if bias else None
    run_and_check(*heads, dtype, [33, 7, 20], [70, 7, 150], [100, 37], [0, 1, 1], block, None, prefix, cap, slopes, seed=block)


# rows per document beyond 128 and many of them: a tile takes the prompt's keys and goes on with its own
MANY = [130 + 3 * d % 40 for d in range(33)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads", [(8, 8, 64), (8, 8, 128)])
@pytest.mark.parametrize("p_lens,of,block,cap,bias", [([1], None, 0, 0.0, False), ([70, 129, 0], [d % 4 - 1 for d in range(33)], 1, 0.0, True),
                                                      ([200], [0] * 20 + [-1] * 13, 32, 10.0, False)])
def test_many_rows(gpu_lib, heads, p_lens, of, block, cap, bias, dtype):
    slopes = [2.0 ** -(1 + h) for h in range(heads[0])] if bias else None
    run_and_check(*heads, dtype, MANY, [n + 5 if i % 3 else n for i, n in enumerate(MANY)], p_lens, of, block, None, None, cap, slopes)
