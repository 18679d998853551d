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
REACH = 0


@pytest.fixture(autouse=True, params=[0, 20000], ids=["short", "long"])
def reach(request, monkeypatch):
    """Calls that are told of prompts no longer than they are, which row tiles may read with their own keys in one go, and
    of far longer ones, whose keys are dealt as units: rows of no number behind the prompts make the slabs as long."""
    monkeypatch.setitem(globals(), "REACH", request.param)


HEADS = [(4, 4, 64), (4, 2, 128), (7, 1, 128), (28, 4, 128), (16, 2, 64)]


def starts(lens):
    return np.concatenate([[0], np.cumsum(lens)[:-1]]).astype(int) if len(lens) else np.zeros(0, int)


def longer(t, rows):
    """Rows of NaN behind the prompts of a slab ([.., P, Hkv, hd])."""
    return torch.cat([t, t.new_full((*t.shape[:-3], rows, *t.shape[-2:]), float("nan"))], dim=-3) if rows else t


def run_and_check(Hq, Hkv, hd, dtype, q_lens, kv_lens, p_lens, of=None, block=0, q_pos=None, prefix=None, cap=0.0, slopes=None,
                  scale=None, seed=0, std=1.3, pad=3, mutate=None, check=True, reach=None):
    """Packed documents and prompts (pad rows behind the last one); mutate(q, k, v, pk, pv) changes the inputs first."""
    reach = REACH if reach is None else reach
    T, S, P = sum(q_lens), sum(kv_lens), sum(p_lens)
    say(f"shared {Hq}/{Hkv}x{hd} {dtype} q{q_lens[:40]} kv{kv_lens[:40]} prompts {p_lens} of {of if of is None else of[:40]} block {block} pos "
        f"{q_pos} prefix {prefix} cap {cap} slopes {slopes is not None}")
    q, k, v, pk, pv = (randn((n + pad, H, hd), dtype, seed + i, std)
                       for i, (n, H) in enumerate([(T, Hq), (S, Hkv), (S, Hkv), (P, Hkv), (P, Hkv)]))
    pk, pv = longer(pk, reach), longer(pv, reach)
    if mutate:
        mutate(q, k, v, pk, pv)
    out = randn((T + pad, Hq, hd), dtype, seed + 5)
    behind = out[T:].clone()
    docs, prompts = B.Docs.packed(q_lens, kv_lens, q_pos, prefix), B.Prompts.packed(p_lens, of)
    prompts.max = max(prompts.max, reach)
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


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("q_lens,kv_lens,p_lens,of", [([150, 10], [600, 300], [1500], None), ([1, 64, 65, 33], [1, 64, 700, 33], [2000, 129], [0, 1, 1, 0]),
                                                      ([300], [300], [1], None)])
def test_long_prompts_and_tiles_of_many_rows(gpu_lib, q_lens, kv_lens, p_lens, of, dtype):
    run_and_check(4, 2, 128, dtype, q_lens, kv_lens, p_lens, of, block=32, slopes=[0.5, 0.1, 0.01, 0.001], seed=7)


@pytest.mark.parametrize("n,dtype", [(64, F32), (65, BF16), (65, F32), (257, BF16), (1100, BF16), (2500, BF16)])
def test_many_documents(gpu_lib, n, dtype):
    """Planned by each workgroup, by one of 256 threads, of 1024, and in several goes; empty documents among them."""
    rng = np.random.default_rng(n)
    q, kv = rng.integers(0, 4, n).tolist(), rng.integers(0, 40, n).tolist()
    of = np.sort(rng.integers(-1, 4, n)).tolist()
    run_and_check(4, 2, 64, dtype, q, kv, [300, 0, 65, 1000], of, block=1, slopes=[0.5, 0.25, 0.1, 0.01])


@pytest.mark.parametrize("n", [64, 130])
def test_more_units_than_workgroups(gpu_lib, n):
    """Documents that change between two prompts each time: as many stacks as documents."""
    run_and_check(32, 32, 64, BF16, [1] * n, [3 + d % 5 for d in range(n)], [40, 200], [d % 2 for d in range(n)])


def slabs(Hq, Hkv, hd, dtype, docs, T, S, P, prompts, seed=0):
    q, k, v = randn((docs, T, Hq, hd), dtype, seed), randn((docs, S, Hkv, hd), dtype, seed + 1), randn((docs, S, Hkv, hd), dtype, seed + 2)
    return q, k, v, randn((prompts, P, Hkv, hd), dtype, seed + 3), randn((prompts, P, Hkv, hd), dtype, seed + 4)


def ints(v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda")


def check_slabs(got, q, k, v, pk, pv, ql, kl, pl, of, dtype, **kw):
    for d in range(q.shape[0]):
        p = of[d]
        a, b, n = ql[d], kl[d], pl[p] if 0 <= p < len(pl) else 0
        one = dict(block=0, q_pos=None, prefix=None, cap=0.0, slopes=None, scale=None)
        one.update(kw)
        verify(got[d, :a], q[d, :a], k[d, :b], v[d, :b], pk[max(p, 0), :n], pv[max(p, 0), :n], [a], [b], [n], [0 if n else -1], dtype=dtype, **one)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("docs", [5, 70])
def test_padded_batches_in_slabs(gpu_lib, docs, dtype):
    """Dense slabs of documents and of prompts with lengths; rows behind a document keep what they held."""
    q, k, v, pk, pv = slabs(6, 2, 64, dtype, docs, 9, 50, 140, 3)
    pk, pv = longer(pk, REACH), longer(pv, REACH)
    ql, kl, pl, of = [d * 2 % 10 for d in range(docs)], [50 - d % 30 for d in range(docs)], [140, 1, 77], [d * 3 // docs for d in range(docs)]
    out = randn(q.shape, dtype, 9)
    before = out.clone()
    got = B.shared_attention(q, k, v, pk, pv, B.Docs(q_len=ints(ql), kv_len=ints(kl)), B.Prompts(len=ints(pl), of=ints(of)), block=1, out=out)
    check_slabs(got, q, k, v, pk, pv, ql, kl, pl, of, dtype, block=1)
    for d in range(docs):
        assert torch.equal(got[d, ql[d]:], before[d, ql[d]:])


def test_queries_that_are_one_slab_expanded(gpu_lib):
    """The same queries for every document, out a slab each; and heads of k and v that lie apart."""
    q, k, v, pk, pv = slabs(4, 2, 64, BF16, 7, 3, 20, 100, 1)
    q = q[:1].expand(7, -1, -1, -1)
    pk, pv = (longer(t, REACH).transpose(1, 2).contiguous().transpose(1, 2) for t in (pk, pv))
    out = torch.empty((7, 3, 4, 64), dtype=BF16, device="cuda")
    ws = B.device_buffer(B.shared_attention_workspace_size(q, k, v, pk, pv))
    got = B.shared_attention(q, k, v, pk, pv, out=out, ws=ws, prompts=B.Prompts(len=ints([100]), of=ints([0] * 7)))
    check_slabs(got, q, k, v, pk, pv, [3] * 7, [20] * 7, [100], [0] * 7, BF16)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("many", [False, True])
def test_broken_numbers(gpu_lib, many, dtype):
    """What lies behind a prompt and behind what a query sees reaches nothing; what is seen reaches its queries alone."""
    heads = (8, 8, 64)
    q_lens = [130] * 33 if many else [3, 2, 4]
    kv_lens = [n + 20 for n in q_lens]
    of = [d % 2 for d in range(len(q_lens))] if many else [0, 1, 0]
    inf, nan = float("inf"), float("nan")

    def behind(q, k, v, pk, pv):
        pk[70 + 33:], pv[70 + 33:] = nan, inf
        for t in (k, v):
            t[sum(kv_lens):] = nan

    base, (q, k, v, pk, pv, docs, prompts, _) = run_and_check(*heads, dtype, q_lens, kv_lens, [70, 33], of, block=1, q_pos=[0] * len(q_lens), mutate=behind)
    clean = base.clone()
    # own keys that no query sees (position 0 .. q - 1 of q + 20 keys)
    k0 = starts(kv_lens)
    for d, n in enumerate(q_lens):
        k[k0[d] + n + 1:k0[d] + n + 20], v[k0[d] + n:k0[d] + n + 20] = nan, inf
    n = sum(q_lens)
    assert torch.equal(B.shared_attention(q, k, v, pk, pv, docs, prompts, block=1)[:n], clean[:n])
    # a value of prompt 1: its documents' rows, in that dimension
    pv[70 + 5, 3, 11] = nan
    got = B.shared_attention(q, k, v, pk, pv, docs, prompts, block=1)[:n]
    hit = torch.zeros_like(got, dtype=torch.bool)
    for d, a in enumerate(starts(q_lens)):
        if of[d] == 1:
            hit[a:a + q_lens[d], 3, 11] = True
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], clean[:n][~hit])


def test_rows_that_see_nothing(gpu_lib):
    """No prompt and no visible key: zeros; infinite slopes beside a prompt; scores of -inf."""
    got, _ = run_and_check(4, 2, 64, F32, [2, 1, 2], [0, 4, 4], [0, 8], [-1, 0, 1], block=1, q_pos=[0, -3, -3])
    assert not got[:3].any()
    run_and_check(4, 4, 64, BF16, [2, 1], [3, 4], [8], None, block=1, slopes=[float("inf"), 0.0, 1e30, -0.5], q_pos=[0, 3])
    run_and_check(4, 4, 64, BF16, [2, 1], [3, 4], [8], None, slopes=[float("inf"), 0.0, 1e30, -0.5], q_pos=[10, -20])
    run_and_check(4, 4, 64, BF16, [2, 1], [3, 4], [8], None, scale=-0.1)
    run_and_check(4, 4, 64, F32, [2, 1], [3, 4], [8], None, scale=0.0)


@pytest.mark.parametrize("docs", [3, 70])
def test_arrays_that_make_no_sense(gpu_lib, docs):
    """Ranges are cut to their slabs and to the maxima, prompts that are none are none."""
    big, low = 2 ** 31 - 1, -2 ** 31
    q, k, v, pk, pv = slabs(4, 2, 64, BF16, docs, 4, 30, 60 + REACH, 3)
    most = 40 + REACH
    pad = lambda v, rest: ints(list(v) + [rest] * (docs - 3))  # noqa: E731
    d = B.Docs(q_start=pad([low, 1, big], 0), q_len=pad([2, big, 5], 1), kv_start=pad([0, 20, low], 0), kv_len=pad([big, big, -4], 3), max_q=3, max_kv=25,
               q_pos=pad([big, low, 0], 0), prefix=pad([low, big, 7], 0))
    p = B.Prompts(start=ints([low, 50, big]), len=ints([big, big, 9]), max=most, of=pad([0, 1, big], low))
    out = randn(q.shape, BF16, 5)
    before = out.clone()
    got = B.shared_attention(q, k, v, pk, pv, d, p, block=4, out=out)
    sl = lambda t, d, a, n: t[d:d + 1, a:a + n]  # noqa: E731
    verify(got[0, :2], q[0, :2], k[0, :25], v[0, :25], pk[0, :most], pv[0, :most], [2], [25], [most], [0], 4, [big], [low], 0.0, None, None, BF16)
    verify(got[1, 1:4], q[1, 1:4], k[1, 20:30], v[1, 20:30], pk[1, 50:], pv[1, 50:], [3], [10], [10 + REACH], [0], 4, [low], [big], 0.0, None, None, BF16)
    assert torch.equal(got[0, 2:], before[0, 2:]) and torch.equal(got[1, :1], before[1, :1]) and torch.equal(got[2], before[2])


def test_far_apart_and_far_away(gpu_lib):
    """Prompts further apart than 2^32 bytes; positions far behind every key keep their biases' precision."""
    far = torch.zeros((2, 40_000_000, 64), dtype=BF16, device="cuda")
    pk, pv = randn((2, 90, 1, 64), BF16, 1), randn((2, 90, 1, 64), BF16, 2)
    K = far.as_strided((2, 90 + REACH, 1, 64), (40_000_000 * 64, 64 * 100, 64, 1))
    V = far.as_strided((2, 90 + REACH, 1, 64), (40_000_000 * 64, 64 * 100, 64, 1), 64)
    K[:, :90].copy_(pk)
    V[:, :90].copy_(pv)
    q, k, v = randn((5, 2, 64), BF16, 3), randn((9, 1, 64), BF16, 4), randn((9, 1, 64), BF16, 5)
    docs = B.Docs.packed([2, 3], [4, 5], q_pos=[0, 2 ** 31 - 1])
    got = B.shared_attention(q, k, v, K, V, docs, B.Prompts(len=ints([90, 90]), of=ints([1, 0])), slopes=torch.tensor([0.3, 0.01], device="cuda"))
    verify(got, q, k, v, torch.cat([pk[0], pk[1]]), torch.cat([pv[0], pv[1]]), [2, 3], [4, 5], [90, 90], [1, 0], 0, [0, 2 ** 31 - 1], None, 0.0,
           np.float32([0.3, 0.01]), None, BF16)


@pytest.mark.parametrize("docs", [4, 70])
def test_captured_and_on_other_streams(gpu_lib, docs):
    """Two calls in one graph with a workspace each, replayed with other inputs and eager work between; a call on
    another stream."""
    q, k, v, pk, pv = slabs(8, 2, 64, BF16, docs, 2, 40, 300, 1)
    pk, pv, length = longer(pk, REACH), longer(pv, REACH), ints([300])
    n = ints([d % 41 for d in range(docs)])
    call = lambda ws, out, s=None: B.shared_attention(q, k, v, pk, pv, B.Docs(kv_len=n), B.Prompts(len=length, of=ints0), block=1, out=out, ws=ws, stream=s)  # noqa: E731
    ints0 = ints([0] * docs)
    need = B.shared_attention_workspace_size(q, k, v, pk, pv)
    ws, outs = [B.device_buffer(need) for _ in range(3)], [torch.empty_like(q) for _ in range(3)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call(ws[0], outs[0])
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            call(ws[0], outs[0])
            call(ws[1], outs[1])
    for i in range(4):
        q.copy_(randn(q.shape, BF16, 20 + i))
        n.copy_(ints([(d * (i + 3)) % 41 for d in range(docs)]))
        torch.cuda.synchronize()
        g.replay()
        eager = B.shared_attention(q, k, v, pk, pv, B.Docs(kv_len=n), B.Prompts(len=length, of=ints0), block=1)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], eager) and torch.equal(outs[1], eager)
    call(ws[2], outs[2], torch.cuda.Stream())
    torch.cuda.synchronize()
    assert torch.equal(outs[2], eager)


def test_without_prompts_it_is_attention_of_documents(gpu_lib):
    q, k, v, pk, pv = slabs(4, 2, 64, BF16, 3, 5, 60, 10, 1)
    ref = B.attention(q, k, v, block=1)
    for p in (B.Prompts(count=0, max=0), B.Prompts(max=0), B.Prompts(len=ints([0])), B.Prompts(of=ints([-1, 1, 7]))):
        pkp, pvp = (pk[0], pv[0]) if p.count == 0 or p.len is not None else (pk, pv)
        got = B.shared_attention(q, k, v, pkp, pvp, prompts=p, block=1)
        assert (got.float() - ref.float()).abs().max() <= 2.0 ** -7


@pytest.mark.parametrize("heads,dtype,q_lens,kv_lens,p_lens,of,block,units", [
    ((28, 4, 128), BF16, [24, 10, 23], [40, 10, 39], [23], None, 1, False),
    ((28, 4, 128), BF16, [24, 10, 23], [40, 10, 39], [2000, 65], [0, 0, 1], 1, True),
    ((28, 4, 128), BF16, [24, 10, 23], [40, 500, 39], [2000, 65], [0, 1, -1], 32, True),
    ((28, 4, 128), F32, [24, 10, 23], [40, 10, 39], [23], None, 1, False),
    ((28, 4, 128), F32, [24, 10, 23], [40, 10, 39], [500], None, 1, True),
    ((16, 2, 64), BF16, [9, 0, 17], [9, 0, 17], [31, 64], [1, 0, 0], 0, False),
    ((16, 2, 64), BF16, [9, 0, 17], [1009, 0, 17], [31, 1064], [1, 0, 0], 0, True),
    ((8, 8, 128), F32, [128 - d % 7 for d in range(32)], [130 + d for d in range(32)], [60, 0], [d % 3 for d in range(32)], 1, False),
    ((8, 8, 64), F32, [128 - d % 7 for d in range(32)], [130 + d for d in range(32)], [60, 0], [d % 3 for d in range(32)], 32, False),
    ((8, 8, 64), F32, [128 - d % 7 for d in range(8)], [130 + d for d in range(8)], [60, 0], [d % 3 for d in range(8)], 32, False),
    ((8, 8, 64), F32, [128 - d % 7 for d in range(8)], [130 + d for d in range(8)], [7000, 0], [d % 3 for d in range(8)], 32, True),
])
def test_tiles_that_take_all_keys_and_units_of_them(gpu_lib, heads, dtype, q_lens, kv_lens, p_lens, of, block, units):
    """Both sides of the choice, which the workspace shows: tiles that take all their keys need none."""
    slopes = [2.0 ** -(1 + h / 4) for h in range(heads[0])]
    _, (q, k, v, pk, pv, docs, prompts, _) = run_and_check(*heads, dtype, q_lens, kv_lens, p_lens, of, block, None, None, 30.0, slopes, reach=0)
    assert (B.shared_attention_workspace_size(q, k, v, pk, pv, docs, prompts) > 0) == units


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("docs,prompts", [(64, 64), (64, 65), (5, 200), (70, 200)])
def test_many_prompts(gpu_lib, docs, prompts, dtype):
    """More prompts than lanes that ask for their ranges at once, most of them of no document."""
    rng = np.random.default_rng(docs * prompts)
    lens = rng.integers(0, 90, prompts).tolist()
    of = np.sort(rng.integers(-1, prompts + 1, docs)).tolist()
    run_and_check(4, 2, 64, dtype, rng.integers(0, 4, docs).tolist(), rng.integers(4, 40, docs).tolist(), lens, of, block=1)
