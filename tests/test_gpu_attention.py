"""dllm_attention against the float64 oracle, document by document.

Tolerance, per output element, with A the softmax-weighted |v| and u = 2^-24: a score's
error is d = u ((hd + 8) scale max_j sum |q k_j| + 8 max |s|) over the keys that have a probability, and 2^-21 of the cap where
there is one; a probability is off by 2 d + 8 u relative, and where bf16 holds it by half a
step more (2^-8); sums over n keys add n u; the result is rounded once to its type."""
import math

import numpy as np
import pytest
import torch

from helpers import say, to_np
from oracle import operators as oo
from paper_2608_22646_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def randn(shape, dtype, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype).cuda()


def tolerance(ref, mass, top, dot, n, hd, dtype, scale, cap):
    u = 2.0 ** -24
    d = u * ((hd + 8) * abs(scale) * dot + 8 * top) + (2.0 ** -21 * cap if cap else 0.0)
    p = 2 * d + (8 + n) * u + (2.0 ** -8 if dtype == BF16 else 0.0)
    return p[:, :, None] * mass * 1.01 + torch.finfo(dtype).eps / 2 * np.abs(ref) * 1.01 + 1e-37


def run_and_check(Hq, Hkv, hd, dtype, q_lens, kv_lens, block=0, q_pos=None, prefix=None, cap=0.0, slopes=None, scale=None,
                  seed=0, std=1.3, pad=3, mutate=None, acts_as=None):
    """Packed documents (pad rows behind the last one); mutate(q, k, v) changes the inputs first;
    acts_as: the cap that the oracle takes instead."""
    T, S = sum(q_lens), sum(kv_lens)
    say(f"attention {Hq}/{Hkv}x{hd} {dtype} q{q_lens} kv{kv_lens} block {block} pos {q_pos} prefix {prefix} cap {cap} "
        f"slopes {slopes is not None}")
    q, k, v = (randn((n + pad, H, hd), dtype, seed + i, std) for i, (n, H) in enumerate([(T, Hq), (S, Hkv), (S, Hkv)]))
    if mutate:
        mutate(q, k, v)
    out = randn((T + pad, Hq, hd), dtype, seed + 3)
    behind = out[T:].clone()
    docs = B.Docs.packed(q_lens, kv_lens, q_pos, prefix)
    sl = None if slopes is None else torch.tensor(slopes, dtype=F32, device="cuda")
    got = B.attention(q, k, v, docs, block=block, cap=cap, slopes=sl, scale=scale, out=out)
    torch.cuda.synchronize()
    assert got is out and torch.equal(out[T:], behind)
    verify(got, q, k, v, q_lens, kv_lens, block, q_pos, prefix, cap if acts_as is None else acts_as,
           None if slopes is None else np.float32(slopes), scale, dtype)
    return got


def verify(got, q, k, v, q_lens, kv_lens, block, q_pos, prefix, cap, slopes, scale, dtype):
    hd = q.shape[2]
    sc = float(np.float32(1 / math.sqrt(hd) if scale is None else scale))
    q0 = k0 = 0
    for d, (a, b) in enumerate(zip(q_lens, kv_lens)):
        qq, kk, vv = to_np(q[q0:q0 + a], np.float64), to_np(k[k0:k0 + b], np.float64), to_np(v[k0:k0 + b], np.float64)
        with np.errstate(all="ignore"):
            ref, mass, top, dot = oo.attention(qq, kk, vv, (b - a) if q_pos is None else q_pos[d], block,
                                          0 if prefix is None else prefix[d], sc, cap, slopes)
        g = to_np(got[q0:q0 + a], np.float64)
        with np.errstate(all="ignore"):
            tol = tolerance(ref, mass, top, dot, b, hd, dtype, sc, cap)
        fine = np.isfinite(ref)
        assert (np.isfinite(g) == fine).all(), f"document {d}: {(np.isfinite(g) != fine).sum()} elements finite on one side only"
        err = np.where(fine, np.abs(np.where(fine, g, 0) - np.where(fine, ref, 0)), 0)
        tol = np.where(fine, tol, 1)
        assert (err <= tol).all(), f"document {d}: {(err > tol).sum()} off, worst {(err / tol).max():.3g} tolerances"
        q0, k0 = q0 + a, k0 + b


HEADS = [(4, 4, 64), (4, 2, 128), (7, 1, 128), (28, 4, 128), (16, 2, 64), (2, 2, 128)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("q_lens,kv_lens", [([1], [1]), ([1, 1, 1], [5, 64, 65]), ([3, 0, 40, 1], [3, 7, 40, 33]),
                                            ([33, 64], [129, 64]), ([5, 2], [0, 2])])
def test_lengths(gpu_lib, heads, q_lens, kv_lens, dtype):
    run_and_check(*heads, dtype, q_lens, kv_lens, seed=sum(q_lens))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads", [(4, 4, 64), (6, 2, 128)])
@pytest.mark.parametrize("block,prefix", [(1, None), (1, [70, 0]), (32, None), (5, [3, 100]), (64, [1, 500])])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (20.0, False), (0.0, True), (5.0, True)])
def test_masks_caps_and_biases(gpu_lib, heads, block, prefix, cap, bias, dtype):
    slopes = [2.0 ** -(h + 1) for h in range(heads[0])] if bias else None
    run_and_check(*heads, dtype, [97, 130], [150, 130], block, None, prefix, cap, slopes, seed=block)


@pytest.mark.parametrize("cap", [30.0, 200.0])
def test_small_capped_scores_keep_their_precision(gpu_lib, cap):
    """float32, one product a score, two keys of which the other scores 0, values 1 and 0: the
    output is 1 / (1 + e^-s) with s = cap tanh(x / cap).  In units u = 2^-24: s is off by 8 of
    itself (scale, product, tanh of relative 1.3, its sums), the probability by s (1 - p) of that
    and by 8 for exponential, sum, division and rounding."""
    n, hd, u = 256, 64, 2.0 ** -24
    x = torch.arange(-n // 2, n // 2, dtype=F32) / 32 + 2.0 ** -9
    q = torch.zeros(n, 1, hd)
    q[:, 0, 5] = x
    k = torch.zeros(2, 1, hd)
    k[0, 0, 5] = 1
    v = torch.zeros(2, 1, hd)
    v[0] = 1
    say(f"attention two keys cap {cap}")
    got = to_np(B.attention(q.cuda(), k.cuda(), v.cuda(), B.Docs.packed([n], [2]), cap=cap, scale=1.0), np.float64)[:, 0]
    s = cap * np.tanh(x.numpy().astype(np.float64) / cap)
    p = 1 / (1 + np.exp(-s))
    tol = u * p * (8 * np.abs(s) * (1 - p) + 8)
    assert (np.abs(got - p[:, None]) <= tol[:, None]).all(), (np.abs(got - p[:, None]) / tol[:, None]).max()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("q_len,kv", [(1, 4097), (1, 8448), (4, 3001), (32, 2050), (33, 1999), (64, 2048)])
def test_few_queries_over_a_long_cache(gpu_lib, q_len, kv, dtype):
    """Lengths at which the keys of a document are split; the others in the call are short."""
    run_and_check(7, 1, 128, dtype, [q_len, q_len, 1], [kv, 31, 1], block=1, seed=kv)
    run_and_check(4, 4, 64, dtype, [q_len, 2], [kv, 700], block=32, q_pos=[kv // 2 // 32 * 32, 100], seed=kv + 1)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_more_rows_than_one_tile(gpu_lib, dtype):
    run_and_check(2, 1, 128, dtype, [300, 513], [300, 700], block=1, seed=9)
    run_and_check(2, 2, 64, dtype, [700], [700], block=32, prefix=[40], cap=30.0, seed=10)


@pytest.mark.parametrize("heads", [(16, 16, 64), (32, 16, 128)])
@pytest.mark.parametrize("block,cap,bias", [(0, 0.0, False), (1, 0.0, False), (32, 30.0, False), (7, 0.0, True), (0, 4.0, True)])
def test_many_rows(gpu_lib, heads, block, cap, bias):
    """Enough row tiles for two workgroups on every CU: bf16 tiles of 128 rows; ragged documents, some
    without queries or keys, invisible values that are no numbers."""
    g = torch.Generator().manual_seed(block)
    most = 130 * 16 // heads[0]
    q_lens = [most, 0, 1, most - 1] + torch.randint(1, most + 1, (12,), generator=g).tolist()
    kv_lens = [n + int(e) for n, e in zip(q_lens, torch.randint(0, 90, (16,), generator=g))]
    kv_lens[5] = 0
    q_pos = [max(k - q, 0) // 2 for q, k in zip(q_lens, kv_lens)]

    def hide(q, k, v):
        if block:
            end = kv_lens[0]                # what no query of document 0 sees, if there is any
            seen = ((q_pos[0] + q_lens[0] - 1) // block + 1) * block
            k[seen:end], v[seen:end] = math.inf, math.nan
            v[min(seen, end) - 1, :, 5] = math.inf      # and what its last queries see
    run_and_check(*heads, BF16, q_lens, kv_lens, block, q_pos, [0, 5] * 8 if block else None, cap,
                  [2.0 ** -(h % 8 + 1) for h in range(heads[0])] if bias else None, seed=block, mutate=hide)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,heads", [(3, (4, 2, 64)), (64, (2, 1, 64)), (70, (4, 2, 128)), (250, (2, 1, 64))])
def test_documents_of_unlike_lengths_share_the_split(gpu_lib, n, heads, dtype):
    """One long document among short ones, empty ones and ones without queries."""
    g = torch.Generator().manual_seed(n)
    kv_lens = torch.randint(0, 300, (n,), generator=g).tolist()
    kv_lens[n // 2], kv_lens[-1] = 6000, 1300
    q_lens = torch.randint(0, 3, (n,), generator=g).tolist()
    q_lens[n // 2] = 2
    run_and_check(*heads, dtype, q_lens, kv_lens, block=1, seed=n)
    if n == 3:
        run_and_check(*heads, dtype, [1, 2, 40], [300, 6000, 900], block=32, q_pos=[5, 3000, 100], seed=n)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,kv", [(40, 90), (1, 2000), (300, 300)])
def test_rows_without_keys_are_zero(gpu_lib, n, kv, dtype):
    """Queries before position 0 see nothing (and see the prefix where there is one)."""
    got = run_and_check(4, 2, 128, dtype, [n, n], [kv, kv], block=1, q_pos=[-n - 3, -1], seed=1)
    assert torch.count_nonzero(got[:n]) == 0
    got = run_and_check(4, 2, 128, dtype, [n], [kv], block=1, q_pos=[-2 ** 31], prefix=[5], seed=2)
    assert torch.count_nonzero(got[:n])
    got = run_and_check(4, 2, 128, dtype, [n], [kv], block=32, q_pos=[-n], prefix=[-7], seed=3)
    assert torch.count_nonzero(got[:n]) == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("n,kv,q_pos", [(70, 130, 0), (1, 2100, 1000), (200, 200, 0)])
def test_what_lies_at_invisible_keys_reaches_nothing(gpu_lib, n, kv, q_pos, bad, dtype):
    """Keys and values behind every query's reach, past the document, and behind some queries' reach only."""
    def outside(q, k, v):
        k[q_pos + n:kv], v[q_pos + n:kv] = bad, bad
        k[kv:], v[kv:] = bad, bad
    got = run_and_check(4, 2, 128, dtype, [n], [kv], block=1, q_pos=[q_pos], seed=4, mutate=outside)
    assert torch.isfinite(got[:n].float()).all()
    at = q_pos + n // 2

    def inside(q, k, v):
        v[at, 0, 3], v[at, 1, 77] = bad, bad      # reaches dimension 3 and 77 of the queries from `at` on
        k[kv - 1] = bad                           # seen by nobody, or by the last query
    got = run_and_check(4, 2, 128, dtype, [n], [kv], block=1, q_pos=[q_pos], seed=5, mutate=inside)
    assert torch.isfinite(got[:n // 2].float()).all()
    if n > 1:
        assert not torch.isfinite(got[n // 2, :2, 3].float()).any() and not torch.isfinite(got[n // 2, 2:, 77].float()).any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_extreme_scores(gpu_lib, dtype):
    """The type's lowest and largest values in a key (scores overflow to infinities), and very large finite scores."""
    def low(q, k, v):
        q.abs_()
        k[5], k[40] = torch.finfo(dtype).min, torch.finfo(dtype).min
    run_and_check(2, 2, 64, dtype, [50], [50], seed=6, mutate=low)

    def high(q, k, v):
        k[7] *= 3e4
    run_and_check(2, 2, 64, dtype, [50, 1], [50, 900], block=1, seed=7, mutate=high)

    def all_low(q, k, v):           # no score above -inf: zeros
        q.abs_().add_(1)
        k[:] = -math.inf
    got = run_and_check(2, 2, 64, dtype, [3, 40], [70, 41], seed=8, mutate=all_low)
    assert torch.count_nonzero(got[:43]) == 0

    def nan_query(q, k, v):
        q[2, 1] = math.nan
    got = run_and_check(2, 2, 64, dtype, [40], [40], block=1, seed=9, mutate=nan_query)
    assert torch.isnan(got[2, 1].float()).all() and torch.isfinite(got[2, 0].float()).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cap", [1e-40, 1e-20, 1e30])
def test_caps_of_any_size(gpu_lib, cap, dtype):
    """A cap that leaves nothing of the scores, or all; some scores are 0."""
    def zero(q, k, v):
        q[3] = 0
        k[20] = 0
    run_and_check(4, 2, 64, dtype, [40], [70], cap=cap, seed=11, mutate=zero, acts_as=0.0 if cap > 1 else None)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_dense_batch_layouts(gpu_lib, dtype):
    """Slabs per document: [B, T, H, hd], [B, H, T, hd], slices of a packed projection, one key/value head for all."""
    Bn, T, S, Hq, Hkv, hd = 3, 21, 90, 4, 2, 64
    kv_lens = [90, 0, 33]
    lens = torch.tensor(kv_lens, dtype=torch.int32, device="cuda")
    q = randn((Bn, Hq, T, hd), dtype, 1).transpose(1, 2)
    kv = randn((Bn, S, 2 * Hkv + 1, hd), dtype, 2)
    k, v = kv[:, :, :Hkv], kv[:, :, Hkv:2 * Hkv]
    say(f"attention dense {dtype}")
    out = torch.zeros((Bn, Hq, T, hd), dtype=dtype, device="cuda").transpose(1, 2)
    B.attention(q, k, v, B.Docs(kv_len=lens, q_pos=torch.tensor([69, 0, 12], dtype=torch.int32, device="cuda")), block=1, out=out)
    for d in range(Bn):
        n = kv_lens[d]
        verify(out[d], q[d], k[d][:n], v[d][:n], [T], [n], 1, [[69, 0, 12][d]], None, 0.0, None, None, dtype)
    one = k[:, :, :1].expand(Bn, S, Hq, hd)      # every head the same keys: a head stride of 0
    got = B.attention(q, one, one)
    for d in range(Bn):
        verify(got[d], q[d], one[d], one[d], [T], [S], 0, None, None, 0.0, None, None, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_ranges_are_cut(gpu_lib, dtype):
    """Starts and lengths that leave the slab or the maxima are cut; nothing outside is read or written."""
    say(f"attention ranges {dtype}")
    q, k = randn((20, 2, 64), dtype, 1), randn((30, 2, 64), dtype, 2)
    v = randn((30, 2, 64), dtype, 3)
    out = torch.full_like(q, 7.0)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    docs = B.Docs(ints(-5, 12, 50), ints(4, 100, 3), ints(25, -9, 0), ints(9, 2 ** 31 - 1, 5), 6, 28)
    B.attention(q, k, v, docs, out=out)
    verify(out, q, k[25:30], v[25:30], [4], [5], 0, None, None, 0.0, None, None, dtype)
    verify(out[12:], q[12:], k[:28], v[:28], [6], [28], 0, None, None, 0.0, None, None, dtype)
    assert (out[4:12] == 7).all() and (out[18:] == 7).all()


def test_shared_keys(gpu_lib):
    """Documents that read the same keys (a shared prompt) and queries in no order."""
    say("attention shared keys")
    q, k, v = randn((9, 4, 128), BF16, 1), randn((600, 2, 128), BF16, 2), randn((600, 2, 128), BF16, 3)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    got = B.attention(q, k, v, B.Docs(ints(5, 0), ints(4, 5), ints(0, 0), ints(600, 600), 5, 600), block=1)
    for a, n in ((5, 4), (0, 5)):
        verify(got[a:], q[a:], k, v, [n], [600], 1, None, None, 0.0, None, None, BF16)


def test_offsets_past_32_bits(gpu_lib):
    """Keys beyond 4 GiB of the first: a cache of 2.3 million tokens of eight heads."""
    say("attention far offsets")
    S = 2_300_000
    kv = torch.zeros((S, 8, 128), dtype=BF16, device="cuda")
    tail = randn((700, 8, 128), BF16, 5)
    kv[-700:] = tail
    q = randn((2, 8, 128), BF16, 6)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    got = B.attention(q, kv, kv, B.Docs(ints(0), ints(2), ints(S - 700), ints(700), 2, 700))
    verify(got, q, tail, tail, [2], [700], 0, None, None, 0.0, None, None, BF16)
    x = torch.zeros((S, 8, 128), dtype=BF16, device="cuda")
    x[-40:] = q.repeat(20, 1, 1)
    got = B.attention(x, kv[-700:], kv[-700:], B.Docs(ints(S - 40), ints(40), ints(0), ints(700), 40, 700), out=torch.zeros_like(x))
    verify(got[-40:], x[-40:], tail, tail, [40], [700], 0, None, None, 0.0, None, None, BF16)
    assert torch.count_nonzero(got[:-40]) == 0


@pytest.mark.parametrize("q_len", [1, 40])
def test_streams_graphs_and_repeats(gpu_lib, q_len):
    say(f"attention streams and graphs {q_len}")
    q, k, v = randn((2 * q_len, 8, 128), BF16, 1), randn((5000, 2, 128), BF16, 2), randn((5000, 2, 128), BF16, 3)
    docs = B.Docs.packed([q_len, q_len], [3000, 2000])
    want = B.attention(q, k, v, docs, block=1)
    assert torch.equal(B.attention(q, k, v, docs, block=1), want)      # the same bits each time
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = B.attention(q, k, v, docs, block=1, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    out = torch.zeros_like(q)
    n = B.attention_workspace_size(q, k, v, docs)
    ws = B.device_buffer(n) if n else None
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.attention(q, k, v, docs, block=1, out=out, ws=ws)
    for _ in range(3):
        q.mul_(1.5)
        docs.kv_len[0] -= 7
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, B.attention(q, k, v, docs, block=1))


def test_binding_checks_shapes(gpu_lib):
    q, k = torch.zeros((4, 4, 64), device="cuda"), torch.zeros((6, 2, 64), device="cuda")
    i32 = torch.zeros(2, dtype=torch.int32, device="cuda")
    for call in (lambda: B.attention(q, k, k[:5]), lambda: B.attention(q, k.bfloat16(), k), lambda: B.attention(q, k[..., :32], k),
                 lambda: B.attention(q, k, k, B.Docs(q_len=i32, kv_len=i32[:1])), lambda: B.attention(q, k, k, B.Docs(q_len=i32.long())),
                 lambda: B.attention(q, k, k, slopes=torch.zeros(3, device="cuda")), lambda: B.attention(q, k, k, out=q[:3]),
                 lambda: B.attention(q, k, k, B.Docs(max_q=5)), lambda: B.attention(q[None], k, k)):
        with pytest.raises(B.DllmError):
            call()
    assert B.attention(q[:0], k, k).shape == (0, 4, 64)
