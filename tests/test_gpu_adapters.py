"""dllm_adapters against the float64 oracle.

Tolerance, per output element, with M the sum of magnitudes scale |B| |A| |x| and u = 2^-24: the inner product adds K
terms of the type's exact products in float32 (K u of their magnitudes at most), the outer one R parts' (3 R u), the
shares and the scale a few u more; where out is bf16 the inner sum enters with 16 bits, off by 2^-17 of itself; the
result is added to the base and rounded once."""
import numpy as np
import pytest
import torch

from helpers import say, to_np
from oracle import operators as oo
from paper_2608_22646_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
KINDS = [(F32, F32), (BF16, BF16), (BF16, F32)]


def randn(shape, dtype, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype).cuda()


def ints(v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda")


def inputs(M, K, widths, n, R, dtype, kind, seed=0):
    N, S = sum(widths), len(widths)
    return (randn((M, K), dtype, seed), randn((M, N), kind, seed + 1), randn((n, S, R, K), dtype, seed + 2, K ** -0.5),
            randn((n, N, R), dtype, seed + 3, 0.5 * R ** -0.5))


def verify(got, x, base, A, Bm, which, ranks, scales, widths):
    ends = list(np.cumsum(widths))
    n, R = A.shape[0], A.shape[2]
    ranks = [R] * n if ranks is None else ranks
    scales = [1.0] * n if scales is None else [float(np.float32(s)) for s in scales]
    f64 = lambda t: to_np(t, np.float64)  # noqa: E731
    ref, mass = oo.adapters(f64(x), np.zeros(got.shape) if base is None else f64(base), f64(A), f64(Bm), which, ranks, scales, ends)
    u = 2.0 ** -24
    tol = ((x.shape[1] + 3 * R + 8) * u + (2.0 ** -17 if got.dtype == BF16 else 0)) * mass * 1.01
    tol += (torch.finfo(got.dtype).eps / 2 * (np.abs(ref) + tol) + u * np.abs(ref)) * 1.01 + 1e-37
    err = np.abs(f64(got) - ref)
    assert (err <= tol).all(), f"{(~(err <= tol)).sum()} off, worst {(err / tol).max():.3g} tolerances"
    none = [m for m, a in enumerate(which) if not 0 <= a < n]
    if none and base is not None:
        assert torch.equal(got[none], base[none])


def run(M, K, widths, n, R, dtype, kind, which, ranks=None, scales=None, seed=0, **kw):
    say(f"adapters {M} x {K} -> {widths}, {n} of rank {R}, {dtype} {kind}")
    x, base, A, Bm = inputs(M, K, widths, n, R, dtype, kind, seed)
    sc = None if scales is None else torch.tensor(scales, dtype=F32, device="cuda")
    got = B.adapters(x, base, A, Bm, ints(which), ranks=None if ranks is None else ints(ranks), scales=sc, slices=widths, **kw)
    torch.cuda.synchronize()
    verify(got, x, base, A, Bm, which, ranks, scales, widths)
    return got


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("M,K,widths,n,R", [(1, 8, (8,), 1, 1), (1, 4096, (256,), 3, 16), (33, 64, (128, 8, 40), 2, 8), (31, 1000, (136,), 40, 40),
                                            (64, 520, (512, 128), 9, 64), (65, 512, (384,), 1, 16), (200, 96, (264, 24), 5, 24),
                                            (130, 264, (1000,), 3, 256)])
def test_sizes(gpu_lib, M, K, widths, n, R, dtype, kind):
    rng = np.random.default_rng(M + K)
    run(M, K, widths, n, R, dtype, kind, rng.integers(-1, n, M).tolist(), rng.integers(0, R + 3, n).tolist(),
        rng.uniform(-2, 2, n).tolist(), seed=M)


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("M,K,widths,n,R", [(1, 1, (1,), 1, 1), (5, 333, (77, 1, 130), 2, 5), (70, 63, (129,), 4, 3), (97, 37, (3, 250), 6, 17)])
def test_odd_sizes_are_read_by_the_element(gpu_lib, M, K, widths, n, R, dtype, kind):
    run(M, K, widths, n, R, dtype, kind, [(m * 7) % (n + 1) - 1 for m in range(M)], [max(1, R - a) for a in range(n)], [1.0 + a for a in range(n)])


@pytest.mark.parametrize("M", [1, 16, 17, 32, 48, 64, 65, 96, 1100])
@pytest.mark.parametrize("order", ["one", "runs", "each", "none"])
def test_orders_of_rows(gpu_lib, M, order):
    n = 70
    which = {"one": [3] * M, "runs": [m * 5 // M for m in range(M)], "each": [(m * 37) % n for m in range(M)],
             "none": [-1 if m % 2 else n + m for m in range(M)]}[order]
    run(M, 128, (136, 24), n, 16, BF16, BF16, which, seed=M)


def test_a_result_does_not_depend_on_the_other_rows(gpu_lib):
    """The same rows in another order and company, split alike: bit for bit."""
    x, base, A, Bm = inputs(300, 256, (264,), 6, 16, BF16, F32)
    which = [(m * m) % 7 - 1 for m in range(300)]
    one = B.adapters(x, base, A, Bm, ints(which))
    order = torch.randperm(300, generator=torch.Generator().manual_seed(1)).tolist()
    two = B.adapters(x[order], base[order], A, Bm, ints(which[i] for i in order))
    assert torch.equal(one[order], two)
    for _ in range(3):
        assert torch.equal(B.adapters(x, base, A, Bm, ints(which)), one)


@pytest.mark.parametrize("dtype,kind", KINDS)
def test_views_in_place_and_rows_behind(gpu_lib, dtype, kind):
    """Operands inside wider buffers, at odd columns and at aligned ones; out is base, and what lies around it stays."""
    M, K, N, n, R = 50, 72, 136, 3, 16
    which = [m % 4 - 1 for m in range(M)]
    for at in (8, 3):
        X, Y = randn((M + 4, K + 32), dtype, 1), randn((M + 4, N + 32), kind, 2)
        WA, WB = randn((n, 2, R + 8, K + 16), dtype, 3, 0.1), randn((n, N + 3, R + 8), dtype, 4, 0.1)
        x, y, A, Bm = X[2:M + 2, at:at + K], Y[2:M + 2, at:at + N], WA[:, :, 1:R + 1, at:at + K], WB[:, 1:N + 1, at % 8:at % 8 + R]
        before, base = Y.clone(), y.clone()
        got = B.adapters(x, y, A, Bm, ints(which), slices=(100, 36), out=y)
        torch.cuda.synchronize()
        assert got is y
        verify(y, x, base, A, Bm, which, None, None, (100, 36))
        Y[2:M + 2, at:at + N] = base
        assert torch.equal(Y, before)


@pytest.mark.parametrize("M", [20, 100])
@pytest.mark.parametrize("dtype,kind", KINDS)
def test_without_a_base(gpu_lib, M, dtype, kind):
    x, base, A, Bm = inputs(M, 64, (80,), 2, 8, dtype, kind)
    which = [m % 3 - 1 for m in range(M)]
    got = B.adapters(x, None, A, Bm, ints(which), out=base)
    verify(got, x, None, A, Bm, which, None, None, (80,))
    assert not got[0].any()
    assert B.adapters(x, None, A, Bm, ints(which)).dtype == dtype


@pytest.mark.parametrize("M", [40, 150])
@pytest.mark.parametrize("dtype,kind", KINDS)
def test_broken_numbers_stay_in_their_rows(gpu_lib, M, dtype, kind):
    """NaN and infinities of a row, of an adapter, and behind the ranks."""
    n, R = 4, 16
    x, base, A, Bm = inputs(M, 96, (136,), n, R, dtype, kind)
    which = [m % 5 - 1 for m in range(M)]
    ranks = [16, 5, 3, 9]
    clean = B.adapters(x, base, A, Bm, ints(which), ranks=ints(ranks))
    for a, r in enumerate(ranks):
        A[a, :, r:] = float("nan")
        Bm[a, :, r:] = float("inf")
    assert torch.equal(B.adapters(x, base, A, Bm, ints(which), ranks=ints(ranks)), clean)
    x[7, 3], A[2, 0, 1, 5], Bm[2, 9, 0], x[0, 0] = float("inf"), float("nan"), float("nan"), float("nan")
    got = B.adapters(x, base, A, Bm, ints(which), ranks=ints(ranks))
    hit = torch.tensor([which[m] == 2 or m == 7 for m in range(M)], device="cuda")
    assert which[7] == 1 and which[0] == -1
    assert torch.equal(got[~hit], clean[~hit]) and not torch.isfinite(got[hit]).any()


def test_values_of_arrays_that_make_no_sense(gpu_lib):
    x, base, A, Bm = inputs(90, 64, (72,), 3, 8, BF16, BF16)
    which = [(-2 ** 31, 2 ** 31 - 1, 3, 0, 1, 2)[m % 6] for m in range(90)]
    got = B.adapters(x, base, A, Bm, ints(which), ranks=ints([-2 ** 31, 2 ** 31 - 1, 0]))
    verify(got, x, base, A, Bm, which, [-2 ** 31, 2 ** 31 - 1, 0], None, (72,))
    assert torch.equal(B.adapters(x, base, A[:0], Bm[:0], ints(which)), base)
    assert B.adapters(x[:0], base[:0], A, Bm, ints([])).shape == (0, 72)


def test_rows_and_outputs_beyond_32_bit_offsets(gpu_lib):
    """Rows so far apart that their offsets pass 2^32 bytes."""
    M, K, N = 70, 64, 40
    far = torch.zeros((M, 40_000_000), dtype=BF16, device="cuda")
    x, base, A, Bm = inputs(M, K, (N,), 2, 8, BF16, BF16)
    X, Y = far[:, :K], far[:, 20_000_000:20_000_000 + N]
    X.copy_(x)
    Y.copy_(base)
    which = [m % 2 for m in range(M)]
    verify(B.adapters(X, Y, A, Bm, ints(which), out=Y).clone(), x, base, A, Bm, which, None, None, (N,))


@pytest.mark.parametrize("M", [30, 200])
def test_captured_and_on_other_streams(gpu_lib, M):
    """Two calls in one graph with a workspace each, replayed with other inputs and eager work between; a call on
    another stream."""
    x, base, A, Bm = inputs(M, 512, (256, 128), 5, 40, BF16, BF16)
    which = ints(m % 6 - 1 for m in range(M))
    call = lambda ws, out, s=None: B.adapters(x, base, A, Bm, which, slices=(256, 128), out=out, ws=ws, stream=s)  # noqa: E731
    need = B.adapters_workspace_size(x, base, A, Bm, slices=(256, 128))
    assert need == B.adapters_workspace_size(x, None, A, Bm, slices=(256, 128))
    ws, outs = [B.device_buffer(need) for _ in range(3)], [torch.empty_like(base) for _ in range(3)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call(ws[0], outs[0])
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            call(ws[0], outs[0])
            call(ws[1], outs[1])
    for i in range(4):
        x.copy_(randn(x.shape, BF16, 20 + i))
        which.copy_(ints((m * (i + 2)) % 6 - 1 for m in range(M)))
        torch.cuda.synchronize()
        g.replay()
        eager = B.adapters(x, base, A, Bm, which, slices=(256, 128))
        torch.cuda.synchronize()
        assert torch.equal(outs[0], eager) and torch.equal(outs[1], eager)
    call(ws[2], outs[2], torch.cuda.Stream())
    torch.cuda.synchronize()
    assert torch.equal(outs[2], eager)


def test_infinities_follow_the_formula(gpu_lib):
    """An infinite scale, and inner products beyond bf16's pieces: infinities keep their sign, where b is not zero."""
    x, base, A, Bm = inputs(40, 64, (72,), 2, 8, BF16, F32)
    Bm.fill_(0.5)
    x.fill_(1.0)
    A[0], A[1] = 3e37, -3e37
    which = [m % 2 for m in range(40)]
    got = B.adapters(x, base, A, Bm, ints(which))
    assert all(torch.isinf(got[m]).all() and (got[m] > 0).all() == (m % 2 == 0) for m in range(40))
    A.fill_(1.0)
    got = B.adapters(x, base, A, Bm, ints(which), scales=torch.tensor([float("inf"), float("nan")], device="cuda"))
    assert (got[::2] == float("inf")).all() and torch.isnan(got[1::2]).all()


def test_no_adapter_at_all(gpu_lib):
    x, base, A, Bm = inputs(10, 64, (72,), 2, 8, BF16, BF16)
    out = base.clone()
    assert torch.equal(B.adapters(x, out, A, Bm, ints([-1] * 10), out=out), base)
    assert not B.adapters(x, None, A[:0], Bm[:0], ints([0] * 10)).any()


@pytest.mark.parametrize("M", [1024, 1025, 8192, 8193, 9001])
@pytest.mark.parametrize("n", [3, 1500])
def test_sorts_of_many_rows(gpu_lib, M, n):
    """One row of a sorting thread, up to eight, and more of them; fewer and more adapters than sorting threads."""
    which = [(m * 7919) % (n + 2) - 1 for m in range(M)]
    run(M, 64, (40,), n, 8, BF16, BF16, which, ranks=[a % 9 for a in range(n)], seed=M)


def test_most_rows(gpu_lib):
    """2^22 rows: the largest call.  The reference in float64, gathered on the GPU; the tolerance is verify's."""
    M, K, N, n, R = 1 << 22, 8, 8, 4095, 2
    x, base, A, Bm = inputs(M, K, (N,), n, R, BF16, F32)
    which = (torch.arange(M, device="cuda") * 7919 % (n + 1) - 1).to(torch.int32)
    got = B.adapters(x, base, A, Bm, which)
    w = which.clamp(min=0).long()
    has = (which >= 0).double()[:, None]
    prod = A[w, 0].double() * x.double()[:, None, :]                      # [M, R, K]
    terms = Bm[w].double()                                                # [M, N, R]
    ref = base.double() + has * (terms * prod.sum(-1)[:, None, :]).sum(-1)
    mass = has * (terms.abs() * prod.abs().sum(-1)[:, None, :]).sum(-1)
    u = 2.0 ** -24
    tol = (K + 3 * R + 8) * u * mass * 1.01
    tol += 2 * u * (ref.abs() + tol) * 1.01 + 1e-37
    assert bool(((got.double() - ref).abs() <= tol).all())
    assert torch.equal(got[which < 0], base[which < 0])


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("M,K,widths,n,R", [(8200, 33, (77, 9), 4, 5), (8200, 24, (64, 40), 4, 70), (400, 64, (12280, 8), 3, 40), (2100, 39, (2000, 3), 5, 35),
                                            (33000, 8, (520,), 3, 8)])
def test_workgroups_of_more_columns(gpu_lib, M, K, widths, n, R, dtype, kind):
    """As many workgroups of 512 columns as CUs, and enough for 1024."""
    run(M, K, widths, n, R, dtype, kind, [(m * 7) % (n + 1) - 1 for m in range(M)], [max(1, R - 3 * a) for a in range(n)], [1.0 - a for a in range(n)])
