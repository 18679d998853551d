"""dllm_sample against the float64 oracle: tokens equal, conf and prob to float32
accuracy (weights of float32 exponents within 2^-20, one rounding: 2^-19)."""
import math

import numpy as np
import pytest
import torch

from helpers import say, to_np
from oracle import operators as oo
from paper_2608_22646_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def randn(shape, dtype, seed, std):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype)


def uniform(n, seed, lo=0.0, hi=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.rand(n, generator=g) * (hi - lo) + lo).float()


def check(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, mask_id=-1, got=None):
    cuda = lambda t: None if t is None else t.cuda()  # noqa: E731
    if got is None:
        got = B.sample(logits.cuda(), u.cuda(), cuda(temperature), cuda(top_k), cuda(top_p), cuda(min_p), mask_id)
    token, conf, prob = (t.cpu().numpy() for t in got)
    x = to_np(logits, np.float64)
    for r in range(len(x)):
        one = lambda t, d: d if t is None else float(t[r])  # noqa: E731
        t, c, p = oo.sample(x[r], float(u[r]), one(temperature, 1.0), int(one(top_k, 0)), one(top_p, 1.0), one(min_p, 0.0), mask_id)
        assert token[r] == t, f"row {r}: token {token[r]} (prob {prob[r]:.3g}) and not {t} (prob {p:.3g})"
        np.testing.assert_allclose([conf[r], prob[r]], [c, p], rtol=2.0 ** -19, atol=1e-37, err_msg=f"row {r}")
    return token, conf, prob


def controls(R, V, seed, which):
    g = torch.Generator().manual_seed(seed)
    c = {}
    if "t" in which:
        c["temperature"] = uniform(R, seed + 1, 0.2, 2.0)
    if "k" in which:
        c["top_k"] = torch.randint(1, max(2, min(V, 1000)), (R,), generator=g).to(torch.int32)
    if "p" in which:
        c["top_p"] = uniform(R, seed + 2, 0.1, 1.0)
    if "m" in which:
        c["min_p"] = uniform(R, seed + 3, 0.0, 0.2)
    return c


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,V", [(1, 1), (3, 2), (5, 63), (2, 1000), (40, 2048), (9, 3001), (3, 50257), (33, 16384), (2, 152064)])
@pytest.mark.parametrize("which", ["", "t", "k", "p", "m", "tkpm", "tp", "km"])
def test_matches_the_oracle(gpu_lib, R, V, which, dtype):
    say(f"sample {R}x{V} {which} {dtype}")
    for std in (1.2, 6.0):
        seed = R * 1000 + V + len(which)
        check(randn((R, V), dtype, seed, std), uniform(R, seed + 9), mask_id=V - 1 if V > 1 else -1, **controls(R, V, seed, which))


def test_many_random_numbers(gpu_lib):
    """One row's distribution at 4000 random numbers, its borders among them."""
    say("sample many u")
    lg = randn((1, 300), F32, 5, 2.0)
    p = np.exp(to_np(lg[0], np.float64))
    edge = np.cumsum(p / p.sum())[:-1].astype(np.float32)
    u = torch.from_numpy(np.concatenate([uniform(3400, 1).numpy(), edge, np.nextafter(edge, np.float32(0))]))
    check(lg.expand(len(u), 300).contiguous(), u)
    check(lg.expand(len(u), 300).contiguous(), u, top_p=torch.full((len(u),), 0.7), temperature=torch.full((len(u),), 0.8))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [70, 5000, 40000])
def test_ties(gpu_lib, V, dtype):
    """Equal logits: all of them, two levels, few levels; every cut falls inside a tie, and lower indices stay."""
    say(f"sample ties {V} {dtype}")
    R = 24
    u = uniform(R, 3)
    k = torch.randint(1, V, (R,), generator=torch.Generator().manual_seed(4)).to(torch.int32)
    p = uniform(R, 5, 0.05, 0.95)
    flat = torch.full((R, V), 1.5).to(dtype)
    two = flat.clone()
    two[:, V // 3: V // 2] = 3.0
    levels = torch.randint(0, 5, (R, V), generator=torch.Generator().manual_seed(6)).to(dtype)
    for x in (flat, two, levels):
        check(x, u, top_k=k)
        check(x, u, top_p=p)
        check(x, u, top_k=k, top_p=p, temperature=uniform(R, 7, 0.3, 2.0), mask_id=2)
    # -0 and +0 are equal: the lower index is first
    z = torch.zeros((2, V)).to(dtype)
    z[0, 0], z[1, 1:] = -0.0, -0.0
    check(z, torch.tensor([0.9, 0.9]), top_k=torch.tensor([1, 1], dtype=torch.int32))


@pytest.mark.parametrize("many", [100, 9000])
def test_boundary_far_from_top_ks(gpu_lib, many):
    """Few members where top-k cuts, and top-p's share of them reaching over empty ranks into
    many (9000: more than are listed of a row): one logit of 0, many about -0.26 (the largest amid
    them), sixty about -3.47 of which thirty stay."""
    say(f"sample boundary far from top-k's {many}")
    n, R = 300 + many, 64
    lg = torch.full((n,), -30.0)
    lg[17] = 0.0
    lg[100:100 + many] = -3 / 8 * math.log(2) - 1e-3 / many * (torch.arange(many) - many // 2 - 1).abs()
    lg[150 + many:210 + many] = -5 * math.log(2) + 1e-4 * (torch.arange(60) % 7)
    u = torch.arange(R) / R
    mass = 1 + many * 2 ** -0.375
    for share in (1.004, 1.012, 1.83, 3.97, 0.3 * many):
        _, _, prob = check(lg.expand(R, n).contiguous(), u, top_k=torch.full((R,), many + 31, dtype=torch.int32),
                           top_p=torch.full((R,), share / (mass + 0.94)))
    assert prob.max() < 1


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("seed", range(4))
def test_clustered_logits(gpu_lib, seed, dtype):
    """Rows whose logits lie in few narrow clusters of very unlike sizes, with gaps and ties between."""
    say(f"sample clusters {seed} {dtype}")
    R, V = 300, [257, 700, 1200, 9000][seed]
    g = torch.Generator().manual_seed(100 + seed)
    sizes = torch.tensor([1.0, 1, 2, 5, 30, 60, 100, V / 2])
    at = torch.rand(R, 8, generator=g) * 6 * (torch.rand(R, 1, generator=g) > 0.2)
    which = torch.multinomial(sizes.expand(R, 8), V, replacement=True, generator=g)
    step = 10.0 ** -torch.randint(1, 7, (R, 1), generator=g).float()
    lg = -at.gather(1, which) - step * torch.randint(0, 50, (R, V), generator=g) + 3
    which = torch.rand(R, generator=g)
    check(lg.to(dtype), uniform(R, seed + 1), temperature=uniform(R, seed + 2, 0.3, 3.0),
          top_k=torch.where(which < 0.7, torch.randint(1, V, (R,), generator=g), 0).to(torch.int32),
          top_p=torch.where(which > 0.2, uniform(R, seed + 3) ** 2, 1.0), min_p=torch.where(which > 0.8, uniform(R, seed + 4), 0.0))


def test_control_values(gpu_lib):
    """Every control at, around and beyond its ends, in one batch; rows are independent."""
    say("sample control values")
    V = 700
    inf, nan = math.inf, math.nan
    rows = [(t, k, p, m, u)
            for t in (0.0, -1.0, nan, inf, 1e-3, 1e-30, 1e30, 1.0) for k, p, m in
            ((0, 1.0, 0.0), (1, 1.0, 0.0), (V, 0.5, 0.0), (V + 5, nan, nan), (-3, 0.0, 0.0), (5, -1.0, 0.0), (0, 2.0, 1.0), (0, 1.0, 7.0),
             (20, 0.999, 1e-6), (2 ** 31 - 1, 1e-9, -1.0), (-2 ** 31, inf, inf)) for u in (0.0, 0.37, 1.0, -2.0, nan)]
    t, k, p, m, u = (list(c) for c in zip(*rows))
    lg = randn((1, V), F32, 8, 3.0).expand(len(rows), V).contiguous()
    check(lg, torch.tensor(u), torch.tensor(t), torch.tensor(k, dtype=torch.int32), torch.tensor(p), torch.tensor(m), mask_id=1)


@pytest.mark.parametrize("V", [90, 20000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masked_and_broken_rows(gpu_lib, V, dtype):
    say(f"sample masked rows {V} {dtype}")
    inf, low = math.inf, torch.finfo(dtype).min
    x = randn((13, V), dtype, 9, 3.0)
    x[0, :] = -inf                                   # no candidate
    x[1, :], x[1, 7] = -inf, 2.0                     # one
    x[2, 5:] = -inf
    x[3, :] = low                                    # the type's lowest value everywhere
    x[4, :], x[4, V - 2] = low, 0.0
    x[5, 30], x[5, 20] = math.nan, inf
    x[6, V - 1] = math.nan
    x[7, 11], x[7, 3] = inf, -inf
    x[8, 4] = math.nan                               # the mask token's own logit is never looked at
    x[9, 4] = inf
    x[10, :], x[10, 4] = -inf, 1.0                   # nothing but the mask token
    x[11, :] = torch.finfo(dtype).max
    x[12, 0], x[12, 1] = torch.finfo(dtype).max, low
    u = uniform(13, 10)
    ones = torch.ones(13)
    for c in ({}, dict(temperature=ones * 0.5, top_k=(ones * 3).int()), dict(top_p=ones * 0.6), dict(min_p=ones * 0.1),
              dict(temperature=ones * 0), dict(temperature=ones * 1e-20), dict(temperature=ones * 1e20, top_k=(ones * 50).int(), top_p=ones * 0.5)):
        token, conf, prob = check(x, u, mask_id=4, **c)
        assert token[0] == -1 and token[10] == -1 and token[5] == 20 and math.isnan(conf[5])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_any_stride_and_alignment(gpu_lib, dtype):
    say(f"sample strides {dtype}")
    R, V = 6, 4099
    wide = randn((R, V + 14), dtype, 11, 3.0).cuda()
    wide[:, V + 3:] = math.nan
    wide[:, :3] = math.nan
    u = uniform(R, 12)
    x = wide[:, 3:V + 3]
    check(x.cpu(), u, got=B.sample(x, u.cuda(), top_p=torch.full((R,), 0.9, device="cuda")), top_p=torch.full((R,), 0.9))
    x = wide[::2, 3:V + 3]
    check(x.cpu(), u[:3], got=B.sample(x, u[:3].cuda()))


def test_greedy_is_the_heads_answer(gpu_lib):
    """Temperature 0 on the head's logits: dllm_head's argmax, and its confidence to float32 accuracy."""
    from paper_2608_22646_amd import synth
    say("sample greedy against the head")
    cfg = synth.TINY
    model = B.Model(cfg, synth.make_weights(cfg, "cuda"))
    x = synth.make_ints((2, 40), 3, 0, cfg.vocab - 1).cuda()
    conf, arg, lg = model.forward(x, 8, 32, logits=True)
    n = 64
    token, c, p = B.sample(lg.view(n, -1), torch.rand(n, device="cuda"), temperature=torch.zeros(n, device="cuda"), mask_id=cfg.mask_id)
    assert torch.equal(token.view(2, 32), arg) and (p == 1).all()
    assert (c.view(2, 32) / conf - 1).abs().max() <= 2.0 ** -18      # each side within 2^-19


def test_repeats_streams_and_graphs(gpu_lib):
    say("sample repeats, streams, graphs")
    R, V = 20, 60000
    x, u = randn((R, V), F32, 13, 2.0).cuda(), uniform(R, 14).cuda()
    c = {k: v.cuda() for k, v in controls(R, V, 15, "tkpm").items()}
    want = B.sample(x, u, **c)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(B.sample(x, u, **c), want))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = B.sample(x, u, stream=s, **c)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    n = B.sample_workspace_size(R, V)
    ws = B.device_buffer(n) if n else None
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = B.sample(x, u, ws=ws, **c)
    for i in range(3):
        x.copy_(randn((R, V), F32, 20 + i, 2.0 + i))
        u.copy_(uniform(R, 30 + i))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(B.sample(x, u, **c), out))


def test_binding_checks_shapes(gpu_lib):
    x, u = torch.zeros((3, 50), device="cuda"), torch.zeros(3, device="cuda")
    for call in (lambda: B.sample(x.half(), u), lambda: B.sample(x, u[:2]), lambda: B.sample(x, u, top_k=u), lambda: B.sample(x[0], u),
                 lambda: B.sample(x.t(), torch.zeros(50, device="cuda")), lambda: B.sample(x, u.double()), lambda: B.sample(x, u, top_p=u.cpu())):
        with pytest.raises(B.DllmError):
            call()
    assert B.sample(x[:0], u[:0])[0].shape == (0,)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R", [255, 256, 257, 300, 600])
def test_rows_of_one_chunk(gpu_lib, R, dtype):
    """Vocabularies of at most one chunk, on both sides of the row count up to which one launch does it all."""
    for V in (700, 8192):
        say(f"sample one chunk {R}x{V} {dtype}")
        lg = randn((R, V), dtype, R + V, 2.0)
        lg[3], lg[4, 5], lg[5] = -math.inf, math.nan, 0.0
        c = controls(R, V, R, "tkpm")
        c["temperature"][7] = 0.0
        check(lg, uniform(R, V), mask_id=9, **c)
