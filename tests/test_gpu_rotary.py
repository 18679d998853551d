"""dllm_rotary against the float64 oracle.

Tolerance: each output is a cos - b sin with float32 sines (quarter-turn remainder
rounded to float32, sine and cosine within two units, the gain's product: six
half-steps together), two products and a sum (three more), and one rounding to the
type; an angle p f carries p f 2^-48 from the float64 rates of both sides."""
import numpy as np
import pytest
import torch

from helpers import say, to_np
from oracle import operators as oo
from paper_2608_22646_amd import binding as B

pytestmark = pytest.mark.gpu


def check(got, x, pos, kw, dtype, inverse):
    rates = oo.rotary_rates(kw["rot_dim"], kw.get("base", 1e4), kw.get("scaling", "none"), kw.get("factor", 1.0),
                            kw.get("orig_len", 0.0), kw.get("low", 1.0), kw.get("high", 32.0))
    gain = kw.get("gain", 1.0)
    x64 = to_np(x, np.float64)
    ref = oo.rotary(x64, pos, rates, kw.get("interleaved", False), gain, inverse)
    rot, u = kw["rot_dim"], 2.0 ** -24
    big = np.zeros_like(x64)
    a = np.abs(x64[..., :rot])
    pair = a[..., 0::2] + a[..., 1::2] if kw.get("interleaved") else a[..., :rot // 2] + a[..., rot // 2:]
    far = 9 * u + np.abs(np.asarray(pos, dtype=np.float64))[:, :, None, None] * rates * 2.0 ** -48
    both = pair * far * abs(gain)
    big[..., :rot] = np.repeat(both, 2, -1) if kw.get("interleaved") else np.concatenate([both, both], -1)
    tol = torch.finfo(dtype).eps / 2 * np.abs(ref) * 1.01 + big
    err = np.abs(to_np(got, np.float64) - ref)
    assert (err <= tol).all(), f"{(err > tol).sum()} elements off, worst {(err / np.maximum(tol, 1e-30)).max():.3g} tolerances"
    assert torch.equal(got[..., rot:].contiguous().view(torch.uint8), x[..., rot:].contiguous().view(torch.uint8))


def tensors(shape, n_k, dtype, seed, layout="plain"):
    g = torch.Generator().manual_seed(seed)
    Bn, L, H, hd = shape
    if layout == "packed":      # q and k inside a packed projection
        x = torch.randn((Bn, L, H + 2 * n_k, hd), generator=g).to(dtype).cuda()
        return x[:, :, :H], x[:, :, H:H + n_k]
    if layout == "heads":       # [B, H, L, hd]
        x = torch.randn((Bn, H + n_k, L, hd), generator=g).to(dtype).cuda().transpose(1, 2)
        return x[:, :, :H], x[:, :, H:]
    if layout == "odd":         # rows that start at no multiple of 16 bytes
        x = torch.randn((Bn, L, H + n_k, hd + 3), generator=g).to(dtype).cuda()[..., 1:hd + 1]
        return x[:, :, :H], x[:, :, H:]
    x = torch.randn((Bn, L, H, hd), generator=g).to(dtype).cuda()
    return x, torch.randn((Bn, L, n_k, hd), generator=g).to(dtype).cuda()


CASES = [
    ((1, 1, 1, 64), 1, dict(rot_dim=64), "plain"),
    ((2, 7, 4, 128), 2, dict(rot_dim=128), "packed"),
    ((3, 33, 5, 128), 1, dict(rot_dim=64, interleaved=True), "packed"),
    ((2, 19, 4, 64), 4, dict(rot_dim=32, base=5e5), "heads"),
    ((2, 19, 4, 64), 4, dict(rot_dim=64, interleaved=True), "heads"),
    ((1, 9, 3, 80), 2, dict(rot_dim=20), "plain"),               # no whole pieces
    ((1, 9, 3, 80), 2, dict(rot_dim=20, interleaved=True), "plain"),
    ((1, 5, 2, 128), 2, dict(rot_dim=128), "odd"),
    ((1, 5, 2, 128), 2, dict(rot_dim=126, interleaved=True), "odd"),
    ((1, 3, 2, 2), 1, dict(rot_dim=2), "plain"),
    ((1, 3, 2, 3), 1, dict(rot_dim=2, interleaved=True), "plain"),
    ((1, 4, 2, 512), 1, dict(rot_dim=256), "plain"),
    ((1, 2100, 28, 128), 4, dict(rot_dim=128, base=1e6, scaling="parts", factor=16.0, orig_len=8192, gain=1.28), "packed"),
    ((2, 40, 4, 128), 4, dict(rot_dim=128, scaling="linear", factor=4.0, gain=-0.5), "plain"),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_rotary_matches_the_oracle(gpu_lib, i, dtype):
    shape, n_k, kw, layout = CASES[i]
    say(f"rotary {shape} {n_k} {kw} {layout} {dtype}")
    q, k = tensors(shape, n_k, dtype, i, layout)
    Bn, L = shape[:2]
    g = torch.Generator().manual_seed(100 + i)
    pos = torch.randint(-1000, 1 << 20, (Bn, L), generator=g, dtype=torch.int64).to(torch.int32)
    cfg = B.Rotary(head_dim=shape[3], **kw)
    for inverse in (False, True):
        qo, ko = B.rotary(cfg, q, k, pos=pos.cuda(), inverse=inverse)
        check(qo, q, pos.numpy(), kw, dtype, inverse)
        check(ko, k, pos.numpy(), kw, dtype, inverse)


def test_rotary_positions(gpu_lib):
    """No array: pos0 + l.  The ends of int32 (the tolerance takes their angle's float64 rounding into account)."""
    q, _ = tensors((2, 6, 2, 64), 1, torch.float32, 3)
    kw = dict(rot_dim=64)
    say("rotary pos0")
    out, none = B.rotary(B.Rotary(64), q, pos0=17)
    assert none is None
    check(out, q, np.arange(6)[None] + 17 + np.zeros((2, 1)), kw, torch.float32, False)
    pos = torch.tensor([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 123456789]] * 2, dtype=torch.int32)
    out, _ = B.rotary(B.Rotary(64), q, pos=pos.cuda())
    check(out, q, pos.numpy(), kw, torch.float32, False)
    out, _ = B.rotary(B.Rotary(64), q, pos0=2 ** 31 - 3)      # past the end of int32: positions stay whole numbers
    check(out, q, np.arange(6.0)[None] + 2 ** 31 - 3 + np.zeros((2, 1)), kw, torch.float32, False)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_in_place_and_undone(gpu_lib, interleaved):
    say("rotary in place")
    q, k = tensors((2, 50, 4, 128), 2, torch.float32, 4, "packed")
    whole = q._base
    before = whole.clone()
    cfg = B.Rotary(128, 64, interleaved)
    want_q, want_k = B.rotary(cfg, q, k, pos0=5)
    B.rotary(cfg, q, k, pos0=5, q_out=q, k_out=k)
    assert torch.equal(q, want_q) and torch.equal(k, want_k)
    assert torch.equal(whole[:, :, 6:], before[:, :, 6:])      # the values of the projection stay
    B.rotary(cfg, q, k, pos0=5, q_out=q, k_out=k, inverse=True)
    # two rotations of float32: each within 9 half-steps of |a| + |b| plus a rounding
    assert (whole - before).abs().max() <= 24 * 2.0 ** -24 * 2 * before.abs().max()


def test_rotary_inverse_is_the_transpose(gpu_lib):
    """<R x, y> = <x, R^T y>: the direction a gradient takes, gain included."""
    say("rotary transpose")
    x, y = tensors((1, 30, 4, 64), 4, torch.float32, 5)
    cfg = B.Rotary(64, 48, gain=1.5)
    rx, ry = B.rotary(cfg, x, pos0=9)[0], B.rotary(cfg, y, pos0=9, inverse=True)[0]
    left, right = (rx.double() * y.double()).sum(), (x.double() * ry.double()).sum()
    scale = (x.double().abs() * y.double().abs()).sum() * 2 * 1.5
    assert abs(left - right) <= 24 * 2.0 ** -24 * scale


def test_rotary_other_stream_and_graph(gpu_lib):
    say("rotary on another stream, then captured")
    q, k = tensors((1, 16, 4, 128), 4, torch.bfloat16, 6)
    cfg = B.Rotary(128, scaling="parts", factor=8.0, orig_len=4096)
    want = B.rotary(cfg, q, k, pos0=3)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = B.rotary(cfg, q, k, pos0=3, stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    qo, ko = torch.zeros_like(q), torch.zeros_like(k)
    pos = torch.arange(16, dtype=torch.int32, device="cuda")[None] + 3
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.rotary(cfg, q, k, pos=pos, q_out=qo, k_out=ko)
    for step in range(3):
        pos.add_(step)
        q.add_(0.25)
        graph.replay()
        torch.cuda.synchronize()
        ref = B.rotary(cfg, q, k, pos=pos)
        assert torch.equal(qo, ref[0]) and torch.equal(ko, ref[1])


def test_rotary_of_nothing(gpu_lib):
    x = torch.zeros((0, 4, 2, 64), device="cuda")
    assert B.rotary(B.Rotary(64), x)[0].shape == x.shape
