"""The operators' oracle against library routines and worked examples (CPU only)."""
import math

import numpy as np
import pytest
import torch

from oracle import operators as oo


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_is_a_complex_rotation(interleaved):
    rng = np.random.default_rng(1)
    x, pos = rng.normal(size=(2, 5, 3, 16)), rng.integers(-50, 5000, size=(2, 5))
    rates = oo.rotary_rates(12)
    y = oo.rotary(x, pos, rates, interleaved, gain=1.25)
    z = (x[..., 0:12:2] + 1j * x[..., 1:12:2]) if interleaved else (x[..., :6] + 1j * x[..., 6:12])
    z = z * 1.25 * np.exp(1j * pos[:, :, None, None] * rates)
    got = (y[..., 0:12:2] + 1j * y[..., 1:12:2]) if interleaved else (y[..., :6] + 1j * y[..., 6:12])
    np.testing.assert_allclose(got, z, atol=1e-12)
    np.testing.assert_array_equal(y[..., 12:], x[..., 12:])
    np.testing.assert_allclose(oo.rotary(oo.rotary(x, pos, rates, interleaved), pos, rates, interleaved, inverse=True), x,
                               atol=1e-12)


def test_rotary_scalings():
    f = oo.rotary_rates(64, base=1e4)
    np.testing.assert_allclose(oo.rotary_rates(64, base=1e4, scaling="linear", factor=4), f / 4)
    parts = oo.rotary_rates(64, base=1e4, scaling="parts", factor=8, orig_len=4096, low=1, high=32)
    turns = 4096 * f / (2 * math.pi)
    np.testing.assert_allclose(parts[turns >= 32], f[turns >= 32])
    np.testing.assert_allclose(parts[turns <= 1], f[turns <= 1] / 8)
    assert ((parts >= f / 8 * (1 - 1e-12)) & (parts <= f * (1 + 1e-12))).all()


@pytest.mark.parametrize("block,prefix,cap,bias", [(0, 0, 0, 0), (1, 0, 0, 0), (1, 5, 0, 1), (4, 0, 20.0, 0), (4, 6, 5.0, 1)])
def test_attention_is_masked_softmax(block, prefix, cap, bias):
    rng = np.random.default_rng(2)
    T, S, Hq, Hkv, hd, pos = 7, 13, 4, 2, 8, 6
    q, k, v = rng.normal(size=(T, Hq, hd)), rng.normal(size=(S, Hkv, hd)), rng.normal(size=(S, Hkv, hd))
    slopes = np.array([0.5, 0.25, 0.1, 0.0]) if bias else None
    got, mass, _, _ = oo.attention(q, k, v, pos, block, prefix, None, cap, slopes)
    t = lambda x, r: torch.from_numpy(np.repeat(x, r, axis=1)).permute(1, 0, 2)  # noqa: E731
    i, j = torch.arange(T)[:, None] + pos, torch.arange(S)[None]
    add = torch.zeros((Hq, T, S), dtype=torch.float64)
    if bias:
        add -= torch.from_numpy(slopes)[:, None, None] * (i - j).abs()
    if block:
        add = add.masked_fill(~((j // block <= i // block) | (j < prefix)), -math.inf)
    Q, K, V = t(q, 1), t(k, Hq // Hkv), t(v, Hq // Hkv)
    if cap:
        s = cap * torch.tanh(Q @ K.transpose(1, 2) / math.sqrt(hd) / cap) + add
        ref = torch.softmax(s, -1) @ V
    else:
        ref = torch.nn.functional.scaled_dot_product_attention(Q, K, V, attn_mask=add)
    np.testing.assert_allclose(got, ref.permute(1, 0, 2).numpy(), atol=1e-12)
    assert (mass >= np.abs(got) - 1e-12).all()


def test_attention_without_visible_keys_is_zero():
    q, k = np.ones((3, 1, 4)), np.ones((5, 1, 4))
    out, _, _, _ = oo.attention(q, k, k, -2, block=1)          # positions -2, -1, 0
    np.testing.assert_array_equal(out[:2], 0)
    np.testing.assert_array_equal(out[2], 1)


def test_sample_worked_examples():
    lg = np.log([0.1, 0.4, 0.2, 0.3])
    # all kept: cumulative 0.1, 0.5, 0.7, 1
    assert [oo.sample(lg, u)[0] for u in (0.0, 0.05, 0.11, 0.49, 0.51, 0.71, 0.999)] == [0, 0, 1, 1, 2, 3, 3]
    # top_k 2: tokens 1 and 3, shares 4/7 and 3/7
    assert [oo.sample(lg, u, top_k=2)[0] for u in (0.0, 0.57, 0.58)] == [1, 1, 3]
    assert oo.sample(lg, 0.0, top_k=2)[2] == pytest.approx(4 / 7)
    # top_p: ranked masses before: 0, .4, .7, .9
    assert [oo.sample(lg, 0.999, top_p=p)[0] for p in (0.0, 0.39, 0.41, 0.71)] == [1, 1, 3, 3]
    assert oo.sample(lg, 0.0, top_p=0.91)[0] == 0
    # min_p: weights relative to the largest: .25, 1, .5, .75
    assert oo.sample(lg, 0.0, min_p=0.3)[0] == 1 and oo.sample(lg, 0.0, min_p=0.2)[0] == 0
    assert oo.sample(lg, 0.999, min_p=5.0)[0] == 1
    # greedy, masked, ties to the lowest index, no candidate, NaN
    assert oo.sample(lg, 0.9, temperature=0.0) == (1, pytest.approx(0.4), 1.0)
    assert oo.sample(lg, 0.9, temperature=0.0, mask_id=1)[0] == 3
    assert oo.sample([1.0, 2.0, 2.0], 0.999, top_k=1)[0] == 1
    assert oo.sample([-np.inf, 3.0], 0.5, mask_id=1) == (-1, 0.0, 0.0)
    assert oo.sample([0.0, np.nan, np.inf], 0.5)[0] == 1
    # temperature sharpens: weights 1/16, 1, 1/4, 9/16
    assert oo.sample(lg, 0.0, temperature=0.5)[2] == pytest.approx(0.01 / 0.30)
