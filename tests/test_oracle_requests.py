"""The float64 oracle of the operators for batches of many requests against other forms of the same formulas."""
import numpy as np
import pytest

from oracle import operators as oo


@pytest.mark.parametrize("block,prefix", [(0, 0), (1, 0), (1, 3), (4, 0)])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (3.0, False), (0.0, True)])
def test_shared_attention_is_attention_over_both_lists_of_keys(block, prefix, cap, bias):
    """A document behind P keys is one document of P + S keys whose first P + prefix are visible to all (blocks of a length
    that P is a multiple of stay where they are)."""
    r = np.random.default_rng(1)
    T, S, P, Hq, Hkv, hd = 5, 7, 8, 4, 2, 6
    q, k, v = r.normal(size=(T, Hq, hd)), r.normal(size=(S, Hkv, hd)), r.normal(size=(S, Hkv, hd))
    pk, pv = r.normal(size=(P, Hkv, hd)), r.normal(size=(P, Hkv, hd))
    slopes = 0.5 ** np.arange(1, Hq + 1) if bias else None
    for pos in (S - T, 0):
        got = oo.shared_attention(q, k, v, pk, pv, pos, block, prefix, 0.3, cap, slopes)
        ref = oo.attention(q, np.concatenate([pk, k]), np.concatenate([pv, v]), P + pos, block, P + prefix, 0.3, cap, slopes)
        for a, b in zip(got, ref):
            np.testing.assert_allclose(a, b, rtol=1e-12, atol=1e-12)


def test_shared_attention_without_any_key():
    z = np.zeros((0, 1, 4))
    out = oo.shared_attention(np.ones((2, 1, 4)), z, z, z, z, 0)[0]
    assert (out == 0).all()
    pv = np.arange(8.0).reshape(2, 1, 4)
    np.testing.assert_allclose(oo.shared_attention(np.ones((1, 1, 4)), z, z, np.zeros((2, 1, 4)), pv, 0)[0][0, 0], pv.mean((0, 1)))


def test_adapters_are_one_dense_product_each():
    r = np.random.default_rng(2)
    M, K, n, R, ends = 6, 5, 3, 4, [2, 9]
    x, base, A, B = r.normal(size=(M, K)), r.normal(size=(M, 9)), r.normal(size=(n, 2, R, K)), r.normal(size=(n, 9, R))
    which, ranks, scales = [0, 2, -1, 1, 3, 2], [4, 0, 2], [0.5, 3.0, -2.0]
    out, mass = oo.adapters(x, base, A, B, which, ranks, scales, ends)
    for m, a in enumerate(which):
        ref = base[m].copy()
        if 0 <= a < n:
            for s, (c0, c1) in enumerate(((0, 2), (2, 9))):
                ref[c0:c1] += scales[a] * (B[a, c0:c1, :ranks[a]] @ A[a, s, :ranks[a]]) @ x[m]
        np.testing.assert_allclose(out[m], ref, rtol=1e-12, atol=1e-12)
        assert (mass[m] >= np.abs(out[m] - base[m]) - 1e-12).all()
