"""The 64-bit oracle of the attention block's operators, without a GPU: its gradients against central differences of
its own forward passes, and the properties that the formulas fix."""
import numpy as np
import pytest

from oracle import block as K


def _difference(f, x, direction, h=1e-5):
    return (f(x + h * direction) - f(x - h * direction)) / (2 * h)


@pytest.mark.parametrize("c", [1, 2, 7, 16])
def test_layernorm_gradients_are_differences(c):
    rng = np.random.default_rng(c)
    x, r, dy, d = (rng.normal(size=(5, c)) for _ in range(4))
    g, b, dg = rng.normal(size=c), rng.normal(size=c), rng.normal(size=c)
    eps = 1e-3
    s, _, stats = K.layernorm_fwd(x, r, g, b, eps)
    dx, dgamma, dbeta = K.layernorm_bwd(s, stats, g, dy, None)
    loss = lambda x_, g_, b_: (K.layernorm_fwd(x_, r, g_, b_, eps)[1] * dy).sum()
    assert _difference(lambda t: loss(t, g, b), x, d) == pytest.approx((dx * d).sum(), rel=1e-6, abs=1e-8)
    assert _difference(lambda t: loss(x, t, b), g, dg) == pytest.approx((dgamma * dg).sum(), rel=1e-6, abs=1e-8)
    assert _difference(lambda t: loss(x, g, t), b, dg) == pytest.approx((dbeta * dg).sum(), rel=1e-6, abs=1e-8)


def test_rope_turns_and_turns_back():
    rng = np.random.default_rng(3)
    x, pos = rng.normal(size=(9, 3 * 14)), rng.integers(-5, 500, size=(9, 3))
    y = K.rope(x, pos, 3, 2, 14, (3, 2, 1), 100.0, 0.5)
    assert np.allclose(K.rope(y, pos, 3, 2, 14, (3, 2, 1), 100.0, 0.5, inverse=True), x, atol=1e-12)
    assert np.array_equal(y[:, 28:], x[:, 28:])                      # the third head
    assert np.array_equal(y.reshape(9, 3, 14)[:, :, 12:], x.reshape(9, 3, 14)[:, :, 12:])
    # the product of a query and a key depends on the difference of their positions alone
    q, k = rng.normal(size=(1, 14)), rng.normal(size=(1, 14))
    at = lambda v, p: K.rope(v, np.array([p]), 1, 1, 14, (3, 2, 1), 100.0, 1.0)
    a = (at(q, (5, 9, 2)) * at(k, (1, 4, 7))).sum()
    b = (at(q, (105, 29, 42)) * at(k, (101, 24, 47))).sum()
    assert a == pytest.approx(b, rel=1e-9)


@pytest.mark.parametrize("hq,hkv,masked", [(1, 1, False), (4, 2, True), (3, 1, True)])
def test_attention_gradients_are_differences(hq, hkv, masked):
    rng = np.random.default_rng(hq)
    d, qo, ko = 5, [0, 3, 3, 7], [0, 4, 9, 11]
    q, do, u = (rng.normal(size=(7, hq * d)) for _ in range(3))
    k, v, w = (rng.normal(size=(11, hkv * d)) for _ in range(3))
    mask = None
    if masked:
        mask = rng.random(11) < 0.6
        mask[9:] = False                                              # the last shape sees nothing
    args = (qo, ko, mask, hq, hkv, d, 0.7)
    r = K.attention(q, k, v, *args, do=do)
    if masked:
        assert not r["o"][3:].any() and np.isneginf(r["lse"][3:]).all() and not r["dq"][3:].any() and not r["dk"][9:].any()
    loss = lambda q_, k_, v_: (K.attention(q_, k_, v_, *args)["o"] * do).sum()
    assert _difference(lambda t: loss(t, k, v), q, u) == pytest.approx((r["dq"] * u).sum(), rel=1e-6, abs=1e-8)
    assert _difference(lambda t: loss(q, t, v), k, w) == pytest.approx((r["dk"] * w).sum(), rel=1e-6, abs=1e-8)
    assert _difference(lambda t: loss(q, k, t), v, w) == pytest.approx((r["dv"] * w).sum(), rel=1e-6, abs=1e-8)
