"""The 64-bit definitions of differential attention and of the gradients, pinned against full attention, closed forms and differences."""
import numpy as np
import pytest

import oracle
from oracle import differential as diff

RNG = np.random.default_rng


def _inputs(seed, B, H, G, n_q, n_k, W, per_head=False):
    r = RNG(seed)
    lam = tuple(r.normal(size=(H, W // 2) if per_head else W // 2) * 0.3 for _ in range(4))
    return r.normal(size=(B, H, n_q, W)), r.normal(size=(B, G, n_k, W)), r.normal(size=(B, G, n_k, W)), lam, r.normal(size=(B, H, n_q, W))


def test_second_map_without_weight_leaves_full_attention():
    """lambda = 0: the first map alone, which is the oracle's full attention of the first halves padded with zeros."""
    q, k, v, _, _ = _inputs(1, 1, 2, 2, 12, 12, 64)
    q, k, v = (x.astype(np.float32) for x in (q, k, v))
    zero = tuple(np.zeros(32) for _ in range(4))
    o, _ = diff.diff_attn(q, k, v, zero, 0.0)
    half = [np.concatenate([x[..., :32], np.zeros_like(x[..., 32:])], -1) for x in (q, k)]
    np.testing.assert_allclose(o, oracle.full_attn(*half, v, 1 / np.sqrt(32)), rtol=1e-12, atol=1e-12)


def test_equal_maps_with_weight_one_cancel():
    q, k, v, _, _ = _inputs(2, 2, 2, 1, 9, 7, 64)
    q[..., 32:], k[..., 32:] = q[..., :32], k[..., :32]
    zero = tuple(np.zeros(32) for _ in range(4))
    o, _ = diff.diff_attn(q, k, v, zero, 1.0)
    assert np.abs(o).max() < 1e-14


def test_rows_that_see_nothing_and_padding_that_is_not_read():
    q, k, v, lam, d_o = _inputs(3, 2, 2, 2, 6, 4, 64)
    lens = dict(q_lengths=[6, 3], k_lengths=[4, 0], causal=True)
    o, g = diff.diff_attn(q, k, v, lam, 0.5, d_o=d_o, **lens)
    assert not o[0, :, :2].any() and o[0, :, 2:].all() and not o[1].any()
    for x in (q, k, v, d_o):
        x[1] = np.nan
    o2, g2 = diff.diff_attn(q, k, v, lam, 0.5, d_o=d_o, **lens)
    assert np.array_equal(o, o2) and all(np.array_equal(g[x], g2[x]) for x in "qkv")


@pytest.mark.parametrize("causal,group,per_head,lengths", [(False, 1, False, None), (True, 2, True, ([5, 2, 0], [7, 5, 3]))])
def test_gradients_are_those_of_differences(causal, group, per_head, lengths):
    B, H, n_q, n_k, W = 3, 2, 5, 7, 8
    q, k, v, lam, d_o = _inputs(4, B, H, H // group, n_q, n_k, W, per_head)
    kw = dict(causal=causal)
    if lengths:
        kw.update(q_lengths=lengths[0], k_lengths=lengths[1])
    _, g = diff.diff_attn(q, k, v, lam, 0.4, d_o=d_o, **kw)

    def loss(q, k, v, lam):
        return (diff.diff_attn(q, k, v, lam, 0.4, **kw)[0] * d_o).sum()
    step, r = 1e-5, RNG(5)
    for name, at in (("q", 0), ("k", 1), ("v", 2)):
        for _ in range(6):
            way = r.normal(size=(q, k, v)[at].shape)
            args = [[x + s * way if i == at else x for i, x in enumerate((q, k, v))] for s in (step, -step)]
            slope = (loss(*args[0], lam) - loss(*args[1], lam)) / (2 * step)
            assert abs(slope - (g[name] * way).sum()) < 1e-7 * max(1, abs(slope))
    for i in range(4):
        way = r.normal(size=lam[i].shape)
        both = [tuple(x + s * way if j == i else x for j, x in enumerate(lam)) for s in (step, -step)]
        slope = (loss(q, k, v, both[0]) - loss(q, k, v, both[1])) / (2 * step)
        assert abs(slope - (g["lam"][i] * way).sum()) < 1e-7 * max(1, abs(slope))


def test_layernorm_gradient_is_that_of_differences():
    r = RNG(6)
    x, gamma, dy, eps = r.normal(size=(3, 24)) + 2, r.normal(size=24), r.normal(size=(3, 24)), 1e-3
    beta = r.normal(size=24)

    def loss(x, gamma, beta):
        c = x - x.mean(1, keepdims=True)
        return ((c / np.sqrt((c * c).mean(1, keepdims=True) + eps) * gamma + beta) * dy).sum()
    dx, dgamma, dbeta = diff.layernorm_grad(x, gamma, dy, eps)
    step = 1e-5
    for i, (value, grad) in enumerate(((x, dx), (gamma, dgamma), (beta, dbeta))):
        way = r.normal(size=value.shape)
        ends = [loss(*[a + s * way if j == i else a for j, a in enumerate((x, gamma, beta))]) for s in (step, -step)]
        assert abs((ends[0] - ends[1]) / (2 * step) - (grad * way).sum()) < 1e-7
    # a row of one value: xh = 0, dx = (g - mean(g)) / sqrt(eps)
    flat, _, _ = diff.layernorm_grad(np.full((1, 24), 3.0), gamma, dy[:1], eps)
    g = dy[:1] * gamma
    np.testing.assert_allclose(flat, (g - g.mean()) / np.sqrt(eps), rtol=1e-12)
