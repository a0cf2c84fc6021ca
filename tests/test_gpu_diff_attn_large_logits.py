"""Gradients of differential attention at logits so large that whole units of log2 lie between neighbouring fp32 numbers: weights are formed again as the forward
pass formed them."""
import numpy as np
import pytest
import torch

import differential as D
from oracle import differential as diff

pytestmark = pytest.mark.gpu

KINDS = [("bf16", 64), ("bf16", 128), ("fp32", 64), ("fp32", 128)]


def same_sum(gen, n, d, total):
    """n rows of d whole numbers between -8 and 8 or so, all of one sum."""
    x = torch.randint(-4, 5, (n, d), generator=gen).float()
    while True:
        rest = total - x.sum(1)
        if not rest.any():
            return x
        at = torch.randint(0, d, (n, 1), generator=gen)
        x.scatter_add_(1, at, rest.clamp(-2, 2)[:, None])


@pytest.mark.parametrize("power", [4, 9, 12, 16, 20, 22, 28, 80])
@pytest.mark.parametrize("n_q,n_k", [(30, 50), (200, 300)])
@pytest.mark.parametrize("dtype,W", KINDS)
def test_gradients_of_equal_logits_of_any_size(dtype, W, n_q, n_k, power):
    """Queries of one power of two and keys of whole numbers with one sum: all logits of a row are the same number, 1e2 to 1e25, exactly, and the
    weights those of logits near zero.  dK is the only result that has the power in it.  (bf16: dK and dV are documented to need logits below 2^20.)"""
    gen = torch.Generator().manual_seed(power + W)
    x = D.make(33, 1, 2, 1, n_q, n_k, W, dtype)
    x["k"][0, 0] = torch.cat([same_sum(gen, n_k, W // 2, total) for total in (24, -40)], 1).to(x["k"].dtype)
    assert x["k"].float().abs().max() < 256
    x["q"][:] = 2.0 ** -20
    want = D.Bounds(x, dtype, backward=True)
    x["q"][:] = 2.0 ** power
    out = D.run(x, backward=True)
    out["k"] = out["k"].float() * 2.0 ** (-20 - power)
    for n in ("o", "q", "k", "v"):
        if dtype == "fp32" or n in "oq":
            D.Bounds.one(n, D.host(out[n]), want.o if n == "o" else want.grad[n], want.off[n])
    for i in range(4):
        D.Bounds.one("lam %d" % i, D.host(out["lam"][i]), want.grad["lam"][i], want.off["lam"][i])


@pytest.mark.parametrize("spread", [3e7, 1e9, 1e12])
@pytest.mark.parametrize("dtype,W", KINDS)
def test_gradients_of_peaked_rows(dtype, W, spread):
    """Logits of such a size leave one weight of 1 a row and map (the largest logit leads by more than its rounding, which the reference is asked for), and
    logit gradients of zero but for the rounding of dP and D.  Weights are formed again from the same scores: any that differed by one
    rounding would be off by 2^(logit 2^-24)."""
    n_q, n_k, d = 130, 200, W // 2
    x = D.make(34, 1, 2, 1, n_q, n_k, W, dtype, spread=spread)
    out = D.run(x, backward=True, d_lam=False)
    q, k, v, do = (D.host(x[n]) for n in ("q", "k", "v", "d_o"))
    value = diff.lambdas(tuple(D.host(t) for t in x["lam"]), 0.5, 2)[0][0]
    s = 2.0 ** -8 if dtype == "bf16" else D.EPS
    want_v, off_v, sure_all = np.zeros_like(v), np.zeros_like(v), 0
    for h in range(2):
        first = []
        sure = np.ones(n_q, bool)
        for m in (0, 1):
            at = slice(m * d, (m + 1) * d)
            logit = q[0, h][:, at] @ k[0, 0][:, at].T
            size = (abs(q[0, h][:, at]) @ abs(k[0, 0][:, at]).T).max(1)
            top = np.sort(logit, 1)
            # a lead of 2 (d + 6) roundings, and of 150 in units of log2 behind the scaling: the second weight is zero
            sure &= top[:, -1] - top[:, -2] > 4 * D.EPS * (d + 6) * size + 150 * d ** 0.5
            first.append(logit.argmax(1))
        sure_all += int(sure.sum())
        o = v[0, 0][first[0]] - value * v[0, 0][first[1]]
        off = 8 * (s + 64 * D.EPS) * (abs(v[0, 0][first[0]]) + abs(value * v[0, 0][first[1]]))
        assert (abs(D.host(out["o"])[0, h] - o) <= off)[sure].all()
        # dS: what is left of dP - D, whose rows of O and P2 V are rounded by s; a weight each, two maps
        ad = abs(do[0, h])
        near = (ad * 4 * off).sum(1) + D.EPS * (W + 8) * 8 * (ad * (abs(v[0, 0][first[0]]) + abs(v[0, 0][first[1]]))).sum(1)
        got = abs(D.host(out["q"])[0, h])
        size = np.concatenate([abs(k[0, 0][first[m]])[:, m * d:(m + 1) * d] for m in (0, 1)], 1) * d ** -0.5 * (1 + abs(value))
        assert np.isfinite(got[sure]).all() and (got <= near[:, None] * size * (1 + 2 * s) + 1e-30)[sure].all(), "dQ"
        for i in range(n_q):
            want_v[0, 0][first[0][i]] += do[0, h, i]
            want_v[0, 0][first[1][i]] -= value * do[0, h, i]
            off_v[0, 0][first[0][i]] += (s + 64 * D.EPS) * ad[i]
            off_v[0, 0][first[1][i]] += (s + 64 * D.EPS) * abs(value) * ad[i]
    print(sure_all, "rows of", 2 * n_q)
    assert sure_all > n_q
    if dtype == "fp32" and sure_all == 2 * n_q:
        D.Bounds.one("dV", D.host(out["v"]), want_v, 8 * off_v + 1e-30)
        assert torch.isfinite(out["k"]).all()
