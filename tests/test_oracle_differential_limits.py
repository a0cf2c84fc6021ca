"""What the GPU tests of logits that overflow rest on, asked of the 64-bit definition: such keys weigh nothing, and as much as keys far below the others."""
import numpy as np
import pytest

from oracle import differential as diff


@pytest.mark.parametrize("W", [64, 128])
@pytest.mark.parametrize("m", [0, 1])
def test_keys_whose_logits_overflow_in_fp32_weigh_nothing(W, m):
    """Finite numbers whose product is beyond fp32: weights of exactly zero in 64 bits, in that map alone, as of keys whose logits lie 750 below."""
    r, d, n_q, n_k = np.random.default_rng(W + m), W // 2, 9, 40
    q, k, v, d_o = (r.normal(size=(1, 1, n, W)) for n in (n_q, n_k, n_k, n_q))
    lam = tuple(r.normal(size=d) * 0.3 for _ in range(4))
    at = slice(m * d, (m + 1) * d)
    q[..., at] = abs(q[..., at]) * 0.25 + 0.5
    results = []
    for value in (-1500.0 / d ** 0.5, -3e38):
        k[0, 0, 32:, at] = value
        with np.errstate(over="ignore"):
            logits = (q[0, 0][:, at].astype(np.float32) @ k[0, 0][32:, at].astype(np.float32).T)
        assert np.isneginf(logits).all() == (value < -1e38)
        o, g = diff.diff_attn(q, k, v, lam, 0.5, d_o=d_o)
        weights = g["parts"][0, 0]["p%d" % (m + 1)], g["parts"][0, 0]["p%d" % (2 - m)]
        assert not weights[0][:, 32:].any() and weights[1][:, 32:].all()
        results.append([o, g["q"], g["k"], g["v"], *g["lam"]])
    for a, b in zip(*results):
        assert np.array_equal(a, b)
