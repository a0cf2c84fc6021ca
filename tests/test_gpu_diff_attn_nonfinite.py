"""Differential attention where numbers are not finite: NaN in a query, infinities in a key, logits that overflow in one map; whole calls and calls
whose keys are cut into parts, forward and backward pass."""
import numpy as np
import pytest
import torch

import differential as D
from oracle import differential as diff

pytestmark = pytest.mark.gpu

KINDS = [("bf16", 64), ("bf16", 128), ("fp32", 64), ("fp32", 128)]
ROWS = [(2, 8), (1, 17), (1, 65)]       # heads of one kv head, queries: both maps in one block, a wavefront, four of them
KEYS = [20, 33, 330, 1100, 8190]        # one part up to more than eight of them


@pytest.mark.parametrize("half", [0, 1])
@pytest.mark.parametrize("heads,n_q", ROWS)
@pytest.mark.parametrize("dtype,W", KINDS)
def test_nan_in_a_query_is_nan_in_its_row(dtype, W, heads, n_q, half):
    for n_k in KEYS:
        x = D.make(n_k + W, 1, heads, 1, n_q, n_k, W, dtype)
        want = D.Bounds(x, dtype)
        x["q"][0, 0, 5, half * W // 2 + 3] = float("nan")
        got = D.host(D.run(x)["o"])
        print(n_k, flush=True)
        assert np.isnan(got[0, 0, 5]).all(), n_k
        got[0, 0, 5] = want.o[0, 0, 5]
        D.Bounds.one("other rows", got, want.o, want.off["o"])


@pytest.mark.parametrize("n_q,n_k", [(17, 20), (40, 330), (200, 300)])
@pytest.mark.parametrize("half", [0, 1])
@pytest.mark.parametrize("dtype,W", KINDS)
def test_nan_in_a_query_is_nan_in_its_gradients(dtype, W, half, n_q, n_k):
    """A query's gradient and those of the keys and values that it sees; the other queries and the other head keep theirs."""
    x = D.make(31, 1, 2, 2, n_q, n_k, W, dtype)
    want = D.Bounds(x, dtype, backward=True)
    x["q"][0, 0, 5, half * W // 2 + 3] = float("nan")
    out = {n: D.host(t) for n, t in D.run(x, backward=True, d_lam=False).items() if n != "lam"}
    at = slice(half * W // 2, half * W // 2 + W // 2)   # (the other map's channels may be numbers)
    assert np.isnan(out["o"][0, 0, 5]).all() and np.isnan(out["q"][0, 0, 5, at]).all()
    assert np.isnan(out["k"][0, 0, :, at]).all() and np.isnan(out["v"][0, 0]).all()
    out["o"][0, 0, 5], out["q"][0, 0, 5], out["k"][0, 0], out["v"][0, 0] = want.o[0, 0, 5], want.grad["q"][0, 0, 5], want.grad["k"][0, 0], want.grad["v"][0, 0]
    for n in "oqkv":
        D.Bounds.one(n, out[n], want.o if n == "o" else want.grad[n], want.off[n])


@pytest.mark.parametrize("heads,n_q", ROWS)
@pytest.mark.parametrize("W", [64, 128])
def test_infinity_in_the_last_key_of_fp32_tensors_is_nan(W, heads, n_q):
    for n_k in KEYS + [65, 1025]:
        x = D.make(n_k + W, 1, heads, 1, n_q, n_k, W, "fp32")
        x["k"][0, 0, n_k - 1, 2] = float("inf")
        assert torch.isnan(D.run(x)["o"]).all(), n_k


@pytest.mark.parametrize("heads,n_q", ROWS + [(1, 200)])
@pytest.mark.parametrize("dtype,W", KINDS)
def test_logits_that_overflow_in_one_map(dtype, W, heads, n_q):
    """Keys whose logits of one map are -inf in fp32 (finite numbers of -3e38) weigh nothing there, and what they weigh in the other: as keys
    whose logits lie 750 below the others, which weigh nothing in 64 bits either."""
    d = W // 2
    for n_k in (40, 64, 330, 1100):
        for m in (0, 1):
            x = D.make(n_k + W, 1, heads, 1, n_q, n_k, W, dtype)
            x["q"][..., m * d:(m + 1) * d] = x["q"][..., m * d:(m + 1) * d].abs() * 0.25 + 0.5
            hidden = slice(32, n_k)   # all parts but the first
            x["k"][0, 0, hidden, m * d:(m + 1) * d] = -1500.0 / d ** 0.5
            want = D.Bounds(x, dtype, backward=True)
            x["k"][0, 0, hidden, m * d:(m + 1) * d] = -3e38
            print(n_k, m, flush=True)
            want.check(D.run(x, backward=True))


@pytest.mark.parametrize("heads,n_q", ROWS + [(1, 200)])
@pytest.mark.parametrize("dtype,W", KINDS)
def test_a_map_whose_logits_all_overflow_weighs_nothing(dtype, W, heads, n_q):
    """All logits of one map -inf: O = P1 V or -lambda P2 V, and the gradients are the other map's.  Relative 2-norms: two roundings to bf16, of the
    weights (or logit gradients) and of the result, and for fp32 sums of n_k, n_q or W terms, each formed from one before."""
    d = W // 2
    for n_k in (40, 330):
        for m in (0, 1):
            x = D.make(n_k + W, 1, heads, 1, n_q, n_k, W, dtype)
            x["q"][..., m * d:(m + 1) * d] = x["q"][..., m * d:(m + 1) * d].abs() * 0.25 + 0.5
            x["k"][..., m * d:(m + 1) * d] = -3e38
            out = D.run(x, backward=True, d_lam=False)
            q, k, v, do = (D.host(x[n]) for n in ("q", "k", "v", "d_o"))
            value = diff.lambdas(tuple(D.host(t) for t in x["lam"]), 0.5, heads)[0][0]
            f, at, scale = (1.0 if m else -value), slice((1 - m) * d, (2 - m) * d), d ** -0.5
            ref = {"o": np.zeros_like(q), "q": np.zeros_like(q), "k": np.zeros_like(k), "v": np.zeros_like(v)}
            for h in range(heads):
                p = diff.weights(q[0, h][:, at], k[0, 0][:, at], scale, np.ones((n_q, n_k), bool))
                o, dp = p @ v[0, 0], do[0, h] @ v[0, 0].T
                ds = f * p * (dp - (do[0, h] * o).sum(1, keepdims=True))
                ref["o"][0, h] = f * o
                ref["q"][0, h][:, at] = scale * ds @ k[0, 0][:, at]
                ref["k"][0, 0][:, at] += scale * ds.T @ q[0, h][:, at]
                ref["v"][0, 0] += f * p.T @ do[0, h]
            tol = 2 * 2.0 ** -8 if dtype == "bf16" else 8 * D.EPS * (n_k + n_q * heads + W)
            for n in ref:
                got = D.host(out[n])
                assert np.isfinite(got).all(), (n_k, m, n)
                rel = np.linalg.norm(got - ref[n]) / np.linalg.norm(ref[n])
                print(n_k, m, n, rel, flush=True)
                assert rel <= tol, (n_k, m, n)


@pytest.mark.parametrize("heads,n_q", ROWS)
@pytest.mark.parametrize("at", [2, "second map"])
@pytest.mark.parametrize("W", [64, 128])
def test_infinity_in_a_key_of_bf16_tensors(W, at, heads, n_q):
    """It makes a logit of +inf, which is NaN, or of -inf, which takes no part in its map and does not touch the other: by the sign of the query's number."""
    at = W // 2 + 2 if at == "second map" else at
    for n_k in KEYS:
        for key in {0, n_k // 2, n_k - 1}:
            x = D.make(n_k + W, 1, heads, 1, n_q, n_k, W, "bf16")
            near = x["q"][..., at].abs() < 0.25
            x["q"][..., at][near] = -0.25
            nan = D.host(x["q"])[..., at] > 0
            # a logit of -256 / sqrt(W / 2) or less weighs 2^-46 of the others at most
            x["k"][0, 0, key, at] = 2.0 ** 10
            want = D.Bounds(x, "bf16")
            x["k"][0, 0, key, at] = float("inf")
            got = D.host(D.run(x)["o"])
            assert np.isnan(got[nan]).all(), (n_k, key)
            assert np.isfinite(got[~nan]).all(), (n_k, key)
            D.Bounds.one(f"{n_k} {key}", np.where(nan[..., None], want.o, got), want.o, want.off["o"])


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype,W", KINDS)
def test_rows_that_see_no_key_stay_zero_beside_rows_that_are_nan(dtype, W, value):
    """Queries behind a sequence's end, and causal ones in front of all keys, beside a key or a value that is not finite."""
    for causal, lengths, n_q, n_k in ((False, ([20, 0], [50, 50]), 45, 50), (True, (None, None), 150, 40), (False, (None, [0, 300]), 40, 300)):
        for n in ("k", "v"):
            x = D.make(32, 2, 2, 1, n_q, n_k, W, dtype)
            x[n][:, :, 3, 7] = value
            out = D.run(x, causal=causal, lengths=lengths, backward=True, d_lam=False)
            keep = [diff.visible(n_q, n_k, causal, *(None if l is None else l[b] for l in lengths)).any(1) for b in range(2)]
            assert not all(x.all() for x in keep)
            for b in range(2):
                for t in ("o", "q"):
                    assert not out[t][b][:, ~torch.from_numpy(keep[b])].cpu().float().abs().nan_to_num(1.0).any(), (causal, n, t, b)
