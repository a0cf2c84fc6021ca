"""Differential attention, its gradient and LayerNorm's gradient in 64 bits, row by row of their definitions.

TEST INFRASTRUCTURE ONLY, like the rest of this package: numpy arrays in, float64 out, nothing of the product used.
"""
import numpy as np


def visible(n_q, n_k, causal, len_q=None, len_k=None):
    """[n_q, n_k] truth values: does query i see key j?"""
    len_q = n_q if len_q is None else min(max(int(len_q), 0), n_q)
    len_k = n_k if len_k is None else min(max(int(len_k), 0), n_k)
    i, j = np.arange(n_q)[:, None], np.arange(n_k)[None]
    keep = (i < len_q) & (j < len_k)
    return keep & (j <= i + len_k - len_q) if causal else keep


def weights(q, k, scale, keep):
    """softmax(scale q k^T) over the kept keys; zero rows where none is kept."""
    s = np.where(keep, (q @ k.T) * scale, -np.inf)
    top = s.max(1, keepdims=True)
    e = np.exp(s - np.where(np.isinf(top), 0.0, top), where=keep, out=np.zeros_like(s))
    total = e.sum(1, keepdims=True)
    return e / np.where(total > 0, total, 1.0)


def lambdas(lam, init, heads):
    """lambda of every head and its two exponentials; lam: four arrays [d] or [heads, d]."""
    q1, k1, q2, k2 = (np.broadcast_to(np.asarray(x, np.float64), (heads, np.shape(x)[-1])) for x in lam)
    e1, e2 = np.exp((q1 * k1).sum(1)), np.exp((q2 * k2).sum(1))
    return e1 - e2 + init, e1, e2


def diff_attn(q, k, v, lam, init, scale=None, causal=False, q_lengths=None, k_lengths=None, d_o=None):
    """O of [B, heads, n_q, W] queries and [B, kv_heads, n_k, W] keys and values, and with d_o also a dict of the gradients
    ("q", "k", "v", "lam") and of what bounds of their errors are made of (per batch entry and head: "parts")."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    B, H, n_q, W = q.shape
    G, n_k, d = k.shape[1], k.shape[2], W // 2
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    value, e1, e2 = lambdas(lam, init, H)
    o = np.zeros_like(q)
    grad = {"q": np.zeros_like(q), "k": np.zeros_like(k), "v": np.zeros_like(v)}
    d_value, parts = np.zeros(H), {}
    for b in range(B):
        keep = visible(n_q, n_k, causal, None if q_lengths is None else q_lengths[b], None if k_lengths is None else k_lengths[b])
        seen_k = keep.any(0)[:, None]
        for h in range(H):
            g = h // (H // G)
            kh, vh = np.where(seen_k, k[b, g], 0.0), np.where(seen_k, v[b, g], 0.0)   # what no query sees is not read
            qh = np.where(keep.any(1)[:, None], q[b, h], 0.0)
            p1, p2 = weights(qh[:, :d], kh[:, :d], scale, keep), weights(qh[:, d:], kh[:, d:], scale, keep)
            o1, o2 = p1 @ vh, p2 @ vh
            o[b, h] = o1 - value[h] * o2
            parts[b, h] = dict(p1=p1, p2=p2, o1=o1, o2=o2, q=qh, k=kh, v=vh, lam=value[h], keep=keep)
            if d_o is None:
                continue
            do = np.where(keep.any(1)[:, None], np.asarray(d_o, np.float64)[b, h], 0.0)
            dp = do @ vh.T
            ds1 = p1 * (dp - (do * o1).sum(1, keepdims=True))
            ds2 = -value[h] * p2 * (dp - (do * o2).sum(1, keepdims=True))
            grad["q"][b, h] = scale * np.concatenate([ds1 @ kh[:, :d], ds2 @ kh[:, d:]], 1)
            grad["k"][b, g] += scale * np.concatenate([ds1.T @ qh[:, :d], ds2.T @ qh[:, d:]], 1)
            grad["v"][b, g] += (p1 - value[h] * p2).T @ do
            d_value[h] -= (p2 * dp).sum()
            parts[b, h].update(do=do, dp=dp, ds1=ds1, ds2=ds2)
    if d_o is None:
        return o, parts
    q1, k1, q2, k2 = (np.asarray(x, np.float64) for x in lam)
    f1, f2 = d_value * e1, -d_value * e2
    if q1.ndim == 1:
        grad["lam"] = tuple(f.sum() * x for f, x in ((f1, k1), (f1, q1), (f2, k2), (f2, q2)))
    else:
        grad["lam"] = tuple(f[:, None] * x for f, x in ((f1, k1), (f1, q1), (f2, k2), (f2, q2)))
    grad["parts"] = parts
    return o, grad


def layernorm_grad(x, gamma, dy, eps, residual=None):
    """(dx, dgamma, dbeta) of LayerNorm over the last axis of [rows, cols]."""
    x, gamma, dy = (np.asarray(a, np.float64) for a in (x, gamma, dy))
    centred = x - x.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt((centred * centred).mean(1, keepdims=True) + eps)
    xh, g = centred * rstd, dy * gamma
    dx = rstd * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    if residual is not None:
        dx = dx + np.asarray(residual, np.float64)
    return dx, (dy * xh).sum(0), dy.sum(0)
