"""Inputs, calls and error bounds shared by the tests of differential attention (not a test module).

Bounds are derived element by element from the 64-bit reference's parts.  EPS: half a step of fp32 (2^-24); u: half a step of
the type that softmax weights and logit gradients are rounded to in front of a matrix product (bf16: 2^-8; fp32 tensors: none);
s: half a step of the type a result is stored in.  A logit is a sum of d products and a scaling: off by EPS (d + 6) sum|q||k| scale;
a weight by twice the largest of those in its row, and by the sum of n_k of them."""
import numpy as np
import torch

from oracle import differential as diff
from paper_2605_26636_amd import binding

EPS = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def make(seed, B, H, G, n_q, n_k, W, dtype, per_head=False, spread=1.0, lam=0.3):
    gen = torch.Generator().manual_seed(seed)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=gen) * scale).to(TYPES[dtype])
    vec = (H, W // 2) if per_head else (W // 2,)
    return dict(q=normal(B, H, n_q, W, scale=spread), k=normal(B, G, n_k, W), v=normal(B, G, n_k, W), d_o=normal(B, H, n_q, W),
                lam=tuple(torch.randn(*vec, generator=gen) * lam for _ in range(4)))


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def guarded(shape, dtype):
    """A tensor of NaN with NaN around it: (view, whole buffer)."""
    n = int(np.prod(shape))
    whole = torch.full((n + 512,), float("nan"), dtype=dtype, device="cuda")
    return whole[256:256 + n].view(shape), whole


def intact(whole):
    return bool(torch.isnan(whole[:256].float()).all() and torch.isnan(whole[-256:].float()).all())


def run(x, init=0.5, scale=0.0, causal=False, lengths=(None, None), backward=False, o_dtype=None, d_lam=True, stream=None):
    """Forward (and backward) pass on the GPU; every output starts as NaN between guards, scratch as garbage."""
    dev = {n: x[n].cuda() for n in ("q", "k", "v", "d_o")}
    lam = tuple(t.cuda() for t in x["lam"])
    lens = [None if l is None else torch.tensor(l, dtype=torch.int32, device="cuda") for l in lengths]
    kind = x["q"].dtype
    o, whole = guarded(tuple(dev["q"].shape), o_dtype or kind)
    kw = dict(lambda_init=init, scale=scale, causal=causal, q_lengths=lens[0], k_lengths=lens[1], stream=stream)
    desc = binding.make_diff_desc(dev["q"], dev["k"], dev["v"], o, causal, *lens)

    def scratch(n):
        return torch.full((max(n, 256),), 0xff, dtype=torch.uint8, device="cuda")
    saved = scratch(binding.jv_diff_attn_saved_bytes(desc)) if backward else None
    binding.jv_diff_attn_fwd(dev["q"], dev["k"], dev["v"], lam, o, saved=saved, workspace=scratch(binding.jv_diff_attn_workspace_bytes(desc)), **kw)
    wholes, out = [whole], {"o": o}
    if backward:
        grads = {n: guarded(tuple(dev[n].shape), kind) for n in ("q", "k", "v")}
        vecs = [guarded(tuple(t.shape), torch.float32) for t in lam] if d_lam else None
        binding.jv_diff_attn_bwd(dev["q"], dev["k"], dev["v"], lam, o, saved, dev["d_o"], grads["q"][0], grads["k"][0], grads["v"][0],
                                 tuple(t for t, _ in vecs) if d_lam else None, workspace=scratch(binding.jv_diff_attn_bwd_workspace_bytes(desc)), **kw)
        out.update({n: grads[n][0] for n in grads}, lam=[t for t, _ in vecs] if d_lam else None)
        wholes += [w for _, w in grads.values()] + ([w for _, w in vecs] if d_lam else [])
    torch.cuda.synchronize()
    assert all(intact(w) for w in wholes), "bytes around an output were written"
    for n in ("q", "k", "v", "d_o"):
        assert torch.equal(dev[n].cpu().view(torch.int16), x[n].view(torch.int16)), "an input was written"
    return out


class Bounds:
    """Reference of a call and how far each result may be from it."""

    def __init__(self, x, dtype, init=0.5, scale=None, causal=False, lengths=(None, None), backward=False, stored=None):
        a = {n: host(x[n]) for n in ("q", "k", "v", "d_o")}
        lam = tuple(host(t) for t in x["lam"])
        B, H, n_q, W = a["q"].shape
        G, n_k, d = a["k"].shape[1], a["k"].shape[2], W // 2
        scale = 1.0 / np.sqrt(d) if not scale or scale <= 0 else scale
        u = 2.0 ** -8 if dtype == "bf16" else 0.0
        s = {"bf16": 2.0 ** -8, "fp32": EPS}[stored or dtype]
        self.o, more = diff.diff_attn(a["q"], a["k"], a["v"], lam, init, scale, causal, *lengths, d_o=a["d_o"] if backward else None)
        parts = more["parts"] if backward else more
        self.grad = more if backward else None
        value, e1, e2 = diff.lambdas(lam, init, H)
        dots = [np.abs(np.broadcast_to(lam[i], (H, d)) * np.broadcast_to(lam[i + 1], (H, d))).sum(1) for i in (0, 2)]
        off_lam = EPS * ((d + 8) * (e1 * (1 + dots[0]) + e2 * (1 + dots[1])) + 4 * abs(value) + 4 * abs(init))
        self.off = {"o": np.zeros_like(a["q"]), "q": np.zeros_like(a["q"]), "k": np.zeros_like(a["k"]), "v": np.zeros_like(a["v"])}
        sums = np.zeros(H)
        for (b, h), p in parts.items():
            g, l, dl = h // (H // G), abs(value[h]), off_lam[h]
            aq, ak, av = abs(p["q"]), abs(p["k"]), abs(p["v"])
            rho, off_o, top = [], [], []
            for m in (0, 1):
                size = (aq[:, m * d:(m + 1) * d] @ ak[:, m * d:(m + 1) * d].T) * scale * p["keep"]
                worst = size.max(1, keepdims=True) if n_k else 0.0
                top.append(worst)
                rho.append(2 * EPS * (d + 6) * worst + EPS * (n_k + 32))
                off_o.append((u + rho[m] + EPS * (n_k + 8)) * (p["p%d" % (m + 1)] @ av))
            off = off_o[0] + (l + dl) * off_o[1] + dl * abs(p["o2"]) + 4 * EPS * (abs(p["o1"]) + l * abs(p["o2"]))
            self.off["o"][b, h] = off + s * (abs(self.o[b, h]) + off)
            if not backward:
                continue
            ado, adp = abs(p["do"]), abs(p["do"]) @ av.T
            # D1 and D2 are formed from the stored rows of O and P2 V
            off2 = off_o[1] + s * (abs(p["o2"]) + off_o[1])
            off1 = self.off["o"][b, h] + (l + dl) * off2 + dl * abs(p["o2"])
            off_d = [(ado * f).sum(1, keepdims=True) + EPS * (W + 8) * (ado * abs(p[n])).sum(1, keepdims=True) for f, n in ((off1, "o1"), (off2, "o2"))]
            off_dp = EPS * (W + 8) * adp
            rho = [r * 2 + 8 * EPS * (1.5 * t + 24) for r, t in zip(rho, top)]   # through the stored logarithm of the denominator
            off_s = []
            for m, weight in ((0, 1.0), (1, l + dl)):
                P, D = p["p%d" % (m + 1)], (p["do"] * p["o%d" % (m + 1)]).sum(1, keepdims=True)
                ds = abs(p["ds%d" % (m + 1)])
                e = weight * P * (off_dp + off_d[m]) + (rho[m] + 8 * EPS) * weight * P * (abs(p["dp"]) + abs(D))
                if m:
                    e = e + dl * P * (abs(p["dp"]) + abs(D))
                off_s.append(e + u * (ds + e))
            n = n_q * (H // G) + 8
            for m in (0, 1):
                at, ds = slice(m * d, (m + 1) * d), abs(p["ds%d" % (m + 1)]) + off_s[m]
                self.off["q"][b, h][:, at] += scale * (off_s[m] @ ak[:, at] + EPS * (n_k + 8) * ds @ ak[:, at])
                self.off["k"][b, g][:, at] += scale * (off_s[m].T @ aq[:, at] + EPS * n * ds.T @ aq[:, at])
            both = p["p1"] + (l + dl) * p["p2"]
            w = u * abs(p["p1"] - value[h] * p["p2"]) + (np.maximum(*rho) + 8 * EPS) * both + dl * p["p2"]
            self.off["v"][b, g] += (w * (1 + u) + EPS * n * both).T @ ado
            sums[h] += (p["p2"] * (off_dp + (rho[1] + EPS * (n_k + n_q + 64)) * abs(p["dp"]))).sum()
        if not backward:
            return
        for n in "qkv":
            self.off[n] += s * (abs(self.grad[n]) + self.off[n])
        # lambda's vectors: the sum's own error, and what forming f = dlambda e and its product with a vector adds
        vec = [np.broadcast_to(x, (H, d)) for x in lam]
        grads = -np.array([sum((p["p2"] * p["dp"]).sum() for (b, hh), p in parts.items() if hh == h) for h in range(H)])
        self.off["lam"] = []
        for e, dot, other in ((e1, dots[0], vec[1]), (e1, dots[0], vec[0]), (e2, dots[1], vec[3]), (e2, dots[1], vec[2])):
            x = ((sums + EPS * ((d + 16) * (1 + dot)) * (abs(grads) + sums)) * e)[:, None] * abs(other)
            self.off["lam"].append(x if lam[0].ndim == 2 else x.sum(0))

    def check(self, out):
        names = ["o"] + (["q", "k", "v"] if self.grad else [])
        for n in names:
            want = self.o if n == "o" else self.grad[n]
            self.one(n, host(out[n]), want, self.off[n])
        if self.grad and out["lam"] is not None:
            for i in range(4):
                self.one("lam %d" % i, host(out["lam"][i]), self.grad["lam"][i], self.off["lam"][i])

    @staticmethod
    def one(name, got, want, off):
        assert np.isfinite(got).all(), f"{name}: not finite"
        far = abs(got - want)
        share = float((far / np.maximum(off, 1e-300)).max()) if far.any() else 0.0
        print(f"    {name}: error up to {share:.3f} of its bound, {far.max():.2e}")
        assert share <= 1.0, f"{name}: {share:.3f} of the bound"
