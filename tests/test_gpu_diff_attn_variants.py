"""Every way a call of differential attention or of LayerNorm's gradient is cut, on the GPU: wavefronts by rows, parts of the keys and
their joins, parts of the gradient's passes, rows of every width at every number of workgroups; and calls from a program's side:
a stream given by name, two captured graphs, tensors that the calls refuse."""
import pytest
import torch

import differential as D
import test_gpu_layernorm_bwd as N
from oracle import differential as diff
from paper_2605_26636_amd import binding

pytestmark = pytest.mark.gpu

ROWS = [(2, 8), (1, 17), (4, 16), (5, 13)]   # heads of one kv head, queries: 16, 17, 64, 65 rows
KEYS = [20, 50, 70, 140, 200, 270, 330, 530, 900, 1540, 2040, 8190, 33000]
# B, heads, kv_heads, n_q, n_k, causal
GRADIENTS = [(1, 2, 1, 150, 2100, False), (1, 1, 1, 2100, 150, False), (1, 2, 2, 1100, 1100, True), (2, 2, 1, 300, 260, True), (3, 4, 4, 200, 200, False),
             (2, 1, 1, 50, 45, True)]
# rows of 64 columns, 64 rows a step: 256, 257, 512, 513, 1 024 and 1 025 steps
NORMS = [(64 * 256, 64), (64 * 256 + 1, 64), (64 * 512 - 5, 64), (64 * 512 + 1, 64), (64 * 1024, 64), (64 * 1024 + 7, 64), (1100, 1032), (1030, 8192)]


@pytest.mark.parametrize("heads,n_q", ROWS)
@pytest.mark.parametrize("dtype,W", [("bf16", 64), ("bf16", 128), ("fp32", 64), ("fp32", 128)])
def test_parts_of_the_keys(dtype, W, heads, n_q):
    for n_k in KEYS:
        x = D.make(n_k + W, 1, heads, 1, n_q, n_k, W, dtype)
        print(n_k, flush=True)
        D.Bounds(x, dtype).check(D.run(x))


@pytest.mark.parametrize("B,H,G,n_q,n_k,causal", GRADIENTS)
@pytest.mark.parametrize("dtype,W", [("bf16", 64), ("bf16", 128), ("fp32", 64), ("fp32", 128)])
def test_parts_of_the_gradient(dtype, W, B, H, G, n_q, n_k, causal):
    x = D.make(n_q + n_k + W, B, H, G, n_q, n_k, W, dtype)
    D.Bounds(x, dtype, causal=causal, backward=True).check(D.run(x, causal=causal, backward=True))


@pytest.mark.parametrize("H,G,n_q", [(32, 1, 1), (16, 1, 1), (12, 1, 3), (80, 2, 1), (6, 6, 3)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_lambda_a_head_where_a_wavefront_holds_many(dtype, H, G, n_q):
    x = D.make(H + n_q, 3, H, G, n_q, 40, 64, dtype, per_head=True)
    out = D.run(x, backward=True)
    D.Bounds(x, dtype, backward=True).check(out)
    longer = D.make(H + n_q, 1, H, G, n_q, 700, 64, dtype, per_head=True)
    D.Bounds(longer, dtype).check(D.run(longer))


def test_fp32_rows_that_fill_more_than_half_of_the_units():
    """143 workgroups, and 25 tiles of keys: forward and backward pass are cut."""
    for W in (64, 128):
        x = D.make(28, 1, 11, 11, 1537, 800, W, "fp32")
        D.Bounds(x, "fp32", backward=True).check(D.run(x, backward=True))


def test_fp32_output_of_parts():
    """A bf16 output is an fp32 one, rounded, however the keys are cut."""
    for H, n_q, n_k in ((2, 8, 70), (2, 8, 140), (2, 8, 330), (2, 8, 2040), (1, 17, 300), (5, 13, 530), (1, 300, 900)):
        x = D.make(n_k, 1, H, 1, n_q, n_k, 128, "bf16")
        o32, o16 = (D.run(x, o_dtype=t)["o"] for t in (torch.float32, torch.bfloat16))
        assert torch.equal(o32.to(torch.bfloat16), o16), (n_q, n_k)
        D.Bounds(x, "bf16", stored="fp32").check({"o": o32})


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_65535_heads_of_one_key(dtype):
    """As many (batch, head)s as a call takes.  One key has all weight in both maps: O = (1 - lambda) V, dV = (1 - lambda) dO, dQ = dK = 0,
    dlambda = -sum dO V.  (1 - lambda) V is formed as V - lambda V, each rounded once; D2 and dP are sums of 64 products."""
    B, H = 13107, 5
    x = D.make(26, B, H, H, 1, 1, 64, dtype)
    out = D.run(x, backward=True)
    value, e1, e2 = diff.lambdas(tuple(D.host(t) for t in x["lam"]), 0.5, 1)
    s = 2.0 ** -8 if dtype == "bf16" else D.EPS
    v, d_o = (D.host(x[n]) for n in ("v", "d_o"))
    for n, full in (("o", v), ("v", d_o)):
        D.Bounds.one(n, D.host(out[n]), (1 - value[0]) * full, (s * (1 + 2 * abs(value[0])) + 64 * D.EPS) * abs(full) * 2 + 1e-30)
    # dS = P (dP - D): the difference of two sums of 64 products, whose rows of O and P2 V are rounded by s; times scale and a row of K or Q
    size = (abs(d_o) * abs(v)).sum(-1, keepdims=True) * (s * (3 + 2 * abs(value[0])) + 80 * D.EPS) * (1 + abs(value[0])) / 32 ** 0.5
    for n, other in (("q", "k"), ("k", "q")):
        D.Bounds.one(n, D.host(out[n]), 0 * v, size * abs(D.host(x[other])) * (1 + 2 * s) + 1e-30)
    dots = abs(d_o * v).sum()
    d_value = -(d_o * v).sum()
    for i, (e, other) in enumerate(((e1, 1), (e1, 0), (-e2, 3), (-e2, 2))):
        want = d_value * e[0] * D.host(x["lam"][other])
        D.Bounds.one("lam %d" % i, D.host(out["lam"][i]), want, 100 * D.EPS * (dots + abs(d_value)) * abs(e[0]) * abs(D.host(x["lam"][other])) * 2)


def test_a_cache_that_grows_between_replays():
    """Lengths are read on the GPU: a captured step answers for the caches' present lengths."""
    x = D.make(27, 3, 8, 2, 1, 1500, 64, "bf16")
    q, k, v = (x[n].cuda() for n in "qkv")
    lam = tuple(t.cuda() for t in x["lam"])
    lengths = torch.zeros(3, dtype=torch.int32, device="cuda")
    o = torch.empty_like(q)
    ws = torch.empty(binding.jv_diff_attn_workspace_bytes(binding.make_diff_desc(q, k, v, o, False, None, lengths)), dtype=torch.uint8, device="cuda")
    binding.jv_diff_attn_fwd(q, k, v, lam, o, lambda_init=0.5, k_lengths=lengths, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.jv_diff_attn_fwd(q, k, v, lam, o, lambda_init=0.5, k_lengths=lengths, workspace=ws)
    for present in ([0, 1, 2], [1, 33, 700], [1500, 1499, 0], [640, 1500, 31]):
        lengths.copy_(torch.tensor(present, dtype=torch.int32))
        o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        D.Bounds(x, "bf16", lengths=(None, present)).check({"o": o})


@pytest.mark.parametrize("dtype,W", [("bf16", 64), ("bf16", 128), ("fp32", 64), ("fp32", 128)])
def test_lambda_s_gradient_is_not_biased(dtype, W):
    """dlambda_h = -Sum P2 o dP sums numbers of both signs.  Errors of its terms, at most 8 half steps of fp32 each (score, exponential, dP, sum),
    and of its rows (reference, denominator), as many, that do not know of each other add up like a random walk: six standard deviations."""
    B, H, N = 2, 6, 2600
    x = D.make(25, B, H, H, N, N, W, dtype, per_head=True)
    out = D.run(x, backward=True)
    q, k, v, d_o = (x[n].double().cuda() for n in ("q", "k", "v", "d_o"))
    lam = [t.double().cuda() for t in x["lam"]]
    d = W // 2
    terms = (torch.matmul(q[..., d:], k[..., d:].transpose(-1, -2)) / d ** 0.5).softmax(-1) * torch.matmul(d_o, v.transpose(-1, -2))
    rows = terms.sum(-1)
    far = 6 * 8 * D.EPS * ((terms * terms).sum((0, 2, 3)).sqrt() + (rows * rows).sum((0, 2)).sqrt())
    want = rows.sum((0, 2)) * (lam[2] * lam[3]).sum(-1).exp()
    far = far * (lam[2] * lam[3]).sum(-1).exp() + 8 * D.EPS * want.abs()
    got = (out["lam"][3].double() * lam[2]).sum(-1) / (lam[2] * lam[2]).sum(-1)   # d_k2 = -dlambda e2 q2
    D.Bounds.one("dlambda", got.cpu().numpy(), want.cpu().numpy(), far.cpu().numpy())


@pytest.mark.parametrize("size", [1e-12, 1e12])
def test_fp32_numbers_far_from_one(size):
    """Each number goes into its products as a sum of three of bf16, whatever its exponent: relative errors stay those of numbers near one."""
    x = D.make(21, 1, 2, 1, 40, 90, 64, "fp32")
    want = D.run(x, backward=True)
    scaled = dict(x, q=x["q"] * 2.0 ** 40, k=x["k"] * 2.0 ** -40)
    got = D.run(scaled, backward=True)
    for n, f in (("o", 0), ("v", 0), ("q", -40), ("k", 40)):   # powers of two change no bit of a significand
        assert torch.equal(got[n], want[n] * 2.0 ** f), n
    big = dict(x, v=x["v"] * size)
    D.Bounds(big, "fp32", backward=True).check(D.run(big, backward=True))


@pytest.mark.parametrize("rows,cols", NORMS)
@pytest.mark.parametrize("x_type,dy_type", [("bf16", "bf16"), ("fp32", "fp32")])
def test_workgroups_of_a_norm(rows, cols, x_type, dy_type):
    gen = torch.Generator().manual_seed(rows + cols)
    x = (torch.randn(rows, cols, generator=gen) + torch.randn(rows, 1, generator=gen)).to(D.TYPES[x_type])
    dy = torch.randn(rows, cols, generator=gen).to(D.TYPES[dy_type])
    gamma = 1 + 0.3 * torch.randn(cols, generator=gen)
    dx, w0 = D.guarded((rows, cols), x.dtype)
    (dgamma, w1), (dbeta, w2) = (D.guarded((cols,), torch.float32) for _ in range(2))
    ws = torch.full((binding.jv_layernorm_bwd_workspace_bytes(rows, cols),), 0xff, dtype=torch.uint8, device="cuda")
    binding.jv_layernorm_bwd(x.cuda(), gamma.cuda(), dy.cuda(), dx, dgamma, dbeta, eps=1e-5, workspace=ws)
    torch.cuda.synchronize()
    assert D.intact(w0) and D.intact(w1) and D.intact(w2)
    args = [D.host(t) for t in (x, gamma, dy)] + [1e-5, None]
    for name, got, want, off in zip(("dx", "dgamma", "dbeta"), (dx, dgamma, dbeta), diff.layernorm_grad(*args), N.bounds(*args, x_type == "bf16")):
        D.Bounds.one(name, D.host(got), want, off)


def test_a_stream_given_by_name():
    """stream= runs a call there, whatever the current stream is."""
    x = D.make(22, 2, 4, 2, 33, 500, 64, "bf16")
    want = D.run(x, backward=True)
    side = torch.cuda.Stream()
    q, k, v, d_o = (x[n].cuda() for n in ("q", "k", "v", "d_o"))
    lam = tuple(t.cuda() for t in x["lam"])
    got = {n: torch.empty_like(t) for n, t in (("o", q), ("q", q), ("k", k), ("v", v))}
    desc = binding.make_diff_desc(q, k, v, got["o"])
    saved, ws, ws_bwd = (torch.empty(max(n, 256), dtype=torch.uint8, device="cuda") for n in (
        binding.jv_diff_attn_saved_bytes(desc), binding.jv_diff_attn_workspace_bytes(desc), binding.jv_diff_attn_bwd_workspace_bytes(desc)))
    torch.cuda.synchronize()
    binding.jv_diff_attn_fwd(q, k, v, lam, got["o"], lambda_init=0.5, saved=saved, workspace=ws, stream=side)
    binding.jv_diff_attn_bwd(q, k, v, lam, got["o"], saved, d_o, got["q"], got["k"], got["v"], lambda_init=0.5, workspace=ws_bwd, stream=side)
    torch.cuda.synchronize()
    for n in ("o", "q", "k", "v"):
        assert torch.equal(got[n], want[n]), n
    rows = torch.randn(50, 128).cuda()
    out = [torch.empty_like(rows) for _ in range(2)]
    gamma, dy = torch.ones(128, device="cuda"), rows * 0.5
    torch.cuda.synchronize()
    for o, s in zip(out, (None, side)):
        binding.jv_layernorm_bwd(rows, gamma, dy, o, stream=s)
        torch.cuda.synchronize()
    assert torch.equal(*out)


def test_two_graphs_replayed_in_turn():
    """Two captured steps of different sizes, each with a workspace of its own, replayed in turn and on changed inputs."""
    steps = []
    for seed, n_q, n_k in ((23, 1, 700), (24, 90, 150)):
        x = D.make(seed, 1, 4, 2, n_q, n_k, 64, "bf16")
        t = {n: x[n].cuda() for n in ("q", "k", "v", "d_o")}
        lam = tuple(v.cuda() for v in x["lam"])
        o, dq, dk, dv = (torch.empty_like(t[n]) for n in ("q", "q", "k", "v"))
        desc = binding.make_diff_desc(t["q"], t["k"], t["v"], o)
        saved, ws, ws_bwd = (torch.empty(max(n, 256), dtype=torch.uint8, device="cuda") for n in (
            binding.jv_diff_attn_saved_bytes(desc), binding.jv_diff_attn_workspace_bytes(desc), binding.jv_diff_attn_bwd_workspace_bytes(desc)))

        def step(t=t, lam=lam, o=o, dq=dq, dk=dk, dv=dv, saved=saved, ws=ws, ws_bwd=ws_bwd):
            binding.jv_diff_attn_fwd(t["q"], t["k"], t["v"], lam, o, saved=saved, workspace=ws)
            binding.jv_diff_attn_bwd(t["q"], t["k"], t["v"], lam, o, saved, t["d_o"], dq, dk, dv, workspace=ws_bwd)
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        steps.append((graph, step, t, (o, dq, dk, dv)))
    for turn in range(3):
        want = []
        for graph, step, t, outs in steps:
            t["q"].mul_(-0.5).add_(0.25)
            t["v"].add_(0.125)
            step()
            want.append([a.clone() for a in outs])
            for a in outs:
                a.fill_(float("nan"))
        for graph, *_ in steps:
            graph.replay()
        torch.cuda.synchronize()
        for (*_, outs), w in zip(steps, want):
            assert all(torch.equal(a, b) for a, b in zip(outs, w)), turn


def test_tensors_that_are_refused():
    """None of these reaches the GPU."""
    q, k = (torch.zeros(2, 4, 5, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 2, 7, 64, dtype=torch.bfloat16, device="cuda"))
    lam = tuple(torch.zeros(32, device="cuda") for _ in range(4))
    good = dict(q=q, k=k, v=k, lam=lam, o=torch.empty_like(q))
    lengths = torch.tensor([5, 5], dtype=torch.int32, device="cuda")
    short = torch.empty(256, dtype=torch.uint8, device="cuda")
    for bad in (dict(q=q.cpu()), dict(k=k.float()), dict(v=k[:, :1]), dict(k=k[:1], v=k[:1]), dict(o=q[:, :, :4]), dict(q=q.transpose(2, 3)), dict(lam=lam[:3]),
                dict(lam=tuple(t.double() for t in lam)), dict(lam=tuple(torch.zeros(64, device="cuda") for _ in range(4))), dict(q_lengths=lengths.long()),
                dict(q_lengths=lengths[:1]), dict(k_lengths=lengths.cpu()), dict(k_lengths=torch.zeros(4, dtype=torch.int32, device="cuda")[::2]),
                dict(saved=short), dict(saved=short.expand(1 << 16, 256)), dict(o=q), dict(lambda_init=float("inf")), dict(scale=1e31)):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            binding.jv_diff_attn_fwd(**dict(good, **bad))
    binding.jv_diff_attn_fwd(**good)
    desc = binding.make_diff_desc(q, k, k, good["o"])
    saved = torch.empty(binding.jv_diff_attn_saved_bytes(desc), dtype=torch.uint8, device="cuda")
    grads = dict(good, saved=saved, d_o=torch.zeros_like(q), d_q=torch.empty_like(q), d_k=torch.empty_like(k), d_v=torch.empty_like(k))
    need = binding.jv_diff_attn_bwd_workspace_bytes(desc)
    for bad in (dict(saved=None), dict(saved=saved[:-256]), dict(d_q=torch.empty_like(k)), dict(d_k=torch.empty_like(k).float()), dict(d_v=k), dict(d_o=q.cpu()),
                dict(d_lam=lam[:2]), dict(d_lam=tuple(t.bfloat16() for t in lam)), dict(workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda")),
                dict(workspace=torch.empty(2 * need, dtype=torch.uint8, device="cuda")[::2])):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            binding.jv_diff_attn_bwd(**dict(grads, **bad))
    rows, gamma = torch.zeros(6, 64, device="cuda"), torch.ones(64, device="cuda")
    norm = dict(x=rows, gamma=gamma, dy=rows, dx=torch.empty_like(rows))
    for bad in (dict(x=rows.cpu()), dict(gamma=gamma.bfloat16()), dict(dy=rows[:3]), dict(dx=rows.bfloat16()), dict(dx=rows), dict(dgamma=gamma.clone()), dict(eps=-1.0),
                dict(residual=rows.bfloat16()), dict(x=torch.zeros(64, 6, device="cuda").t()), dict(dgamma=gamma.clone(), dbeta=gamma.clone(), workspace=short[:16])):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            binding.jv_layernorm_bwd(**dict(norm, **bad))
