"""Calls on a stream of their own: work goes there in the order in which it was given, whatever the current stream is and however a call is
marshalled, and scratch memory that a call takes for itself stays the stream's."""
import pytest
import torch

import differential as D
from paper_2605_26636_amd import binding

pytestmark = pytest.mark.gpu

DELAY = 100_000_000   # clock cycles, some 40 to 50 ms: longer than a step's host calls take


@pytest.fixture(params=["extension module", "ctypes"])
def marshalled(request, monkeypatch):
    """Calls through the extension module, and through the descriptors that stand in where it has no form for the arguments."""
    if request.param == "ctypes":
        class Nothing:
            diff_attn_fwd = diff_attn_bwd = layernorm_bwd = staticmethod(lambda *args: None)
        monkeypatch.setattr(binding, "_native", Nothing)
    else:
        binding._load_native()


def waiting(side):
    """The side stream has work before it, and the current one none."""
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(DELAY)


@pytest.mark.parametrize("dtype,n_q,n_k", [("bf16", 33, 500), ("fp32", 130, 200)])
def test_a_step_waits_for_its_own_stream_alone(marshalled, dtype, n_q, n_k):
    """Inputs that the stream brings up to date in front of the call are what the call reads, and the stream's end is the call's."""
    old, new = (D.make(seed, 2, 4, 2, n_q, n_k, 64, dtype) for seed in (41, 42))
    want = D.run(new, backward=True)
    side = torch.cuda.Stream()
    t, after = ({n: x[n].cuda() for n in ("q", "k", "v", "d_o")} for x in (old, new))
    lam, lam_after = (tuple(v.cuda() for v in x["lam"]) for x in (old, new))
    got = {n: torch.full_like(t[n], float("nan")) for n in "qkv"}
    got["o"] = torch.full_like(t["q"], float("nan"))
    got["lam"] = tuple(torch.full_like(v, float("nan")) for v in lam)
    desc = binding.make_diff_desc(t["q"], t["k"], t["v"], got["o"])
    saved, ws, ws_bwd = (torch.empty(max(n, 256), dtype=torch.uint8, device="cuda") for n in (
        binding.jv_diff_attn_saved_bytes(desc), binding.jv_diff_attn_workspace_bytes(desc), binding.jv_diff_attn_bwd_workspace_bytes(desc)))
    waiting(side)
    with torch.cuda.stream(side):
        for n in t:
            t[n].copy_(after[n])
        for a, b in zip(lam, lam_after):
            a.copy_(b)
    binding.jv_diff_attn_fwd(t["q"], t["k"], t["v"], lam, got["o"], lambda_init=0.5, saved=saved, workspace=ws, stream=side)
    binding.jv_diff_attn_bwd(t["q"], t["k"], t["v"], lam, got["o"], saved, t["d_o"], got["q"], got["k"], got["v"], got["lam"], lambda_init=0.5,
                             workspace=ws_bwd, stream=side)
    assert not side.query()   # all of it stands behind the delay
    side.synchronize()
    for n in "oqkv":
        assert torch.equal(got[n], want[n]), n
    assert all(torch.equal(a, b) for a, b in zip(got["lam"], want["lam"]))


def test_a_norm_s_gradient_waits_for_its_own_stream_alone(marshalled):
    gen = torch.Generator().manual_seed(43)
    x, after, dy = (torch.randn(700, 256, generator=gen).cuda() for _ in range(3))
    gamma = torch.randn(256, generator=gen).cuda()
    want, got = ([torch.full_like(t, float("nan")) for t in (x, gamma, gamma)] for _ in range(2))
    binding.jv_layernorm_bwd(after, gamma, dy, *want)
    ws = torch.empty(binding.jv_layernorm_bwd_workspace_bytes(700, 256), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    waiting(side)
    with torch.cuda.stream(side):
        x.copy_(after)
    binding.jv_layernorm_bwd(x, gamma, dy, *got, workspace=ws, stream=side)
    assert not side.query()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_step_on_a_side_stream_and_captured_from_it():
    """A step on a side stream gives the bits of one on the current stream, also through a graph captured from that stream."""
    x = D.make(44, 2, 4, 2, 60, 300, 64, "bf16")
    want = D.run(x, backward=True)
    q, k, v, d_o = (x[n].cuda() for n in ("q", "k", "v", "d_o"))
    lam = tuple(t.cuda() for t in x["lam"])
    outs = {n: torch.empty_like(t) for n, t in (("o", q), ("q", q), ("k", k), ("v", v))}
    desc = binding.make_diff_desc(q, k, v, outs["o"])
    saved, ws = (torch.empty(max(n, 256), dtype=torch.uint8, device="cuda") for n in (
        binding.jv_diff_attn_saved_bytes(desc), max(binding.jv_diff_attn_workspace_bytes(desc), binding.jv_diff_attn_bwd_workspace_bytes(desc))))
    side = torch.cuda.Stream()

    def step():
        binding.jv_diff_attn_fwd(q, k, v, lam, outs["o"], lambda_init=0.5, saved=saved, workspace=ws, stream=side)
        binding.jv_diff_attn_bwd(q, k, v, lam, outs["o"], saved, d_o, outs["q"], outs["k"], outs["v"], lambda_init=0.5, workspace=ws, stream=side)

    def same():
        torch.cuda.synchronize()
        for n, t in outs.items():
            assert torch.equal(t, want[n]), n
            t.fill_(float("nan"))
        torch.cuda.synchronize()
    torch.cuda.synchronize()
    step()
    same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    torch.cuda.synchronize()
    assert all(torch.isnan(t).all() for t in outs.values())   # captured, not run
    for _ in range(3):
        graph.replay()
        same()


@pytest.mark.parametrize("call", ["forward", "backward", "norm", "linear", "block"])
def test_scratch_that_a_call_takes_for_itself_stays_its_stream_s(call):
    """A call on a named stream allocates its scratch there: let go of while the call waits its turn, the memory does not come back to the current
    stream, whose next tensors would be written over."""
    side = torch.cuda.Stream()
    x = D.make(45, 2, 4, 2, 70, 900, 64, "fp32")
    q, k, v, d_o = (x[n].cuda() for n in ("q", "k", "v", "d_o"))
    lam = tuple(t.cuda() for t in x["lam"])
    o, dq, dk, dv = (torch.empty_like(t) for t in (q, q, k, v))
    saved = torch.empty(binding.jv_diff_attn_saved_bytes(binding.make_diff_desc(q, k, v, o)), dtype=torch.uint8, device="cuda")
    rows, gamma = torch.randn(700, 256).cuda(), torch.ones(256, device="cuda")
    out, dgamma, dbeta = torch.empty_like(rows), torch.empty_like(gamma), torch.empty_like(gamma)
    grid = (30, 30)
    binding.jv_diff_attn_fwd(q, k, v, lam, o, saved=saved)

    def run(stream):
        if call == "forward":
            return binding.jv_diff_attn_fwd(q, k, v, lam, o, stream=stream), o
        if call == "backward":
            return binding.jv_diff_attn_bwd(q, k, v, lam, o, saved, d_o, dq, dk, dv, stream=stream), dk
        if call == "norm":
            return binding.jv_layernorm_bwd(rows, gamma, rows, out, dgamma, dbeta, stream=stream), dgamma
        if call == "linear":
            return binding.jv_linear_attn_fwd(k, k, v, dk, grid, stream=stream), dk
        return binding.jv_linear_block_fwd(k, k, v, dk, grid, static_kernel=torch.ones(128, 3, 3, device="cuda"), stream=stream), dk
    want = run(None)[1].clone()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    waiting(side)
    ws, got = run(side)
    at, n = ws.data_ptr(), ws.numel()
    del ws
    mine = [torch.full((n,), 0xff, dtype=torch.uint8, device="cuda") for _ in range(4)]
    assert all(t.data_ptr() != at for t in mine)
    side.synchronize()
    assert torch.equal(got, want)
    assert all(bool((t == 0xff).all()) for t in mine)
