"""LayerNorm's gradient without eps: rows that vary have a deviation of their own to divide by, and rows past the end of a workgroup's step, which are
zeros and have none, stay out of the column sums."""
import pytest
import torch

import differential as D
import test_gpu_layernorm_bwd as N
from oracle import differential as diff
from paper_2605_26636_amd import binding

pytestmark = pytest.mark.gpu


# rows a step of 8 to 512 lanes takes: 64, 32, 16, 8, 4, 2 and 1; a last step that is not full, and several steps a workgroup
@pytest.mark.parametrize("rows,cols", [(1, 8), (61, 64), (65, 40), (33, 128), (17, 256), (9, 520), (5, 2000), (3, 4096), (64 * 600 + 5, 64), (8 * 700 + 3, 1024), (2, 8192)])
@pytest.mark.parametrize("x_type,dy_type", [("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "fp32")])
def test_no_eps(rows, cols, x_type, dy_type):
    gen = torch.Generator().manual_seed(rows + cols)
    x = (torch.randn(rows, cols, generator=gen) * 0.5 + torch.randn(rows, 1, generator=gen)).to(D.TYPES[x_type])
    dy = torch.randn(rows, cols, generator=gen).to(D.TYPES[dy_type])
    gamma = 1 + 0.3 * torch.randn(cols, generator=gen)
    assert (x.float().std(1) > 0.05).all()
    dx, w0 = D.guarded((rows, cols), x.dtype)
    (dgamma, w1), (dbeta, w2) = (D.guarded((cols,), torch.float32) for _ in range(2))
    ws = torch.full((binding.jv_layernorm_bwd_workspace_bytes(rows, cols),), 0xff, dtype=torch.uint8, device="cuda")
    binding.jv_layernorm_bwd(x.cuda(), gamma.cuda(), dy.cuda(), dx, dgamma, dbeta, eps=0.0, workspace=ws)
    torch.cuda.synchronize()
    assert D.intact(w0) and D.intact(w1) and D.intact(w2)
    args = [D.host(t) for t in (x, gamma, dy)] + [0.0, None]
    for name, got, want, off in zip(("dx", "dgamma", "dbeta"), (dx, dgamma, dbeta), diff.layernorm_grad(*args), N.bounds(*args, x_type == "bf16")):
        D.Bounds.one(name, D.host(got), want, off)
