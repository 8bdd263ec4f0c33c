"""GPU tests of dbw_rmsnorm and its gradient where a CTA takes several rows one after another, as it does at the
sizes of training: the next row on its way while one is summed, the two halves of the sums' buffer in turn,
d weight summed over the passes, a last pass that is not full.  The checks and tolerances are test_gpu_norm's.

152 SMs of 1024 threads: at 4096 columns 304 CTAs of one row (fp32) or 608 (bf16, two chunks a warp), so
that 1500 rows are 5 or 3 passes; 3001 x 601 in fp32 3 with 1216 rows at a time."""
import pytest
import torch

from test_gpu_norm import built, gen, test_norm as check_norm, test_norm_gradient as check_gradient  # noqa: F401
from oracle import block_oracle as O
from paper_2004_14696_gb300 import dbw
from test_gpu_norm import check_q, host, rand

pytestmark = pytest.mark.gpu

LAYOUTS = [(0, 0), (3, 1)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad,shift", LAYOUTS)
@pytest.mark.parametrize("M,N", [(1500, 4096), (1301, 1000), (3001, 601), (4001, 300), (700, 8192), (400, 16384),
                                 (400, 16392), (9001, 100)])
def test_norm_in_several_passes(M, N, pad, shift, dtype):
    check_norm(M, N, pad, shift, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad,shift", LAYOUTS)
@pytest.mark.parametrize("M,N,groups", [(2000, 4096, 4), (3003, 1000, 3), (5003, 300, 1), (700, 8192, 1), (500, 16384, 2),
                                        (402, 32768, 1), (2010, 601, 2), (30003, 100, 3)])
def test_norm_gradient_in_several_passes(M, N, groups, pad, shift, dtype):
    check_gradient(M, N, groups, pad, shift, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_norms_over_their_inputs_in_several_passes(dtype):
    """total over x and over the residual, dx over dy and over above: a row read ahead is none that is written."""
    M, N, groups = 1501, 2048, 1
    g = gen(61)
    x, res, dy, above = (rand(g, M, N, dtype) for _ in range(4))
    w = 1 + 0.3 * torch.randn(N, generator=g, device="cuda")
    total, q, scale, rstd = torch.empty_like(x), dbw.fp8_rows(M, N), torch.empty((16, M), device="cuda"), torch.empty(M, device="cuda")
    dbw.dbw_rmsnorm(x, w, 1e-6, residual=res, total=total, q=q, scale=scale, rstd=rstd)
    check_q(q, scale, O.rmsnorm(host(x), host(w), 1e-6, host(res))[1], "q")
    for into in (0, 1):
        pair, q2, r2 = (x.clone(), res.clone()), torch.empty_like(q), torch.empty_like(rstd)
        dbw.dbw_rmsnorm(pair[0], w, 1e-6, residual=pair[1], total=pair[into], q=q2, scale=torch.empty_like(scale), rstd=r2)
        assert torch.equal(pair[into], total) and torch.equal(r2, rstd) and torch.equal(q2.view(torch.uint8), q.view(torch.uint8))
    ws = torch.empty(dbw.dbw_rmsnorm_backward_workspace_bytes(M, N, groups), dtype=torch.uint8, device="cuda")
    dx, dw = torch.empty_like(x), torch.empty((groups, N), device="cuda")
    dbw.dbw_rmsnorm_backward(dy, total, w, rstd, dx, dw, ws, above=above)
    for into in (0, 1):
        pair, dw2 = (dy.clone(), above.clone()), torch.empty_like(dw)
        dbw.dbw_rmsnorm_backward(pair[0], total, w, rstd, pair[into], dw2, ws, above=pair[1])
        assert torch.equal(pair[into], dx) and torch.equal(dw2, dw)
