"""GPU test of grouped products into outputs whose groups lie side by side in each row.

Tolerances as in test_gpu_fp8."""
import pytest
import torch

from paper_2004_14696_gb300 import dbw
from test_gpu_fp8 import check_product, operand
from test_gpu_norm import gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("groups,M,N,K", [(3, 20, 40, 256), (5, 130, 203, 128), (60, 260, 512, 256), (40, 300, 513, 128)])
def test_groups_side_by_side(groups, M, N, K, dtype):
    g = gen(groups + M)
    qa, sa, a = operand(g, M, groups * K)
    qb, sb, b = operand(g, N, groups * K)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for gap in (0, 8):
        whole = torch.full((M, groups, N + gap), 7.0, device="cuda").to(dtype)
        out = whole[:, :, :N].permute(1, 0, 2)
        dbw.dbw_fp8_matmul(qa, sa, qb, sb, out, status, groups=groups)
        check_product(out, a, b, groups, dtype)
        assert (whole[:, :, N:].float() == 7).all() and status.item() == 0


def test_overlapping_groups_are_refused():
    a, s = dbw.fp8_rows(8, 256), torch.empty((2, 8), device="cuda")
    status, buf = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.empty(4096, device="cuda")
    # [2, 8, 8] by (groups apart, rows apart): shared entries in all of them
    for strides in ((0, 8), (7, 16), (8, 15), (63, 8), (16, 16)):
        with pytest.raises(ValueError, match="overlap"):
            dbw.dbw_fp8_matmul(a, s, a, s, buf.as_strided((2, 8, 8), (*strides, 1)), status, groups=2)
