"""GPU test of the bounded waits of the 8-bit products.

dbw_test_arm_wait_timeout keeps the first tile of the next product from loading one stage (no copy is
outstanding for it) and shortens the bound of every wait to 1 ms.  The MMA's wait for that stage runs out and
the others' in turn; the call returns, its status word has bit 0 set, and the next call of the same process,
which allocates the same tensor memory, gives the bits of the one before."""
import pytest
import torch

from paper_2004_14696_gb300 import dbw
from test_gpu_fp8 import operand
from test_gpu_norm import gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


# a single CTA a tile; K over a cluster; pairs in turn and pairs that ask for their tiles, 256 of them with 8 K blocks
SHAPES = [(2100, 300, 1000, True), (40, 200, 4096, False), (4096, 4096, 1024, True), (4096, 4096, 1024, False)]


@pytest.mark.parametrize("stage", [0, 2, 6])
@pytest.mark.parametrize("M,N,K,blocks", SHAPES)
def test_a_stage_that_does_not_come(M, N, K, blocks, stage):
    g = gen(M + N)
    qa, sa, _ = operand(g, M, K)
    qb, sb, _ = operand(g, N, K, blocks)
    out, status = torch.empty((M, N), dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")

    def call():
        status.zero_()
        dbw.dbw_fp8_matmul(qa, sa, qb, sb, out, status, blocks=blocks)
        torch.cuda.synchronize()
        return int(status)

    assert call() == 0
    want = out.clone()
    # (40, 200, 4096): a CTA of the cluster has 4 of 32 K blocks or more, so that its last stage is left out
    dbw.dbw_test_arm_wait_timeout(min(stage, 3) if K == 4096 else stage, 1.0)
    assert call() & 1, "the wait for the stage without its load did not run out"
    for _ in range(2):
        out.zero_()
        assert call() == 0
        assert torch.equal(out, want)


def test_a_lost_stage_of_a_later_tile():
    """Pairs: a tile of 8 K blocks after the first, whose sums wait in tensor memory and shared memory."""
    M, N, K = 4096, 4096, 1024
    g = gen(5)
    for blocks in (False, True):
        qa, sa, _ = operand(g, M, K)
        qb, sb, _ = operand(g, N, K, blocks)
        out, status = torch.empty((M, N), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        dbw.dbw_fp8_matmul(qa, sa, qb, sb, out, status, blocks=blocks)
        want = out.clone()
        dbw.dbw_test_arm_wait_timeout(13, 1.0)
        dbw.dbw_fp8_matmul(qa, sa, qb, sb, torch.empty_like(out), status, blocks=blocks)
        assert int(status) == 1
        status.zero_()
        out.zero_()
        dbw.dbw_fp8_matmul(qa, sa, qb, sb, out, status, blocks=blocks)
        assert int(status) == 0 and torch.equal(out, want)
