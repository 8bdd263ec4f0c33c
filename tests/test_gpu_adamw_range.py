"""GPU tests of dbw_adamw_step at the ends of its range, against the fp64 oracle.

Tolerances as in test_gpu_adamw (u = 2^-24), one rounding more where the gradient is scaled by a
factor that is no power of two; others beside the tests."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as O
from paper_2004_14696_gb300 import dbw
from test_gpu_adamw import F8, HYPER, check8, step_number
from test_gpu_norm import U, gen, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


def fresh(w, g, bits, **more):
    """A tensor with moments of 0."""
    n, nb = w.numel(), -(-w.numel() // 128)
    t = dict(w=w, g=g, **more)
    for k in "mv":
        t[k] = torch.zeros(n, device="cuda") if bits == 32 else torch.zeros(n, device="cuda").to(F8)
        if bits == 8:
            t[k + "_scale"] = torch.zeros(nb, device="cuda")
    return t


@pytest.mark.parametrize("size,factor,bits", [(1e24, 1e-24, 32), (1e24, 1e-24, 8), (1e-24, 1e24, 32), (1e-24, 1e24, 8),
                                              (1.0, 1e-20, 32)])
def test_a_clip_factor_whose_square_fp32_does_not_hold(size, factor, bits):
    """The factor scales the gradient, and the square is the scaled one's."""
    n, seed = 5003, 4
    g = gen(31)
    w0, grad = torch.randn(n, generator=g, device="cuda"), size * torch.randn(n, generator=g, device="cuda")
    w = w0.clone()
    t = fresh(w, grad, bits)
    plan = dbw.AdamWPlan([t])
    gs = torch.full((1,), factor, device="cuda")
    dbw.dbw_adamw_step(plan, step_number(1), **HYPER, grad_scale=gs, seed=seed)
    z = np.zeros(n)
    w1, m1, v1 = O.adamw(host(w0), host(grad), z, z, 1, HYPER["lr"], 0.9, 0.999, 1e-8, 0.0, float(gs.double()))
    step = np.abs(w1 - host(w0))
    assert np.all(np.abs(host(w) - w1) <= 32 * U * step + 2 * U * (np.abs(w1) + np.abs(host(w0))))
    if bits == 32:
        assert np.all(np.abs(host(t["m"]) - m1) <= 6 * U * np.abs(m1) + 2.0 ** -149)
        assert np.all(np.abs(host(t["v"]) - v1) <= 8 * U * v1 + 2.0 ** -149)
    else:
        u1, u2 = O.draws(0, n, seed, 1)
        check8(t["m"], t["m_scale"], m1, u1, [n])
        check8(t["v"], t["v_scale"], np.sqrt(v1), u2, [n])
