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


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("lr", [1e-3, 1e-4, 1e-5, 3e-6, 1e-6])
def test_a_weight_decay_far_below_a_rounding_of_the_weight(lr, bits):
    """Every element is rounded to a multiple of 2^-24 (weights of 0.5 to 1).  Its step (moments at hand, so that no
    two are alike) is spread over several of them, at the least lr a deviation of about five, so that a rounding
    is as likely to go either way: the mean over n elements is off by 2^-24 / sqrt(12 n) (one standard
    deviation; six are allowed), where a decay taken as a multiple of 2^-24 is off by up to half of that."""
    n, decay, steps = 1 << 20, 0.01, 100
    g = gen(32)
    w0 = 0.5 + 0.5 * torch.rand(n, generator=g, device="cuda").clamp(0.01, 0.99)
    grad, m0 = (torch.randn(n, generator=g, device="cuda") for _ in range(2))
    r0 = 0.5 + torch.rand(n, generator=g, device="cuda")
    w = w0.clone()
    t = fresh(w, grad, bits, weight_decay=decay)
    if bits == 32:
        t["m"].copy_(m0)
        t["v"].copy_(r0 * r0)
        before = host(t["m"]), host(t["v"])
    else:
        t["m"].copy_((100 * m0).clamp(-448, 448))
        t["v"].copy_(200 * r0)
        t["m_scale"].fill_(1 / 128)
        t["v_scale"].fill_(1 / 256)
        before = host(t["m"]) / 128, (host(t["v"]) / 256) ** 2
    dbw.dbw_adamw_step(dbw.AdamWPlan([t]), step_number(steps), lr=lr)
    w1, _, _ = O.adamw(host(w0), host(grad), *before, steps, lr, 0.9, 0.999, 1e-8, decay)
    assert abs(np.mean(host(w) - w1)) <= 6 * 2.0 ** -24 / np.sqrt(12 * n)


@pytest.mark.parametrize("bits", [32, 8])
def test_no_eps_and_squares_below_the_normal_numbers(bits):
    """|g| from 3e-21 to 1e-15: v is a multiple of 2^-149, off by 2^-150 at most, so sqrt(v) by 2^-150 / v of itself
    (twice its first order); w starts at 0, and its first step is -lr sign(g)."""
    n = 128 * 50
    mag = 10.0 ** (-20.5 + 5.5 * torch.arange(50, device="cuda", dtype=torch.float64) / 49)
    grad = mag.repeat_interleave(128).float()
    grad[::3] *= -1
    w = torch.zeros(n, device="cuda")
    t = fresh(w, grad, bits)
    dbw.dbw_adamw_step(dbw.AdamWPlan([t]), step_number(1), lr=0.5, eps=0.0)
    z = np.zeros(n)
    w1, m1, v1 = O.adamw(z, host(grad), z, z, 1, 0.5, 0.9, 0.999, 0.0)
    rel = 2.0 ** -150 / v1 + 64 * U
    assert np.all(np.abs(host(w) - w1) <= rel * np.abs(w1))
    if bits == 32:
        assert np.all(np.abs(host(t["v"]) - v1) <= 8 * U * v1 + 2.0 ** -150)
    else:
        one = slice(None, None, 128)
        assert np.all(np.abs(host(t["v_scale"]) * 448 - np.sqrt(v1[one])) <= rel[one] * np.sqrt(v1[one]))
        assert (t["v"].float() == 448).all()
