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


def test_an_8_bit_step_stays_a_step_where_a_block_holds_gradients_of_unlike_size():
    """600 steps, each block's first gradient 2^17 to 2^27 times the others'.  With moments of one step,
    |m| / sqrt(v) of Adam is at most (1 - beta1) / sqrt((1 - beta2)(1 - beta1^2 / beta2)) = 7.3.  Where sqrt(v)
    is held at its least code or above, m / sqrt(v) of the held moments is at most that of the blocks' largest,
    times (1 + 2^-3) / (1 - 2^-3) for an e4m3 step each, and the new gradient's own part at most
    (1 - beta1) / sqrt(1 - beta2) = 3.2: 0.9 * 7.3 * 1.3 + 3.2 = 12 learning rates."""
    n, tensors, sizes = 1280, [], ((1.0, 1e-4), (1.0, 1e-5), (1.0, 1e-6), (1.0, 1e-8), (0.1, 1e-6), (0.01, 1e-6))
    scale = []
    for top, rel in sizes:
        s = torch.full((n,), top * rel, device="cuda")
        s[::128] = top
        scale.append(s)
        tensors.append(fresh(torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), 8))
    plan, t, g = dbw.AdamWPlan(tensors), step_number(0), gen(33)
    largest = torch.zeros(len(sizes), device="cuda")
    for _ in range(600):
        t += 1
        for x, s in zip(tensors, scale):
            x["g"].copy_(s * torch.randn(n, generator=g, device="cuda"))
        before = [x["w"].clone() for x in tensors]
        dbw.dbw_adamw_step(plan, t, lr=1.0, seed=11)
        largest = torch.maximum(largest, torch.stack([(x["w"] - b).abs().max() for x, b in zip(tensors, before)]))
    assert (largest <= 12).all(), largest.tolist()
    for x in tensors:       # every entry has had a gradient: none stands for 0
        assert (x["v"].float() > 0).all()


@pytest.mark.parametrize("gtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("t,in_place", [(1, False), (300, True)])
def test_draws_below_the_least_code(gtype, t, in_place):
    """Gradients of a block over 2^50 and more: entries far below the least code, whose first moment is drawn to 0 or
    to it, and whose second is held at it."""
    n, seed = 128 * 200 + 37, 21
    g = gen(34)
    size = torch.exp(6 * torch.randn(n, generator=g, device="cuda"))
    grad = (size * torch.randn(n, generator=g, device="cuda")).to(gtype)
    x = fresh(torch.randn(n, generator=g, device="cuda"), grad, 8)
    x["m"].copy_(64 * torch.randn(n, generator=g, device="cuda"))
    x["v"].copy_(torch.exp2(19 * torch.rand(n, generator=g, device="cuda") - 10.5))
    x["m_scale"].fill_(2.0 ** -12)
    x["v_scale"].fill_(2.0 ** -12)
    state = [host(x["m"]) * 2.0 ** -12, (host(x["v"]) * 2.0 ** -12) ** 2]
    assert (host(x["v"]) == 0).any()
    if not in_place:
        x.update({k + "_out": torch.empty_like(x[k]) for k in ("w", "m", "v", "m_scale", "v_scale")})
    w0 = host(x["w"])
    dbw.dbw_adamw_step(dbw.AdamWPlan([x]), step_number(t), **HYPER, seed=seed)
    _, m1, v1 = O.adamw(w0, host(grad), *state, t, HYPER["lr"], 0.9, 0.999, 1e-8)
    low = 0
    for key, exact, u, moment in zip("mv", (m1, np.sqrt(v1)), O.draws(0, n, seed, t), (1, 2)):
        q, s = (host(x[key + k + ("" if in_place else "_out")]) for k in ("", "_scale"))
        lo, hi, over, sign, s0 = O.draw_quantize(exact, u, moment)
        assert np.allclose(s, s0, rtol=8 * U, atol=0)
        # the draw decides, unless it or the quotient is closer to its limit than the quotient's own error
        fraction = over - u + 1
        sure = (np.abs(over) > 2.0 ** -13) & (np.abs(fraction - 0.5) < 0.5 - 2.0 ** -13) | (lo == hi)
        assert np.all((np.abs(q) == np.where(over >= 0, hi, lo))[sure])
        assert np.all((sign * q >= 0) & (np.abs(q) <= 448))
        low += int(np.sum(sure & (hi == 2.0 ** -9)))
        if moment == 2:
            assert np.all((q > 0) == (exact > 0))
    assert low > 1000


def test_a_second_moment_of_0_stays_0():
    w, g = torch.ones(300, device="cuda"), torch.zeros(300, device="cuda")
    g[7] = 1.0
    t = fresh(w, g, 8)
    dbw.dbw_adamw_step(dbw.AdamWPlan([t]), step_number(1), **HYPER)
    few = torch.arange(300, device="cuda") != 7
    assert (t["v"].float()[few] == 0).all() and t["v"].float()[7] == 448 and (w[few] == 1).all()


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
