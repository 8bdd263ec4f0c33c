"""GPU tests of dbw_adamw_step where a CTA takes many parts of a tensor one after another: the next part's
elements on their way while one is stepped.  Every element is checked, with test_gpu_adamw's tolerances but for
the draws: among millions there are first moments whose two terms all but cancel, so that 4 u of the terms is
more than 2^-13 of a step.  See check_draws.

608 CTAs of 1024 elements a part: 3,000,037 elements are 2930 parts, five a CTA at most, and a ragged one."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as O
from paper_2004_14696_gb300 import dbw
from test_gpu_adamw import HYPER, state8, step_number
from test_gpu_norm import U, gen, host

pytestmark = pytest.mark.gpu

SIZES = [3_000_037, 300, 700_000]


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


def check_draws(q, s, x, terms, u, moment):
    """Codes and scales of the exact x.  x is off by at most 4 u of ``terms``, the sum of its terms' magnitudes, its
    quotient by 8 u of itself more, and a fraction of the way between two neighbours by a 2^-20 more: where the
    draw is further than that from its limit it decides, else either neighbour is right."""
    q, s = host(q), host(s)
    lo, hi, over, sign, s0 = O.draw_quantize(x, u, moment)
    assert np.allclose(s, s0, rtol=8 * U, atol=0)
    per = np.repeat(s0, 128)[:x.size]
    off = (4 * U * terms + 8 * U * np.abs(x)) / per / np.maximum(hi - lo, 2.0 ** -9) + 2.0 ** -20
    # within that of a neighbour the pair itself may be the next one
    fraction = over - u + 1
    sure = (np.abs(over) > off) & (fraction > off) & (fraction < 1 - off)
    mine, step = np.abs(q), np.maximum(hi - lo, 2.0 ** -9)
    assert np.all((mine == np.where(over >= 0, hi, lo))[sure])
    assert np.all((mine >= lo - step) & (mine <= hi + step))
    assert np.all((sign * q >= 0)[np.abs(x) > 4 * U * terms])
    assert np.mean(sure) > 0.9


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("in_place,gtype", [(True, torch.float32), (False, torch.bfloat16)])
def test_many_parts_a_cta(in_place, gtype, bits):
    seed, t, clip = 99, 41, 0.75
    decay, scale = [0.1, 0.0, 0.02], [1.0, 0.5, 2.0]
    g, tensors, before = gen(51), [], []
    for n, wd, ls in zip(SIZES, decay, scale):
        size = torch.exp(2 * torch.randn(-(-n // 128), generator=g, device="cuda")).repeat_interleave(128)[:n]
        x = dict(w=torch.randn(n, generator=g, device="cuda"), weight_decay=wd, lr_scale=ls,
                 g=(1e-3 * size * torch.randn(n, generator=g, device="cuda")).to(gtype),
                 w_bf16=torch.empty(n, dtype=torch.bfloat16, device="cuda"))
        m = 1e-3 * size * torch.randn(n, generator=g, device="cuda")
        r = 1e-3 * size * (0.1 + torch.rand(n, generator=g, device="cuda"))
        if bits == 8:
            (x["m"], x["m_scale"]), (x["v"], x["v_scale"]) = state8(m, [n]), state8(r, [n])
            wide = lambda q, s: host(q) * np.repeat(host(s), 128)[:n]  # noqa: E731
            old = [wide(x["m"], x["m_scale"]), wide(x["v"], x["v_scale"]) ** 2]
        else:
            x["m"], x["v"] = m, r * r
            old = [host(x["m"]), host(x["v"])]
        before.append([host(x["w"]), host(x["g"])] + old)
        if not in_place:
            x.update({k + "_out": torch.empty_like(x[k]) for k in ("w", "m", "v", "m_scale", "v_scale") if k in x})
        tensors.append(x)
    plan = dbw.AdamWPlan(tensors)
    dbw.dbw_adamw_step(plan, step_number(t), **HYPER, grad_scale=torch.full((1,), clip, device="cuda"), seed=seed)
    first = 0
    for x, old, wd, ls, n in zip(tensors, before, decay, scale, SIZES):
        out = lambda k: x[k if in_place else k + "_out"]  # noqa: E731
        lr = HYPER["lr"] * ls
        w1, m1, v1 = O.adamw(*old, t, lr, 0.9, 0.999, 1e-8, wd, clip)
        gg = np.abs(old[1]) * clip
        step = np.abs(w1 - old[0])
        cancel = lr * (0.9 * np.abs(old[2]) + 0.1 * gg) / (1 - 0.9 ** t) / (np.sqrt(v1 / (1 - 0.999 ** t)) + 1e-8)
        assert np.all(np.abs(host(out("w")) - w1) <= 32 * U * (step + cancel) + 2 * U * (np.abs(w1) + np.abs(old[0])))
        assert torch.equal(x["w_bf16"], out("w").to(torch.bfloat16))
        if bits == 8:
            u1, u2 = O.draws(first, n, seed, t)
            check_draws(out("m"), out("m_scale"), m1, 0.9 * np.abs(old[2]) + 0.1 * gg, u1, 1)
            check_draws(out("v"), out("v_scale"), np.sqrt(v1), np.sqrt(v1), u2, 2)
        else:
            assert np.all(np.abs(host(out("m")) - m1) <= 4 * U * (0.9 * np.abs(old[2]) + 0.1 * gg) + 2.0 ** -149)
            assert np.all(np.abs(host(out("v")) - v1) <= 6 * U * v1 + 2.0 ** -149)
        first += n
    assert plan.status.item() == 0
