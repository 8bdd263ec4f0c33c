"""GPU test of every link of the residual network's forward and backward pass, from the tensors that the iteration
itself left behind: what each call had to make of its inputs, in fp64.

(A whole pass cannot be held so closely: a bf16 entry that fp32's sum rounds the other way changes a row by 2^-9 of
itself, after which so many e4m3 entries of it fall on the other side of a rounding that it differs by 1e-2.)

Tolerances: an operand's entries are x * (448 / amax) rounded twice in fp32 and then to e4m3, which numpy does alike:
equal.  Products as in test_gpu_fp8, norms as in test_gpu_norm.  The logits' gradient is a softmax in fp32, 2^-18 of the
1 that it differs from, and a rounding to bf16."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as O
from paper_2004_14696_gb300 import residual
from test_gpu_fp8 import check_product
from test_gpu_norm import HALF, U, check_q, host

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
ONE = dict(blocks=1, S=2000)
WORKLOADS = [residual.ResidualWorkload(key="small", width=136, hidden=200, classes=7, n=3, B=128, **ONE),
             residual.ResidualWorkload(key="longer minibatches", width=96, hidden=320, classes=10, n=2, B=384, **ONE),
             residual.ResidualWorkload(key="default width", **ONE)]


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


def operand(x, r, c):
    """(entries, scales) of x with a scale per r x c block, in fp32's two roundings."""
    R, C = x.shape
    x = np.asarray(x, np.float32)
    p = np.zeros((-(-R // r) * r, -(-C // c) * c), np.float32)
    p[:R, :C] = np.abs(x)
    top = np.maximum(p.reshape(-(-R // r), r, -(-C // c), c).max(axis=(1, 3)), np.float32(O.TINY))
    inv = np.repeat(np.repeat(np.float32(O.TOP) / top, r, axis=0)[:R], c, axis=1)[:, :C]
    return O.nearest(x * inv), top / np.float32(O.TOP)


def same_operand(op, x, blocks=False, forward=True):
    """op holds x, both ways (``forward`` False: the transpose alone is held to x)."""
    if blocks:
        q, s = operand(x, 128, 128)
        assert np.array_equal(host(op.q), q) and np.array_equal(host(op.scale), s)
        assert np.array_equal(host(op.qt), q.T) and np.array_equal(host(op.scale_t), s.T)
        return
    if forward:
        q, s = operand(x, 1, 128)
        assert np.array_equal(host(op.q), q) and np.array_equal(host(op.scale), s.T)
    q, s = operand(x.T, 1, 128)
    assert np.array_equal(host(op.qt), q) and np.array_equal(host(op.scale_t), s.T)


def rows(op):
    return O.widen_rows(host(op.q), host(op.scale))


def rows_t(op):
    return O.widen_rows(host(op.qt), host(op.scale_t))


@pytest.mark.parametrize("wl", WORKLOADS, ids=lambda w: w.key)
def test_every_link(wl):
    it = residual.ResidualIteration(wl)
    it.load_inputs(0)
    w = {k: host(v) for k, v in it.p.items()}
    x, seen = host(it.pool[it.idx.long()]), {}
    # the tensors that a later call writes over
    fill = {k: getattr(it, k).fill for k in ("qC", "qD", "qH")}
    it.u[0].fill_t = (lambda f: lambda y: (seen.update(y0=y.clone()), f(y)))(it.u[0].fill_t)
    for k in fill:
        getattr(it, k).fill = (lambda k: lambda v, gate=None: (seen.update({k: v.clone()}), fill[k](v, gate)))(k)
    product, made = it._product, []

    def record(a, a_scale, b, b_scale, out, **kw):
        product(a, a_scale, b, b_scale, out, **kw)
        if out is it.du:
            made.append(out.clone())
    it._product = record
    it.forward()
    W = {k: (O.widen_blocks(host(v.q), host(v.scale)), v) for k, v in it.W.items()}
    for name, (_, op) in W.items():
        same_operand(op, w[name], blocks=True)

    # t_0 = x; its norm, in 8 bits unrounded, in bf16 for the transpose
    assert np.array_equal(host(it.t[0]), x)
    _, y, r = O.rmsnorm(x, w["norm0"], it.EPS)
    assert np.allclose(host(it.rstd[0]), r, rtol=40 * U, atol=0)
    check_q(it.u[0].q, it.u[0].scale, y, "u0")
    assert np.all(np.abs(host(seen["y0"]) - y) <= (48 * U + HALF[BF16] * 1.01) * np.abs(y))
    same_operand(it.u[0], host(seen["y0"]), forward=False)
    check_product(it.z[0], rows(it.u[0]), W["W1_0"][0], 1, BF16)
    same_operand(it.h[0], np.maximum(host(it.z[0]), 0))
    check_product(it.o, rows(it.h[0]), W["W2_0"][0], 1, BF16)
    # t_1 = t_0 + o
    t, y, r = O.rmsnorm(x, w["norm"], it.EPS, host(it.o))
    size = np.abs(x) + np.abs(host(it.o))
    assert np.all(np.abs(host(it.t[1]) - t) <= (HALF[BF16] * 1.01 + U) * size)
    assert np.allclose(host(it.rstd[1]), r, rtol=40 * U, atol=0)
    check_q(it.u[1].q, it.u[1].scale, y, "u1")
    same_operand(it.u[1], host(it.y), forward=False)
    check_product(it.logits, rows(it.u[1]), W["Wc"][0], 1, F32)

    d = it.loss_gradient()
    z = host(it.logits)
    e = np.exp(z - z.max(1, keepdims=True))
    p = e / e.sum(1, keepdims=True)
    labels = it.labels[it.idx.long()].cpu().numpy()
    loss = -np.log(p[np.arange(len(p)), labels]).reshape(wl.n, wl.B).mean(1)
    p[np.arange(len(p)), labels] -= 1
    assert np.allclose(host(it.loss), loss, rtol=2.0 ** -16, atol=2.0 ** -16)
    assert np.all(np.abs(host(d) - p / wl.B) <= HALF[BF16] * 1.01 * np.abs(p / wl.B) + 2.0 ** -18 / wl.B)

    it.backward(d)
    norm_size = lambda dy, t, r, g: np.abs(r[:, None] * dy * g) + np.abs(t * r[:, None] ** 2) * np.mean(  # noqa: E731
        np.abs(dy * g * t * r[:, None]), axis=1, keepdims=True)

    def norm_back(du, l, name, above, dx):
        t, r = host(it.t[l]), host(it.rstd[l])
        dx0, dw0 = O.rmsnorm_backward(host(du), t, w[name], r, wl.n, above)
        size = norm_size(host(du), t, r, w[name]) + (0 if above is None else np.abs(above))
        assert np.all(np.abs(host(dx) - dx0) <= 64 * U * size + HALF[BF16] * 1.01 * np.abs(dx0))
        terms = (np.abs(host(du) * t) * r[:, None]).reshape(wl.n, -1, wl.width).sum(1)
        assert np.all(np.abs(host(it.g[name]).reshape(dw0.shape) - dw0) <= (wl.B + 16) * U * terms)

    same_operand(it.qC, host(d))
    check_product(it.g["Wc"], rows_t(it.qC), rows_t(it.u[1]), wl.n, F32)
    check_product(made[0], rows(it.qC), W["Wc"][0].T, 1, BF16)
    dt1 = seen["qD"]                        # as the block's backward pass finds it
    norm_back(made[0], 1, "norm", None, dt1)
    same_operand(it.qD, host(dt1))
    check_product(it.g["W2_0"], rows_t(it.qD), rows_t(it.h[0]), wl.n, F32)
    check_product(seen["qH"], rows(it.qD), W["W2_0"][0].T, 1, BF16)
    same_operand(it.qH, host(seen["qH"]) * (host(it.z[0]) > 0))
    check_product(it.g["W1_0"], rows_t(it.qH), rows_t(it.u[0]), wl.n, F32)
    check_product(made[1], rows(it.qH), W["W1_0"][0].T, 1, BF16)
    norm_back(made[1], 0, "norm0", host(dt1), it.dt)
    assert int(it.status) == 0
