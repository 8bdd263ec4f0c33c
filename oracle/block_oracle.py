"""Plain fp64 oracle of the operators of residual feed-forward blocks.

Written from their definitions alone: the norm with the residual's addition and its
gradient, matrices in 8 bits (e4m3) with a scale per block of 128, products of them, and
AdamW with moments in fp32 or in 8 bits.  numpy only, no code of the GPU path.
"""
import numpy as np

TOP = 448.0
TINY = 2.0 ** -100


# ------------------------------------------------------------------ norm
def rmsnorm(x, weight, eps, residual=None):
    """(total, y, rstd) of the rows of x."""
    t = np.asarray(x, np.float64)
    if residual is not None:
        t = t + np.asarray(residual, np.float64)
    rstd = 1.0 / np.sqrt((t * t).mean(axis=1) + eps)
    return t, t * rstd[:, None] * np.asarray(weight, np.float64), rstd


def rmsnorm_backward(dy, t, weight, rstd, groups=1, above=None):
    """(dx, dweight [groups, N])."""
    dy, t, weight, rstd = (np.asarray(a, np.float64) for a in (dy, t, weight, rstd))
    xh = t * rstd[:, None]
    g = dy * weight
    dx = rstd[:, None] * (g - xh * (g * xh).mean(axis=1, keepdims=True))
    if above is not None:
        dx = dx + np.asarray(above, np.float64)
    N = t.shape[1]
    return dx, (dy * xh).reshape(groups, -1, N).sum(axis=1)


# ------------------------------------------------------------------ 8 bits
def e4m3_values():
    """The 127 finite magnitudes, by code: bit pattern eeee mmm of bias 7, subnormals of 2^-9."""
    return np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127])


_VALUES = e4m3_values()


def decode(codes):
    """Values of e4m3 bytes."""
    c = np.asarray(codes, np.uint8)
    mag = np.append(_VALUES, np.nan)[c & 0x7F]
    return np.where(c & 0x80, -mag, mag)


def nearest(z):
    """The e4m3 value nearest to z, ties to the even code, by search in the table of values."""
    z = np.asarray(z, np.float64)
    a = np.minimum(np.abs(z), TOP)
    hi = np.clip(np.searchsorted(_VALUES, a), 1, 126)
    lo = hi - 1
    dl, dh = a - _VALUES[lo], _VALUES[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.where(np.isnan(z), np.nan, np.copysign(_VALUES[code], z))


def _tops(x, r, c):
    R, C = x.shape
    p = np.zeros((-(-R // r) * r, -(-C // c) * c))
    p[:R, :C] = np.abs(x)
    return np.maximum(p.reshape(-(-R // r), r, -(-C // c), c).max(axis=(1, 3)), TINY)


def quantize_rows(x):
    """(values [R, C] of the e4m3 entries, scale [ceil(C / 128), R])."""
    x = np.asarray(x, np.float64)
    top = _tops(x, 1, 128)
    q = nearest(x * (TOP / np.repeat(top, 128, axis=1)[:, :x.shape[1]]))
    return q, (top / TOP).T.copy()


def quantize_blocks(x):
    """(values [R, C], scale [ceil(R / 128), ceil(C / 128)])."""
    x = np.asarray(x, np.float64)
    top = _tops(x, 128, 128)
    mine = np.repeat(np.repeat(top, 128, axis=0)[:x.shape[0]], 128, axis=1)[:, :x.shape[1]]
    return nearest(x * (TOP / mine)), top / TOP


def widen_rows(q, scale):
    return np.asarray(q, np.float64) * np.repeat(np.asarray(scale, np.float64).T, 128, axis=1)[:, :q.shape[1]]


def widen_blocks(q, scale):
    s = np.repeat(np.asarray(scale, np.float64), 128, axis=0)[:q.shape[0]]
    return np.asarray(q, np.float64) * np.repeat(s, 128, axis=1)[:, :q.shape[1]]


def matmul(a, b, groups=1):
    """[groups, M, N] of widened operands a [M, groups K], b [N, groups K]."""
    K = a.shape[1] // groups
    return np.stack([a[:, g * K:(g + 1) * K] @ b[:, g * K:(g + 1) * K].T for g in range(groups)])


# ------------------------------------------------------------------ AdamW
def _mix(h):
    h = np.asarray(h, np.uint64)
    m = np.uint64(0xFFFFFFFF)
    h = h ^ (h >> np.uint64(16))
    h = (h * np.uint64(0x7FEB352D)) & m
    h = h ^ (h >> np.uint64(15))
    h = (h * np.uint64(0x846CA68B)) & m
    return h ^ (h >> np.uint64(16))


def draws(first, n, seed, t):
    """The two random numbers of (0, 1) of elements first .. first + n - 1."""
    m = np.uint64(0xFFFFFFFF)
    i = np.arange(first, first + n, dtype=np.uint64)
    key = _mix(np.uint64((seed ^ (t * 0x9E3779B1)) & 0xFFFFFFFF))
    h = _mix((i & m) ^ _mix((i >> np.uint64(32)) ^ key))
    return ((h & np.uint64(0xFFFF)).astype(np.float64) + 0.5) / 65536, (h >> np.uint64(16)).astype(np.float64) / 65536 + 0.5 / 65536


def draw_quantize(x, u, moment=None):
    """x [n] with one scale per 128: (magnitudes of the lower e4m3 neighbour, of the upper one, how far
    the fraction of the way plus u is above 1, signs, scale).  Below the least code the two moments differ:
    the first (``moment`` 1) is drawn like any other entry, the second's root (2), above 0, is held at the least
    code, which both neighbours then are.  None, either of them: 0, undecided, as how far."""
    x = np.asarray(x, np.float64)
    top = _tops(x[None], 1, 128)[0]
    z = np.abs(x) * (TOP / np.repeat(top, 128)[:x.size])
    lo = np.clip(np.searchsorted(_VALUES, z, side="right") - 1, 0, 125)
    frac = (z - _VALUES[lo]) / (_VALUES[lo + 1] - _VALUES[lo])
    low, over, least = _VALUES[lo], frac + u - 1.0, (lo == 0) & (x != 0)
    if moment == 2:
        low = np.where(least, _VALUES[1], low)
    elif moment is None:
        over = np.where(least, 0.0, over)
    return low, _VALUES[lo + 1], over, np.sign(x), top / TOP


def adamw(w, g, m, v, t, lr, beta1, beta2, eps, weight_decay=0.0, grad_scale=1.0):
    """(w, m, v) after one step."""
    w, g, m, v = (np.asarray(a, np.float64) for a in (w, g, m, v))
    g = g * grad_scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    mh, vh = m / (1 - beta1 ** t), v / (1 - beta2 ** t)
    return w - lr * (mh / (np.sqrt(vh) + eps) + weight_decay * w), m, v
