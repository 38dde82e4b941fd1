"""Plain forms in 64 bits (numpy) of the operators on floating-point tensors, with bounds of what fp32 arithmetic may add to them."""
import numpy as np

EPS32 = 2.0 ** -24      # half a step of fp32, relative
HALF_STEP = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8, "i32": 0.0}
TINY = {"fp32": 2.0 ** -149, "fp16": 2.0 ** -25, "bf16": 2.0 ** -134, "i32": 0.0}   # half a step below the normal numbers


def block_form(x, block=32):
    """codes, exponent bytes and restored values of [rows, cols]; the step is the smallest power of two with max <= 127 steps."""
    rows, cols = x.shape
    blocks = -(-cols // block)
    codes = np.zeros((rows, cols), np.int8)
    exps = np.zeros((rows, blocks), np.uint8)
    back = np.zeros((rows, cols))
    for b in range(blocks):
        part = x[:, b * block:(b + 1) * block].astype(np.float64)
        bad = ~np.isfinite(part).all(1)
        amax = np.where(bad, 1.0, np.abs(np.where(np.isfinite(part), part, 0)).max(1))
        m, k = np.frexp(amax / 127.0)                   # the quotient is exact where it is a power of two
        k = np.where(m == 0.5, k - 1, k)
        k = np.where(amax == 0, -126, np.maximum(k, -126))
        step = np.ldexp(1.0, k)
        with np.errstate(invalid="ignore"):
            q = np.rint(part / step[:, None])           # ties to even
        q = np.where((k == 122)[:, None], np.clip(q, -63, 63), q)
        codes[:, b * block:(b + 1) * block] = np.where(bad[:, None], 0, q).astype(np.int8)
        exps[:, b] = np.where(bad, 255, k + 127)
        back[:, b * block:(b + 1) * block] = np.where(bad[:, None], np.nan, q * step[:, None])
    return codes, exps, back


def act(z, kind):
    return z if kind == "none" else np.where(z < 0, 0.0, z) if kind == "relu" else z / (1 + np.exp(-z))


def slope(z, kind):
    if kind == "none":
        return np.ones_like(z)
    if kind == "relu":
        return (z > 0).astype(np.float64)
    q = 1 / (1 + np.exp(-z))
    return q * (1 + z * (1 - q))


def gn_stats(x, groups, eps):
    n, hw, c = x.shape
    v = x.astype(np.float64).reshape(n, hw, groups, c // groups)
    mean = v.mean((1, 3))
    return mean, 1 / np.sqrt(((v - mean[:, None, :, None]) ** 2).mean((1, 3)) + eps)


def _wide(a, c):
    return np.repeat(a, c // a.shape[1], 1)[:, None, :]     # [n, groups] -> [n, 1, c]


def gn_fwd(x, groups, eps, gamma, beta, kind):
    """y, statistics, and a bound of y's error before it is rounded to its type.

    fp32 chain: sums of at most a few hundred terms in a row (a thread's batches, the slots of a block), each addition off by EPS32 of
    the running value, itself no larger than the largest |x|: mean and every x - mean are off by at most 64 EPS32 max|x|, u by rstd
    times that and by the relative error of rstd (half of that of the variance, the same order).  exp is off by 2 + 1.2 |z| steps and the
    quotient by 2, which the activation passes on relative to its value; its slope is at most 1.1."""
    n, hw, c = x.shape
    mean, rstd = gn_stats(x, groups, eps)
    u = (x.astype(np.float64) - _wide(mean, c)) * _wide(rstd, c)
    z = gamma * u + beta
    y = act(z, kind)
    top = np.abs(x.astype(np.float64)).reshape(n, hw, groups, -1).max((1, 3))
    du = 64 * EPS32 * (_wide(top * rstd, c) + np.abs(u) * (1 + _wide(top * rstd, c)))
    bound = 1.1 * (np.abs(gamma) * du + 4 * EPS32 * (np.abs(gamma * u) + np.abs(beta) + np.abs(gamma) * _wide(np.abs(mean) * rstd, c)))
    bound = bound + (np.abs(y) * (8 + 1.2 * np.abs(z)) * 2 * EPS32 if kind == "silu" else 0)
    return y, mean, rstd, bound


def gn_bwd(dy, x, mean, rstd, gamma, beta, kind):
    """dx, dgamma, dbeta and bounds of their errors (see gn_fwd; |second derivative| of the activation <= 1/2).  x: what the gradients
    are taken at; mean, rstd [n, groups]: the forward pass's, in fp32."""
    n, hw, c = x.shape
    groups = mean.shape[1]
    x = x.astype(np.float64)
    m, r = _wide(mean, c), _wide(rstd, c)
    u = (x - m) * r
    z = gamma * u + beta
    dz = dy * slope(z, kind)
    g = gamma * dz
    by = (n, hw, groups, c // groups)
    s1, s2 = g.reshape(by).mean((1, 3)), (g * u).reshape(by).mean((1, 3))
    dx = r * (g - _wide(s1, c) - u * _wide(s2, c))
    # u = (x - mean) rstd: two roundings of its own, and room for a fused form that rounds mean * rstd
    du = 4 * EPS32 * (np.abs(x) * r + np.abs(m) * r + np.abs(u))
    if kind == "none":
        ddz = EPS32 * np.abs(dz)
    elif kind == "relu":
        ddz = EPS32 * np.abs(dz)
    else:
        ddz = np.abs(dy) * (0.5 * (np.abs(gamma) * du + 2 * EPS32 * (np.abs(gamma * u) + np.abs(beta))) + 1.1 * (12 + 1.2 * np.abs(z)) * 2 * EPS32)
    dg = np.abs(gamma) * ddz + EPS32 * np.abs(g)
    mean_abs = lambda a: np.abs(a).reshape(by).mean((1, 3))  # noqa: E731
    d1 = mean_abs(dg) + 256 * EPS32 * mean_abs(g)
    d2 = mean_abs(dg * np.abs(u) + np.abs(g) * du) + 256 * EPS32 * mean_abs(g * u)
    bdx = r * (dg + _wide(d1, c) + np.abs(u) * _wide(d2, c) + du * np.abs(_wide(s2, c)))
    bdx = bdx + 8 * EPS32 * r * (np.abs(g) + np.abs(_wide(s1, c)) + np.abs(u * _wide(s2, c)))
    dgamma, dbeta = (dz * u).sum((0, 1)), dz.sum((0, 1))
    bdgamma = (ddz * np.abs(u) + np.abs(dz) * du).sum((0, 1)) + 256 * EPS32 * np.abs(dz * u).sum((0, 1))
    bdbeta = ddz.sum((0, 1)) + 256 * EPS32 * np.abs(dz).sum((0, 1))
    return dx, dgamma, dbeta, bdx, bdgamma, bdbeta


def within(got, want, bound, dtype="fp32"):
    """|got - want| <= bound plus half a step of the type that holds it, everywhere; NaN where NaN is wanted."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fine = ~np.isnan(want)
    room = (bound + HALF_STEP[dtype] * (np.abs(want) + bound) + TINY[dtype]) * np.ones_like(want)
    off = np.abs(got - want)
    worst = np.nanmax(np.where(fine, off / np.maximum(room, 1e-300), 0.0)) if fine.any() else 0.0
    assert worst <= 1.0, f"{worst:.3g} times the bound"
    return worst
