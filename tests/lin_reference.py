"""Linear layers in 8-bit integers and the norm of gradients, plainly and in 64 bits, with error bounds that count roundings."""
import torch

TINY = 2.0 ** -119
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}      # half a step, relative
LEAST = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}   # half a step of the smallest numbers


def codes_of(v):
    """Codes (as 64-bit floats) and scales of the rows of fp32 values; every product that is rounded is exact in 64 bits (24 + 24 bits)."""
    v = v.float()
    top = v.abs().amax(1).clamp(min=TINY).double()
    bad = ~torch.isfinite(v).all(1)
    top = torch.where(bad, torch.ones_like(top), top)
    seven = torch.full_like(top, 127.0)
    codes = torch.round(v.double() * (seven / top).float().double()[:, None])
    scales = torch.where(bad, torch.full_like(top, float("nan")), (top / seven).float().double())
    return torch.where(bad[:, None], torch.zeros_like(codes), codes), scales


def forward(x_codes, x_scales, w_codes, w_scales, bias, dtype):
    """-> y and how far a result in `dtype` may be off: the sum's conversion and two products of scales in fp32, the addition of the bias, the output's type."""
    exact = (x_codes @ w_codes.t()) * x_scales[:, None] * w_scales
    y = exact if bias is None else exact + bias.double()
    return y, 1.01 * (3 * HALF[torch.float32] * exact.abs() + (HALF[torch.float32] + HALF[dtype]) * y.abs()) + 2 * LEAST[dtype]


def backward(dy, x_codes, x_scales, w_codes, w_scales, dtype):
    """-> {name: (gradient, bound)}"""
    dy = dy.float()
    u, u_scales = codes_of(dy * w_scales.float())
    v, v_scales = codes_of((dy * x_scales.float()[:, None]).t())
    dx = (u @ w_codes) * u_scales[:, None]
    dw = (v @ x_codes) * v_scales[:, None]
    db = dy.double().sum(0)
    f = HALF[torch.float32]
    # sums of dbias: at most 2^23 additions in a row, each off by half a step of a partial sum, which the magnitudes' sum bounds
    return {"dx": (dx, 1.01 * (2 * f + HALF[dtype]) * dx.abs() + 2 * LEAST[dtype]), "dw": (dw, 1.01 * 2 * f * dw.abs() + 2 * LEAST[torch.float32]),
            "db": (db, f * min(dy.shape[0], 1 << 23) * dy.double().abs().sum(0))}


def near(got, want, bound, what=""):
    got, want = got.double(), want.double()
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan), what + ": NaN in other places"
    over = torch.where(nan | (got == want), torch.zeros_like(want), (got - want).abs() - bound)   # (equal infinities are equal)
    worst = over.max().item() if over.numel() else 0.0
    assert worst <= 0, "%s: over its bound by %g at %s" % (what, worst, torch.nonzero(over == over.max())[0].tolist())
