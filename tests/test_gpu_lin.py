"""Linear layers in 8-bit integers on a GPU against the plain forms in 64 bits."""
import math

import pytest
import torch

import lin_reference as ref
from gpu_util import handle, status_clear
from paper_2105_13890_b200 import build, eoq

build.build_lib()
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {torch.float32: eoq.EOQ_F32, torch.float16: eoq.EOQ_F16, torch.bfloat16: eoq.EOQ_BF16}


def normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def rows_in(v, beside=0, offset=0):
    """The matrix as part of wider rows, its first element `offset` elements behind an aligned address."""
    rows, cols = v.shape
    flat = torch.full((rows * (cols + beside) + offset + 16,), float("nan"), dtype=v.dtype, device=DEV)
    out = flat[offset:offset + rows * (cols + beside)].view(rows, cols + beside)[:, :cols]
    out.copy_(v)
    return out


class Layer:
    """Inputs, buffers and calls of a layer."""

    def __init__(self, rows, c_in, c_out, dtype, bias=True, beside=0, offset=0, seed=0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed + rows * 31 + c_in * 7 + c_out)
        self.rows, self.c_in, self.c_out, self.dtype, self.beside, self.offset = rows, c_in, c_out, dtype, beside, offset
        self.x = rows_in((normal(g, rows, c_in) * torch.exp(normal(g, c_in))).to(dtype), beside, offset)
        self.w = normal(g, c_out, c_in) * torch.exp(0.3 * normal(g, c_out, 1)) / math.sqrt(c_in)
        self.bias = normal(g, c_out) if bias else None
        self.dy = rows_in((0.05 * normal(g, rows, c_out) * torch.exp(normal(g, rows, 1))).to(dtype), beside, offset)
        self.desc = eoq.lin_desc(rows, c_in, c_out, TYPES[dtype], c_in + beside, c_out + beside, c_out + beside, c_in + beside)
        self.x_codes, self.w_codes = (torch.full((n, eoq.lin_pitch(c_in)), 77, dtype=torch.int8, device=DEV) for n in (rows, c_out))
        self.x_scales, self.w_scales = torch.empty(rows, device=DEV), torch.empty(c_out, device=DEV)
        self.y, self.dx = (rows_in(torch.zeros(rows, c, dtype=dtype, device=DEV), beside, offset) for c in (c_out, c_in))
        self.dw, self.db = torch.full((c_out, c_in), float("nan"), device=DEV), torch.full((c_out,), float("nan"), device=DEV)
        size = max(eoq.eoq_lin_workspace_size(self.desc, eoq.EOQ_LIN_FWD), eoq.eoq_lin_workspace_size(self.desc, eoq.EOQ_LIN_BWD))
        self.ws = torch.full((size,), 255, dtype=torch.uint8, device=DEV)

    def code_weights(self):
        eoq.eoq_lin_quantize(handle(), self.w, eoq.EOQ_F32, self.c_out, self.c_in, self.c_in, self.w_codes, self.w_scales)

    def forward(self, keep=True):
        eoq.eoq_lin_fwd(handle(), self.desc, self.x, self.x_codes if keep else None, self.x_scales if keep else None, self.w_codes, self.w_scales, self.bias,
                        self.y, self.ws)

    def backward(self, dx=True, dw=True, db=True):
        eoq.eoq_lin_bwd(handle(), self.desc, self.dy, self.x_codes if dw else None, self.x_scales if dw else None, self.w_codes if dx else None,
                        self.w_scales if dx else None, self.dx if dx else None, self.dw if dw else None, self.db if db else None, self.ws)

    def oracle(self):
        xc, xs = ref.codes_of(self.x)
        wc, ws = ref.codes_of(self.w)
        return xc, xs, wc, ws

    def check_forward(self):
        xc, xs, wc, ws = self.oracle()
        y, bound = ref.forward(xc, xs, wc, ws, self.bias, self.dtype)
        ref.near(self.y, y, bound, "y")

    def check_codes(self):
        for got, scales, (codes, exact) in ((self.x_codes, self.x_scales, ref.codes_of(self.x)), (self.w_codes, self.w_scales, ref.codes_of(self.w))):
            assert torch.equal(got[:, :self.c_in].double(), codes)
            assert torch.equal(scales.double().nan_to_num(-1), exact.nan_to_num(-1))

    def check_backward(self, dx=True, dw=True, db=True):
        want = ref.backward(self.dy, *self.oracle(), self.dtype)
        for name, on in (("dx", dx), ("dw", dw), ("db", db)):
            if on:
                ref.near(getattr(self, name), *want[name], name)

    def untouched(self):
        """What lies between the rows of y and dx, and behind the last one, is as it was."""
        for t, c in ((self.y, self.c_out), (self.dx, self.c_in)):
            flat = torch.empty(0, dtype=t.dtype, device=DEV).set_(t.untyped_storage())
            n = self.rows * (c + self.beside)
            inside = flat[self.offset:self.offset + n].view(self.rows, -1)
            around = [bool(torch.isnan(p).all()) for p in (inside[:, c:], flat[:self.offset], flat[self.offset + n:])]
            assert around == [True] * 3


SIZES = [(1, 1, 1), (1, 16, 16), (1, 4096, 512), (2, 1000, 333), (5, 2048, 1000), (7, 129, 65), (8, 640, 48), (9, 64, 100), (16, 31, 17), (17, 128, 128), (31, 257, 300), (33, 513, 40),
         (77, 1024, 640), (98, 512, 300), (128, 128, 128), (129, 127, 129), (200, 96, 700), (300, 384, 257), (1000, 40, 33), (513, 1000, 259), (260, 2050, 520), (4100, 130, 131)]


@pytest.mark.parametrize("dtype", list(TYPES), ids=str)
@pytest.mark.parametrize("rows,c_in,c_out", SIZES)
def test_a_step(rows, c_in, c_out, dtype):
    l = Layer(rows, c_in, c_out, dtype, bias=(rows + c_in) % 3 != 0)
    status_clear()
    l.code_weights()
    l.forward()
    l.backward()
    assert status_clear() == 0
    l.check_codes()
    l.check_forward()
    l.check_backward()
    l.untouched()


@pytest.mark.parametrize("dtype", list(TYPES), ids=str)
@pytest.mark.parametrize("beside,offset", [(8, 0), (24, 8), (3, 0), (1, 1), (2, 6)])
@pytest.mark.parametrize("rows,c_in,c_out", [(3, 72, 40), (130, 264, 136), (70, 101, 57), (600, 48, 320)])
def test_parts_of_wider_rows(rows, c_in, c_out, beside, offset, dtype):
    l = Layer(rows, c_in, c_out, dtype, True, beside, offset)
    l.code_weights()
    l.forward()
    l.backward()
    l.check_codes()
    l.check_forward()
    l.check_backward()
    l.untouched()


@pytest.mark.parametrize("dtype", list(TYPES), ids=str)
@pytest.mark.parametrize("beside,offset", [(0, 0), (8, 8), (5, 3)])
@pytest.mark.parametrize("rows", [1, 2, 3, 5, 8, 9, 12, 16, 17, 25, 32, 33])
@pytest.mark.parametrize("c_in,c_out", [(16, 8), (63, 17), (64, 200), (130, 5000), (1000, 333), (4096, 64)])
def test_few_tokens(rows, c_in, c_out, beside, offset, dtype):
    """Coded by the call or beforehand: the same bits, whichever kernel does it."""
    l = Layer(rows, c_in, c_out, dtype, c_in % 2 == 0, beside, offset)
    l.code_weights()
    l.w_codes[:, c_in:] = 99
    l.forward(keep=False)
    l.check_forward()
    y = l.y.clone()
    l.forward()
    l.check_codes()
    assert torch.equal(l.y, y)
    l.x_codes[:, c_in:] = -5
    eoq.eoq_lin_fwd(handle(), l.desc, None, l.x_codes, l.x_scales, l.w_codes, l.w_scales, l.bias, l.y, l.ws)
    assert torch.equal(l.y, y)
    l.untouched()


@pytest.mark.parametrize("dtype,rows,c_in,c_out", [(torch.bfloat16, 2048, 1024, 1536), (torch.float16, 6272, 64, 256), (torch.float32, 1111, 2000, 999), (torch.bfloat16, 700, 8200, 300),
                                                   (torch.bfloat16, 6, 20000, 40), (torch.float32, 40, 9000, 70), (torch.float16, 257, 256, 6000)])
def test_large(dtype, rows, c_in, c_out):
    l = Layer(rows, c_in, c_out, dtype)
    l.code_weights()
    l.forward()
    l.backward()
    l.check_codes()
    l.check_forward()
    l.check_backward()


def test_calls_that_leave_something_out():
    l = Layer(150, 200, 96, torch.bfloat16)
    l.code_weights()
    l.forward(keep=False)
    assert (l.x_codes == 77).all()
    l.check_forward()
    l.forward()
    y = l.y.clone()
    eoq.eoq_lin_fwd(handle(), l.desc, None, l.x_codes, l.x_scales, l.w_codes, l.w_scales, l.bias, l.y, l.ws)
    assert torch.equal(l.y, y)
    for dx, dw, db in ((True, False, False), (False, True, False), (False, False, True), (True, False, True), (False, True, True), (True, True, False)):
        for t in (l.dx, l.dw, l.db):
            t.fill_(float("nan"))
        l.backward(dx, dw, db)
        l.check_backward(dx, dw, db)
        assert all(on or torch.isnan(t).all() for t, on in ((l.dx, dx), (l.dw, dw), (l.db, db)))


@pytest.mark.parametrize("rows,c_in,c_out", [(3, 40, 50), (140, 300, 130), (400, 64, 300)])
def test_rows_without_codes(rows, c_in, c_out):
    """A NaN or an infinity makes its token's (its channel's) results NaN and no others; zeros, numbers beneath the smallest scale and large ones are fine."""
    l = Layer(rows, c_in, c_out, torch.float32, bias=False)
    l.code_weights()
    l.x[0, c_in // 2], l.x[rows - 1, 0] = float("nan"), float("inf")
    l.x[1] = 0.0
    l.dy[0] = 0.0
    l.dy[2, 3], l.dy[2, c_out - 1] = float("-inf"), 1.0
    status_clear()
    l.forward()
    assert status_clear() == eoq.EOQ_DEV_NONFINITE
    l.check_codes()
    l.check_forward()
    l.x[0] = 1e-30 * torch.linspace(-1, 1, c_in, device=DEV)
    l.x[1] = 1e-37 * torch.linspace(-1, 1, c_in, device=DEV)
    l.x[rows - 1] = 3e38
    l.w[0], l.w[1] = 0.0, 1e-3
    l.code_weights()
    l.forward()
    assert status_clear() == 0
    l.check_codes()
    l.x[rows - 1] = 1.0
    for keep in (True, False):
        l.forward(keep)
        l.check_forward()
    l.x[0, 3] = float("nan")
    l.forward(keep=False)
    assert status_clear() == eoq.EOQ_DEV_NONFINITE
    l.check_forward()
    l.x[0, 3] = 0.0
    l.forward()
    l.backward()
    assert status_clear() == eoq.EOQ_DEV_NONFINITE
    l.check_backward()
    assert torch.isnan(l.dx[2]).all() and torch.isnan(l.dw[3]).all() and not torch.isnan(l.dw[c_out - 1]).any() and not torch.isnan(l.dw[2]).any()


@pytest.mark.parametrize("rows,c_in,c_out", [(5, 64, 48), (40, 70, 33), (700, 512, 600)])
@pytest.mark.parametrize("dtype", list(TYPES), ids=str)
def test_tokens_and_channels_without_codes(rows, c_in, c_out, dtype):
    """A token that is not finite takes its row of y and all of dw with it, a channel its column of y and all of dx; nothing else, whatever stands between the codes' rows."""
    for token, channel in ((1, None), (None, 2)):
        l = Layer(rows, c_in, c_out, dtype)
        if token is not None:
            l.x[token, 5] = float("inf")
        if channel is not None:
            l.w[channel, 0] = float("nan")
        status_clear()
        l.code_weights()
        l.forward()
        l.backward()
        assert status_clear() == eoq.EOQ_DEV_NONFINITE
        l.check_codes()
        l.check_forward()
        l.check_backward()
        assert bool(torch.isnan(l.dw).all()) == (token is not None) and bool(torch.isnan(l.dx).all()) == (channel is not None)
        assert int(torch.isnan(l.y).sum()) == (c_out if token is not None else rows)


@pytest.mark.parametrize("rows,c_in,c_out", [(6, 140000, 64), (300, 33, 140000), (270000, 40, 48)])
def test_sums_longer_than_an_int32_holds(rows, c_in, c_out):
    """Codes at -128 (which a program may hand over), reductions beyond 131,071: the parts are exact and added in 64 bits."""
    l = Layer(rows, c_in, c_out, torch.float32, bias=False)
    for codes, scales in ((l.x_codes, l.x_scales), (l.w_codes, l.w_scales)):
        codes.fill_(-128)
        codes[:, ::3] = 127
        scales.fill_(2.0 ** -10)
    eoq.eoq_lin_fwd(handle(), l.desc, None, l.x_codes, l.x_scales, l.w_codes, l.w_scales, None, l.y, l.ws)
    xc, wc = l.x_codes[:, :c_in].double(), l.w_codes[:, :c_in].double()
    y, bound = ref.forward(xc, l.x_scales.double(), wc, l.w_scales.double(), None, torch.float32)
    ref.near(l.y, y, bound, "y")
    l.backward()
    for name, (want, bound) in ref.backward(l.dy, xc, l.x_scales.double(), wc, l.w_scales.double(), torch.float32).items():
        ref.near(getattr(l, name), want, bound, name)


def test_differences():
    """The gradients are those of the layer's output: along random directions, at the codes' own values, to within the errors' rounding to 8 bits."""
    l = Layer(200, 96, 80, torch.float32)
    l.code_weights()
    l.forward()
    l.backward()
    xc, xs, wc, ws = l.oracle()
    x, w, dy = xc * xs[:, None], wc * ws[:, None], l.dy.double()
    loss = lambda x, w, b: float((dy * (x @ w.t() + b)).sum())  # noqa: E731
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    for name, at in (("dx", 0), ("dw", 1), ("db", 2)):
        here = [x, w, l.bias.double()]
        d = torch.randn(here[at].shape, generator=g, device=DEV, dtype=torch.float64)
        ends = []
        for sign in (0.5, -0.5):
            p = list(here)
            p[at] = p[at] + sign * d
            ends.append(loss(*p))
        got = float((getattr(l, name).double() * d).sum())
        # an error is off by half a step at most, 1/254 of its row's largest: through the weights (tokens) and along d
        u = (dy * ws).abs().amax(1, keepdim=True) / 254 * torch.ones_like(dy)
        v = (dy * xs[:, None]).abs().amax(0, keepdim=True) / 254 * torch.ones_like(dy)
        off = {"dx": float((u * (d @ wc.t()).abs()).sum()) if at == 0 else 0.0, "dw": float((v * (xc @ d.t()).abs()).sum()) if at == 1 else 0.0, "db": 0.0}[name]
        assert abs(got - (ends[0] - ends[1])) <= 1.01 * off + 1e-6 * float((dy.abs() * (x.abs() @ w.abs().t() + 1)).sum())


def test_captured_and_replayed():
    """A step in a graph, replayed on other inputs, gives the calls' own bits; two layers that share a workspace do not meet in it."""
    a, b = Layer(98, 512, 256, torch.bfloat16, seed=1), Layer(300, 256, 130, torch.bfloat16, seed=2)
    a.ws = b.ws = torch.empty(max(a.ws.numel(), b.ws.numel()), dtype=torch.uint8, device=DEV)

    def step():
        for l in (a, b):
            l.code_weights()
            l.forward()
        for l in (b, a):
            l.backward()

    def results():
        return [t.clone() for l in (a, b) for t in (l.y, l.dx, l.dw, l.db, l.x_codes, l.x_scales)]

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        for l in (a, b):
            l.x.mul_(-1.5)
            l.dy.add_(l.dy.flip(0) * 0.25)
            l.w.mul_(0.9)
        graph.replay()
        torch.cuda.synchronize()
        replayed = results()
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(replayed, results()))


def test_two_handles_side_by_side():
    other = eoq.eoq_create(0)
    layers = [Layer(500, 700, 333, torch.float16, seed=k) for k in range(2)]
    streams = [torch.cuda.Stream() for _ in layers]
    torch.cuda.synchronize()
    for _ in range(4):
        for l, s, h in zip(layers, streams, (handle(), other)):
            with torch.cuda.stream(s):
                eoq.eoq_lin_quantize(h, l.w, eoq.EOQ_F32, l.c_out, l.c_in, l.c_in, l.w_codes, l.w_scales)
                eoq.eoq_lin_fwd(h, l.desc, l.x, l.x_codes, l.x_scales, l.w_codes, l.w_scales, l.bias, l.y, l.ws)
                eoq.eoq_lin_bwd(h, l.desc, l.dy, l.x_codes, l.x_scales, l.w_codes, l.w_scales, l.dx, l.dw, l.db, l.ws)
    torch.cuda.synchronize()
    for l in layers:
        l.check_forward()
        l.check_backward()
    eoq.eoq_destroy(other)
