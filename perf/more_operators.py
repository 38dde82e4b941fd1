"""Linear layers in 8-bit integers with a scale for each token and channel, forward and backward, and the norm and clipping of a step's
gradients, as cases that can be timed and compared.

  serve   a linear layer whose weights are kept as codes, on floating-point tokens: the tokens are coded, multiplied, scaled.
  train   one step of such a layer: tokens and weights coded, the output, then from its errors the gradients of tokens, weights and bias.
  norm    the norm of all gradients of a step together.
  clip    that norm, and the gradients scaled down to it where it is too large, into another buffer.

Codes: a row of values has the scale max(largest magnitude, 2^-119) / 127 and the codes R(value * per), ties to even, with
per = 127 / max(largest magnitude, 2^-119) rounded to fp32.  A token is a row of the input, a channel a row of the weights [c_out][c_in].
Errors are coded twice: with the weights' scales multiplied in (in fp32) and a scale for each token, for the gradient of the tokens; with the
tokens' scales multiplied in and a scale for each channel, for the gradient of the weights.  Every product is then one of integers.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "fp16": 2, "bf16": 2}
TINY = 2.0 ** -119
MOST_SERVE = 8192 * 4096 * 4096     # multiply-adds of a drawn product: those of the largest listed one
MOST_TRAIN = 16384 * 1024 * 4096
MOST_CLIP = 200_000_000             # gradients of a drawn step


def listed():
    return [
        # a single token through a square layer: the weights' bytes, latency
        _lin("serve 1 x 4096 to 4096", "serve", 1, 4096, 4096, "bf16", False),
        # a handful of images in front of the classifier of a bottleneck network
        _lin("serve 5 x 2048 to 1000", "serve", 5, 2048, 1000, "fp16", True),
        # tokens of a short batch: neither many nor one
        _lin("serve 77 x 1024 to 4096", "serve", 77, 1024, 4096, "bf16", True),
        # a 1x1 convolution of a bottleneck network, 56 x 56 at batch 32: many pixels, few channels
        _lin("serve 100352 x 64 to 256", "serve", 32 * 56 * 56, 64, 256, "fp16", True),
        # a long prompt or a large batch through a wide layer: the tensor cores
        _lin("serve 8192 x 4096 to 4096", "serve", 8192, 4096, 4096, "bf16", True),
        # small-batch training, a 1x1 convolution of the last stage at 7 x 7 and batch 2: launches
        _lin("train 98 x 512 to 2048", "train", 98, 512, 2048, "bf16", True),
        # odd sizes, tokens that are part of wider rows, in fp32
        _lin("train 5365 x 1000 to 333", "train", 5365, 1000, 333, "fp32", True, 24),
        # a wide linear layer over many tokens
        _lin("train 16384 x 1024 to 4096", "train", 16384, 1024, 4096, "bf16", False),
        # the gradients of a small network: launch latency
        _grad("norm 24 tensors 0.1M", "norm", 24, 100_000, "fp32", False, 0.5),
        # a bottleneck network's gradients in two types, as a mixed-precision step has them, packed one behind the other
        _grad("norm 161 tensors 25.6M mixed", "norm", 161, 25_600_000, "mixed", True, 2.0),
        # a residual network of 18 layers, norm too large: every gradient is scaled
        _grad("clip 62 tensors 11.7M", "clip", 62, 11_700_000, "fp32", False, 3.0),
        # the gradients of a large model in two types, more than the cache holds
        _grad("clip 290 tensors 200M mixed", "clip", 290, 200_000_000, "mixed", True, 1.5),
    ]


def _lin(name, kind, rows, c_in, c_out, dtype, bias, beside=0):
    return {"name": name, "kind": kind, "rows": rows, "c_in": c_in, "c_out": c_out, "dtype": dtype, "bias": bias, "beside": beside}


def _grad(name, kind, count, total, dtype, packed, norm):
    """norm: of all gradients together, about; the limit is 1."""
    return {"name": name, "kind": kind, "count": count, "total": total, "dtype": dtype, "packed": packed, "norm": norm}


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("serve", "serve", "train", "train", "norm", "clip"))
    if kind in ("serve", "train"):
        most = MOST_SERVE if kind == "serve" else MOST_TRAIN
        while True:
            rows, c_in, c_out = _log_int(rng, 1, 1 << 17), _log_int(rng, 16, 8192), _log_int(rng, 16, 8192)
            if rng.random() < 0.5:
                c_in, c_out = -(-c_in // 16) * 16, -(-c_out // 16) * 16
            if (1 << 18) <= rows * c_in * c_out <= most and rows * max(c_in, c_out) <= 1 << 26:
                break
        case = _lin("", kind, rows, c_in, c_out, rng.choice(sorted(TYPES)), rng.random() < 0.5, rng.choice((0, 0, 8, 24)))
    else:
        total = _log_int(rng, 1000, MOST_CLIP)
        case = _grad("", kind, _log_int(rng, 1, min(400, total // 8)), total, rng.choice(("fp32", "bf16", "fp16", "mixed")), rng.random() < 0.5,
                     rng.choice((0.5, 3.0)))
    del case["name"]
    return case


def _sizes(case):
    """Elements of each tensor of a step, and for each whether it is in fp32: some hold most of them, the others are vectors of channels."""
    rng = random.Random(case["count"] * 7919 + case["total"])
    share = [math.exp(rng.gauss(0.0, 2.0)) for _ in range(case["count"])]
    whole = sum(share)
    sizes = [max(1, int(case["total"] * s / whole)) for s in share]
    wide = [case["dtype"] == "fp32" or (case["dtype"] == "mixed" and rng.random() < 0.3) for _ in sizes]
    return sizes, wide


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    s = {"case": case}
    if case["kind"] in ("norm", "clip"):
        sizes, wide = _sizes(case)
        narrow = torch.float16 if case["dtype"] == "fp16" else torch.bfloat16
        places, ends = [], {True: 0, False: 0}
        for n, w in zip(sizes, wide):
            step = 1 if case["packed"] else 64
            places.append(ends[w])
            ends[w] += -(-n // step) * step
        # a bucket for each type; layers have gradients of different size
        spread = [math.exp(0.5 * random.Random(seed + k).gauss(0.0, 1.0)) for k in range(len(sizes))]
        whole = math.sqrt(sum(n * v * v for n, v in zip(sizes, spread)))
        s["buckets"], s["out"] = {}, {}
        for w in (True, False):
            if ends[w]:
                flat = normal(ends[w])
                at = 0
                for n, p, k, v in zip(sizes, places, wide, spread):
                    if k == w:
                        flat[at:p].zero_()
                        flat[p:p + n].mul_(case["norm"] * v / whole)
                        at = p + n
                flat[at:].zero_()
                s["buckets"][w] = flat.to(torch.float32 if w else narrow)
                if case["kind"] == "clip":
                    s["out"][w] = torch.zeros_like(s["buckets"][w])
        s["tensors"] = [s["buckets"][w][p:p + n] for n, p, w in zip(sizes, places, wide)]
        s["clipped"] = [s["out"][w][p:p + n] for n, p, w in zip(sizes, places, wide)] if case["kind"] == "clip" else None
        s["norm"] = torch.empty(1, device=DEV)
        return s
    rows, c_in, c_out, dt = case["rows"], case["c_in"], case["c_out"], TYPES[case["dtype"]]
    # behind an activation: half of the values small, channels of different size
    x = normal(rows, c_in + case["beside"])
    x.mul_(torch.sigmoid(2.0 * x)).mul_(torch.exp(0.5 * normal(c_in + case["beside"])))
    s["x"] = x.to(dt)[:, :c_in]
    w = normal(c_out, c_in) * (torch.exp(0.3 * normal(c_out, 1)) / math.sqrt(c_in))
    s["bias"] = 0.1 * normal(c_out) if case["bias"] else None
    s["y"] = torch.empty(rows, c_out, dtype=dt, device=DEV)
    pitch = -(-c_in // 16) * 16
    if case["kind"] == "serve":
        codes, s["w_scales"] = _to_codes(w)
        s["w_codes"] = torch.zeros(c_out, pitch, dtype=torch.int8, device=DEV)
        s["w_codes"][:, :c_in] = codes
        return s
    s["w"] = w
    s["w_codes"], s["w_scales"] = torch.empty(c_out, pitch, dtype=torch.int8, device=DEV), torch.empty(c_out, device=DEV)
    s["x_codes"], s["x_scales"] = torch.empty(rows, pitch, dtype=torch.int8, device=DEV), torch.empty(rows, device=DEV)
    s["dy"] = (0.05 * normal(rows, c_out + case["beside"]) * torch.exp(0.5 * normal(rows, 1))).to(dt)[:, :c_out]
    s["dx"], s["dw"], s["db"] = torch.empty(rows, c_in, dtype=dt, device=DEV), torch.empty(c_out, c_in, device=DEV), torch.empty(c_out, device=DEV)
    return s


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    if case["kind"] in ("norm", "clip"):
        sizes, wide = _sizes(case)
        b = sum(n * (4 if w else 2) for n, w in zip(sizes, wide))
        return {"bytes": b * (2 if case["kind"] == "clip" else 1) + 4, "flops": sum(sizes) * (3 if case["kind"] == "clip" else 2)}
    e, rows, c_in, c_out = SIZE[case["dtype"]], case["rows"], case["c_in"], case["c_out"]
    vectors = 4 * c_out * (2 if case["bias"] else 1)
    if case["kind"] == "serve":
        return {"bytes": rows * (c_in + c_out) * e + c_in * c_out + vectors, "flops": 2 * rows * c_in * c_out}
    # x, w, bias and the errors read; y, the gradients of x, w and bias written
    return {"bytes": 2 * rows * (c_in + c_out) * e + 8 * c_in * c_out + vectors, "flops": 6 * rows * c_in * c_out}


# ------------------------------------------------------------------ the plain forms

def _to_codes(v, dim=1):
    """Codes of fp32 values and their scales, one for each row (dim = 1) or column (dim = 0); the product that is rounded is exact in 64 bits."""
    top = v.abs().amax(dim, keepdim=True).clamp(min=TINY).double()
    codes = torch.round(v.double() * (127.0 / top).float().double()).to(torch.int8)
    return codes, (top / 127.0).float().squeeze(dim)


def _run_plain(s):
    case = s["case"]
    if case["kind"] in ("norm", "clip"):
        # gaps between tensors hold zeros
        norm = torch.sqrt(sum(b.double().square().sum() for b in s["buckets"].values()))
        if case["kind"] == "norm":
            return {"norm": norm.float().view(1)}
        scale = torch.where(norm > 1.0, 1.0 / norm, 1.0).float()
        return {"norm": norm.float().view(1), "clipped": {str(w): (b.float() * scale).to(b.dtype) for w, b in s["buckets"].items()}}
    dt, c_in = TYPES[case["dtype"]], case["c_in"]
    x, x_scales = _to_codes(s["x"].float())
    w, w_scales = _to_codes(s["w"]) if case["kind"] == "train" else (s["w_codes"][:, :c_in], s["w_scales"])
    x, w = x.float(), w.float()
    y = (x @ w.t()) * x_scales[:, None] * w_scales
    if s["bias"] is not None:
        y = y + s["bias"]
    if case["kind"] == "serve":
        return {"y": y.to(dt)}
    dy = s["dy"].float()
    by_token, token_scales = _to_codes(dy * w_scales)
    by_channel, channel_scales = _to_codes(dy * x_scales[:, None], 0)
    dx = (by_token.float() @ w) * token_scales[:, None]
    dw = (by_channel.float().t() @ x) * channel_scales[:, None]
    return {"y": y.to(dt), "dx": dx.to(dt), "dw": dw, "db": dy.sum(0)}


# ------------------------------------------------------------------ the framework's calls

_eoq = None
_handle = None


def _library():
    global _eoq, _handle
    if _eoq is None:
        from paper_2105_13890_b200 import eoq

        _handle = eoq.eoq_create(0)
        _eoq = eoq
    return _eoq


def _workspace(size):
    return torch.empty(max(size, 256), dtype=torch.uint8, device=DEV)


def _run_own(s):
    eoq = _library()
    case = s["case"]
    if case["kind"] in ("norm", "clip"):
        if "list" not in s:   # a program keeps the list of its gradients, and a workspace
            s["list"] = eoq.grad_list(s["tensors"], s["clipped"])
            s["ws"] = _workspace(eoq.eoq_grad_workspace_size(s["list"]))
        if case["kind"] == "norm":
            eoq.eoq_grad_norm(_handle, s["list"], s["norm"], s["ws"])
            return {"norm": s["norm"]}
        eoq.eoq_grad_clip(_handle, s["list"], 1.0, s["norm"], s["ws"])
        return {"norm": s["norm"], "clipped": {str(w): b for w, b in s["out"].items()}}
    if "desc" not in s:
        dtype = {"fp32": eoq.EOQ_F32, "fp16": eoq.EOQ_F16, "bf16": eoq.EOQ_BF16}[case["dtype"]]
        s["desc"] = eoq.lin_desc(case["rows"], case["c_in"], case["c_out"], dtype, x_stride=case["c_in"] + case["beside"],
                                 dy_stride=case["c_out"] + case["beside"])
        s["ws"] = _workspace(max(eoq.eoq_lin_workspace_size(s["desc"], eoq.EOQ_LIN_FWD), eoq.eoq_lin_workspace_size(s["desc"], eoq.EOQ_LIN_BWD)
                                 if case["kind"] == "train" else 0))
    if case["kind"] == "serve":
        eoq.eoq_lin_fwd(_handle, s["desc"], s["x"], None, None, s["w_codes"], s["w_scales"], s["bias"], s["y"], s["ws"])
        return {"y": s["y"]}
    eoq.eoq_lin_quantize(_handle, s["w"], eoq.EOQ_F32, case["c_out"], case["c_in"], case["c_in"], s["w_codes"], s["w_scales"])
    eoq.eoq_lin_fwd(_handle, s["desc"], s["x"], s["x_codes"], s["x_scales"], s["w_codes"], s["w_scales"], s["bias"], s["y"], s["ws"])
    eoq.eoq_lin_bwd(_handle, s["desc"], s["dy"], s["x_codes"], s["x_scales"], s["w_codes"], s["w_scales"], s["dx"], s["dw"], s["db"], s["ws"])
    return {"y": s["y"], "dx": s["dx"], "dw": s["dw"], "db": s["db"]}


# ------------------------------------------------------------------ 64 bits

def _exact_codes(v):
    """Codes in 64 bits and scales of the rows of fp32 values: the step back to a value is the scale, the step to a code an fp32 number."""
    top = torch.maximum(v.abs().max(1).values, torch.tensor(TINY, device=v.device)).double()
    per = torch.div(torch.full_like(top, 127.0), top).float().double()
    up = torch.floor(v.double() * per[:, None] + 0.5)
    tie = (up - v.double() * per[:, None] == 0.5) & (torch.remainder(up, 2.0) == 1.0)
    return up - tie.double(), torch.div(top, torch.full_like(top, 127.0)).float().double()


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("norm", "clip"):
        total = torch.zeros((), dtype=torch.float64, device=DEV)
        for t in s["tensors"]:
            total += torch.dot(t.double(), t.double())
        norm = total ** 0.5
        if case["kind"] == "norm":
            return {"norm": norm.view(1)}
        for t, c in zip(s["tensors"], s["clipped"]):
            c.copy_(t)
        limit = torch.clamp(norm, min=1.0)
        return {"norm": norm.view(1), "clipped": {str(w): b.double() / limit for w, b in s["out"].items()}}
    x, x_scales = _exact_codes(s["x"].float())
    if case["kind"] == "serve":
        w, w_scales = s["w_codes"][:, :case["c_in"]].double(), s["w_scales"].double()
    else:
        w, w_scales = _exact_codes(s["w"])
    y = torch.einsum("tk,nk->tn", x * x_scales[:, None], w * w_scales[:, None])
    if s["bias"] is not None:
        y += s["bias"].double()
    if case["kind"] == "serve":
        return {"y": y}
    dy = s["dy"].double()
    tokens, token_scales = _exact_codes((dy * w_scales).float())
    channels, channel_scales = _exact_codes((dy * x_scales[:, None]).float().t().contiguous())
    return {"y": y, "dx": torch.einsum("tn,nk->tk", tokens * token_scales[:, None], w),
            "dw": torch.einsum("nt,tk->nk", channels * channel_scales[:, None], x), "db": dy.sum(0)}
