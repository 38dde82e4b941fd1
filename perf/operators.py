"""Group normalisation with an activation, activations kept in 8 bits, and the gradients taken from them, as cases that can be timed and
compared.

  norm      group norm and its activation on a channels-last tensor.  "forward": the output alone, as for a validation image.  "train": the
            forward pass, its backward pass, and between the two the input kept either as it is or in 8 bits ("kept").
  store     a tensor put away in 8 bits and read back: what a program does with the input of a layer that has no pass of its own here.
  weights   the weight gradient of a 1x1 convolution (a linear layer) from the errors and its input's 8-bit form.

8-bit form: int8 codes, and for every 32 neighbouring channels of a pixel one byte s; a value is code * 2^(s - 127), with the smallest step
2^(s - 127) that holds the block's largest magnitude in 127 steps (s at least 1).
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "fp16": 2, "bf16": 2}
BLOCK = 32
EPS = 1e-5
MOST_NORM = 64 * 112 * 112 * 64      # elements of a drawn normalisation: those of the largest listed one
MOST_STORE = 64 * 56 * 56 * 128
MOST_PRODUCTS = 16384 * 1024 * 4096  # multiply-adds of a drawn weight gradient


def listed():
    return [
        # a single image in the last stage of an ImageNet network: launch latency
        _norm("norm forward 512ch 7x7 b1", 1, 7, 7, 512, 32, "bf16", "silu", "forward", "none"),
        # a validation batch in the first stage of a bottleneck network: memory bandwidth
        _norm("norm forward 256ch 56x56 b32", 32, 56, 56, 256, 32, "fp16", "relu", "forward", "none"),
        # small-batch training, one layer's step: launches count
        _norm("norm train 256ch 14x14 b2", 2, 14, 14, 256, 32, "bf16", "silu", "train", "codes"),
        # the CIFAR-shaped network's widest images at its usual batch
        _norm("norm train 32ch 32x32 b128", 128, 32, 32, 32, 8, "fp32", "silu", "train", "codes"),
        # the first layer of an ImageNet network, the largest activation there is
        _norm("norm train 64ch 112x112 b64", 64, 112, 112, 64, 16, "bf16", "silu", "train", "codes"),
        # odd images, channels that are no power of two, groups of 15 channels, part of a wider tensor; the input kept as it is
        _norm("norm train ragged 120 of 144ch", 13, 45, 45, 120, 8, "fp16", "silu", "train", "input", 24),
        # one layer's input put away and fetched back, small
        _store("store 784 x 512", 784, 512, "bf16"),
        # an activation of the first stage at batch 64
        _store("store 200704 x 128", 64 * 56 * 56, 128, "bf16"),
        # rows that end inside a block
        _store("store 5365 x 1000", 5 * 37 * 29, 1000, "fp32"),
        # 1x1 convolutions of a bottleneck network: few pixels and wide, many pixels and narrow; and a wide linear layer
        _weights("weights 512 to 2048 7x7 b32", 32 * 7 * 7, 512, 2048, "bf16"),
        _weights("weights 64 to 256 56x56 b32", 32 * 56 * 56, 64, 256, "fp16"),
        _weights("weights 1024 to 4096 b16384", 16384, 1024, 4096, "bf16"),
    ]


def _norm(name, n, h, w, c, groups, dtype, act, what, kept, beside=0):
    return {"name": name, "kind": "norm", "n": n, "h": h, "w": w, "c": c, "groups": groups, "dtype": dtype, "act": act, "what": what, "kept": kept,
            "beside": beside}


def _store(name, rows, cols, dtype):
    return {"name": name, "kind": "store", "rows": rows, "cols": cols, "dtype": dtype}


def _weights(name, rows, c_in, c_out, dtype):
    return {"name": name, "kind": "weights", "rows": rows, "c_in": c_in, "c_out": c_out, "dtype": dtype}


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("norm", "norm", "store", "weights"))
    dtype = rng.choice(sorted(TYPES))
    if kind == "norm":
        while True:
            groups = rng.choice((1, 2, 4, 5, 8, 16, 32))
            c = groups * _log_int(rng, 1, 64)
            n, h, w = _log_int(rng, 1, 128), _log_int(rng, 1, 128), _log_int(rng, 1, 128)
            if 8 <= c <= 2048 and 4096 <= n * h * w * c <= MOST_NORM and (c // groups) * h * w >= 16:
                break
        what = rng.choice(("forward", "train", "train"))
        act = rng.choice(("none", "relu", "silu") if what == "forward" else ("none", "silu"))
        kept = "none" if what == "forward" else rng.choice(("codes", "input"))
        return {k: v for k, v in _norm("", n, h, w, c, groups, dtype, act, what, kept, rng.choice((0, 0, 8, 24))).items() if k != "name"}
    if kind == "store":
        while True:
            rows, cols = _log_int(rng, 1, 1 << 18), _log_int(rng, 16, 4096)
            if 4096 <= rows * cols <= MOST_STORE:
                break
        return {"kind": "store", "rows": rows, "cols": cols, "dtype": dtype}
    while True:
        rows, c_in, c_out = _log_int(rng, 1, 1 << 17), _log_int(rng, 8, 4096), _log_int(rng, 8, 4096)
        if (1 << 18) <= rows * c_in * c_out <= (MOST_PRODUCTS // 4 if dtype == "fp32" else MOST_PRODUCTS) and rows * max(c_in, c_out) <= 1 << 26:
            break
    return {"kind": "weights", "rows": rows, "c_in": c_in, "c_out": c_out, "dtype": dtype}


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    if case["kind"] == "norm":
        n, h, w, c, groups = (case[k] for k in ("n", "h", "w", "c", "groups"))
        # channels with spreads and means of their own, as a convolution leaves them
        x = normal(n, h, w, c + case["beside"])
        x.mul_(1.0 + 0.3 * normal(c + case["beside"])).add_(0.5 * normal(c + case["beside"]))
        x = x.to(dt)[..., :c]
        s = {"x": x, "gamma": 1.0 + 0.2 * normal(c), "beta": 0.2 * normal(c), "y": torch.empty(n, h, w, c, dtype=dt, device=DEV)}
        if case["what"] == "train":
            s["dy"] = (0.05 * normal(n, h, w, c)).to(dt)
            s["stats"] = torch.empty(n, groups, 2, device=DEV)
            s["dx"] = torch.empty_like(s["y"])
            s["dgamma"], s["dbeta"] = torch.empty(c, device=DEV), torch.empty(c, device=DEV)
            if case["kept"] == "codes":
                s["codes"] = torch.empty(n, h, w, c, dtype=torch.int8, device=DEV)
                s["exps"] = torch.empty(n * h * w, -(-c // BLOCK), dtype=torch.uint8, device=DEV)
    elif case["kind"] == "store":
        rows, cols = case["rows"], case["cols"]
        # behind an activation: half of the values small, channels of different size
        x = normal(rows, cols)
        x.mul_(torch.sigmoid(2.0 * x)).mul_(torch.exp(normal(cols)))
        s = {"x": x.to(dt), "back": torch.empty(rows, cols, dtype=dt, device=DEV), "codes": torch.empty(rows, cols, dtype=torch.int8, device=DEV),
             "exps": torch.empty(rows, -(-cols // BLOCK), dtype=torch.uint8, device=DEV)}
    else:
        rows, c_in, c_out = case["rows"], case["c_in"], case["c_out"]
        x = normal(rows, c_in)
        x.mul_(torch.sigmoid(2.0 * x)).mul_(torch.exp(0.5 * normal(c_in)))
        codes, exps = _to_codes(x)
        s = {"dy": (0.05 * normal(rows, c_out)).to(dt), "codes": codes, "exps": exps, "dw": torch.empty(c_out, c_in, device=DEV)}
    s["case"] = case
    return s


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    e = SIZE[case["dtype"]]
    if case["kind"] == "norm":
        pixels, c = case["n"] * case["h"] * case["w"], case["c"]
        kept = c + -(-c // BLOCK) if case["kept"] == "codes" else 0   # bytes a pixel
        b, f = pixels * c * 2 * e, pixels * c * 12
        if case["what"] == "train":
            # forward: x read, y and the 8-bit form written; backward: the errors and x in its kept form read, dx written
            b += pixels * (2 * c * e + (2 * kept if kept else c * e))
            f += pixels * c * 28
        return {"bytes": b + 4 * c * (2 if case["what"] == "forward" else 6), "flops": f}
    if case["kind"] == "store":
        rows, cols = case["rows"], case["cols"]
        return {"bytes": 2 * rows * (cols * (e + 1) + -(-cols // BLOCK)), "flops": 6 * rows * cols}
    rows, c_in, c_out = case["rows"], case["c_in"], case["c_out"]
    return {"bytes": rows * (c_out * e + c_in + -(-c_in // BLOCK)) + 4 * c_in * c_out, "flops": 2 * rows * c_in * c_out}


# ------------------------------------------------------------------ the plain forms

def _to_codes(x):
    """The 8-bit form of fp32 values [rows, cols]: integer arithmetic on the bits of each block's largest magnitude, then an exact scaling."""
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    v = torch.nn.functional.pad(x, (0, blocks * BLOCK - cols)).view(rows, blocks, BLOCK)
    s = ((v.abs().amax(2).view(torch.int32) + 0x1FFFF) >> 23).sub_(6).clamp_(min=1)
    per = ((254 - s) << 23).view(torch.float32)
    codes = torch.round(v * per[..., None]).to(torch.int8).view(rows, blocks * BLOCK)[:, :cols].contiguous()
    return codes, s.to(torch.uint8)


def _from_codes(codes, exps):
    rows, cols = codes.shape
    step = (exps.to(torch.int32) << 23).view(torch.float32)
    return codes.float() * step.repeat_interleave(BLOCK, 1)[:, :cols]


def _act(z, act):
    return z if act == "none" else z.clamp(min=0) if act == "relu" else z * torch.sigmoid(z)


def _act_slope(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).float()
    q = torch.sigmoid(z)
    return q * (1 + z * (1 - q))


def _run_plain(s):
    case = s["case"]
    dt = TYPES[case["dtype"]]
    if case["kind"] == "store":
        return {"back": _from_codes(*_to_codes(s["x"].float())).to(dt)}
    if case["kind"] == "weights":
        return {"dw": s["dy"].float().t() @ _from_codes(s["codes"], s["exps"])}
    n, h, w, c, groups = (case[k] for k in ("n", "h", "w", "c", "groups"))
    by_group = (n, h * w, groups, c // groups)
    x = s["x"].float()
    v = x.reshape(by_group)
    mean = v.mean((1, 3), keepdim=True)
    inv = 1.0 / torch.sqrt((v - mean).square().mean((1, 3), keepdim=True) + EPS)
    gamma, beta = s["gamma"].view(groups, c // groups), s["beta"].view(groups, c // groups)
    y = _act((v - mean) * inv * gamma + beta, case["act"]).view(n, h, w, c).to(dt)
    if case["what"] == "forward":
        return {"y": y}
    if case["kept"] == "codes":
        v = _from_codes(*_to_codes(x.reshape(-1, c))).view(by_group)
    unit = (v - mean) * inv
    dz = s["dy"].float().view(by_group) * _act_slope(unit * gamma + beta, case["act"])
    dgamma, dbeta = (dz * unit).sum((0, 1)).view(c), dz.sum((0, 1)).view(c)
    dz = dz * gamma
    dx = inv * (dz - dz.mean((1, 3), keepdim=True) - unit * (dz * unit).mean((1, 3), keepdim=True))
    return {"y": y, "dx": dx.view(n, h, w, c).to(dt), "dgamma": dgamma, "dbeta": dbeta}


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


def _workspace(s, size):
    """A program keeps the workspace of a layer beside its other buffers."""
    if "ws" not in s:
        s["ws"] = torch.empty(max(size, 256), dtype=torch.uint8, device=DEV)
    return s["ws"]


def _run_own(s):
    eoq = _library()
    case = s["case"]
    if "dtype" not in s:
        s["dtype"] = {"fp32": eoq.EOQ_F32, "fp16": eoq.EOQ_F16, "bf16": eoq.EOQ_BF16}[case["dtype"]]
    if case["kind"] == "store":
        rows, cols = case["rows"], case["cols"]
        eoq.eoq_ckpt_save(_handle, s["x"], s["dtype"], 0, rows, cols, cols, s["codes"], s["exps"])
        eoq.eoq_ckpt_load(_handle, s["codes"], s["exps"], rows, cols, s["back"], s["dtype"], cols)
        return {"back": s["back"]}
    if case["kind"] == "weights":
        rows, c_in, c_out = case["rows"], case["c_in"], case["c_out"]
        if "ws" not in s:
            _workspace(s, eoq.eoq_ckpt_wgrad_workspace_size(rows, c_out, c_in, s["dtype"]))
        eoq.eoq_ckpt_wgrad(_handle, s["dy"], s["dtype"], rows, c_out, c_out, s["codes"], s["exps"], c_in, s["dw"], s["ws"])
        return {"dw": s["dw"]}
    if "desc" not in s:
        act = {"none": eoq.EOQ_ACT_NONE, "relu": eoq.EOQ_ACT_RELU, "silu": eoq.EOQ_ACT_SILU}[case["act"]]
        s["desc"] = eoq.gn_desc(case["n"], case["h"] * case["w"], case["c"], case["groups"], s["dtype"], act, EPS, x_stride=case["c"] + case["beside"])
        _workspace(s, eoq.eoq_gn_workspace_size(s["desc"]))
    if case["what"] == "forward":
        eoq.eoq_gn_fwd(_handle, s["desc"], s["x"], s["gamma"], s["beta"], s["y"], None, None, None, s["ws"])
        return {"y": s["y"]}
    codes, exps = s.get("codes"), s.get("exps")
    eoq.eoq_gn_fwd(_handle, s["desc"], s["x"], s["gamma"], s["beta"], s["y"], s["stats"], codes, exps, s["ws"])
    eoq.eoq_gn_bwd(_handle, s["desc"], s["dy"], None, None if codes is not None else s["x"], codes, exps, s["gamma"], s["beta"], s["stats"],
                   s["dx"], s["dgamma"], s["dbeta"], s["ws"])
    return {"y": s["y"], "dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}


# ------------------------------------------------------------------ 64 bits

def _exact_restored(x):
    """Nearest multiples of each block's step, the step found from the quotient of the largest magnitude and 127 (exact at powers of two)."""
    rows, cols = x.shape
    out = torch.empty_like(x)
    for a in range(0, cols, BLOCK):
        part = x[:, a:a + BLOCK]
        m, k = torch.frexp(part.abs().amax(1, keepdim=True) / 127.0)
        k = torch.where(m == 0.5, k - 1, k)                      # the smallest power of two at or above the quotient
        k = torch.where(m == 0, torch.full_like(k, -126), k).clamp(min=-126)
        step = torch.ldexp(torch.ones_like(m), k)
        out[:, a:a + BLOCK] = torch.round(part / step) * step
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "store":
        return {"back": _exact_restored(s["x"].double())}
    if case["kind"] == "weights":
        codes, exps = s["codes"].double(), s["exps"].double()
        x = torch.cat([codes[:, BLOCK * b:BLOCK * (b + 1)] * torch.exp2(exps[:, b:b + 1] - 127.0) for b in range(exps.shape[1])], 1)
        return {"dw": torch.einsum("ro,ri->oi", s["dy"].double(), x)}
    n, h, w, c, groups = (case[k] for k in ("n", "h", "w", "c", "groups"))
    gamma, beta = s["gamma"].double(), s["beta"].double()
    train = case["what"] == "train"
    y = torch.empty(n, h * w, c, dtype=torch.float64, device=DEV)
    dx = torch.empty_like(y) if train else None
    dgamma, dbeta = torch.zeros_like(gamma), torch.zeros_like(beta)
    stats = torch.empty(n, groups, 2, dtype=torch.float64, device=DEV)
    for k in range(groups):                                      # a group at a time: [n, pixels * channels of the group]
        at = slice(k * (c // groups), (k + 1) * (c // groups))
        v = s["x"].reshape(n, h * w, c)[..., at].double().reshape(n, -1)
        mean = v.sum(1, keepdim=True) / v.shape[1]
        inv = ((v * v).sum(1, keepdim=True) / v.shape[1] - mean * mean + EPS) ** -0.5
        z = ((v - mean) * inv).view(n, h * w, -1) * gamma[at] + beta[at]
        y[..., at] = z if case["act"] == "none" else torch.maximum(z, torch.zeros_like(z)) if case["act"] == "relu" else z / (1 + torch.exp(-z))
        if train:
            stats[:, k, 0], stats[:, k, 1] = mean[:, 0], inv[:, 0]
    if not train:
        return {"y": y.view(n, h, w, c)}
    kept = s["x"].reshape(n * h * w, c).double()
    if case["kept"] == "codes":
        kept = _exact_restored(kept)
    kept = kept.view(n, h * w, c)
    for k in range(groups):
        at = slice(k * (c // groups), (k + 1) * (c // groups))
        mean, inv = (stats[:, k, j].view(n, 1, 1) for j in (0, 1))
        u = (kept[..., at] - mean) * inv
        z = u * gamma[at] + beta[at]
        e = s["dy"].view(n, h * w, c)[..., at].double()
        if case["act"] == "relu":
            e = e * (z > 0)
        elif case["act"] == "silu":
            q = 1 / (1 + torch.exp(-z))
            e = e * (q + z * q * (1 - q))
        dgamma[at], dbeta[at] = (e * u).sum((0, 1)), e.sum((0, 1))
        e = e * gamma[at]
        count = h * w * (c // groups)
        dx[..., at] = (e - e.sum((1, 2), keepdim=True) / count - u * ((e * u).sum((1, 2), keepdim=True) / count)) * inv
    return {"y": y.view(n, h, w, c), "dx": dx.view(n, h, w, c), "dgamma": dgamma, "dbeta": dbeta}
