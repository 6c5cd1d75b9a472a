"""Workloads of the group-norm, 8-bit checkpoint and linear weight-gradient operators, as a training or evaluation program calls them.

A case is one pass through an operator of `paper_1412_2302_b200.operators`:

  norm           group_norm: y = act(norm(x) * weight + bias) on channels-last x [n, h, w, c], with the statistics a backward
                 pass needs
  norm_backward  group_norm_backward from x and the statistics that the forward pass kept
  norm_train     group_norm, which keeps its input as an 8-bit checkpoint, then group_norm_backward from that checkpoint
  checkpoint     checkpoint_encode, then checkpoint_decode: an activation laid away and fetched again
  linear_grad    linear_weight_grad: dw = dy^T x of a linear layer whose input x was kept as an 8-bit checkpoint

A checkpoint holds blocks of 32 consecutive channels of one position (the last block of a row may be shorter): a byte per value and one
byte E per block; a value is code * 2^(E - 127).  E is the smallest exponent with which the block's largest magnitude stays within 127
(codes int8) or 448 (codes float8 e4m3), codes are rounded to nearest even, and a block with an infinity or NaN has E = 255 and stands
for NaN throughout.

Ranges: 1 to 512 samples of 1 x 1 to 256 x 256 positions, 1 to 32 groups of 1 to 64 channels, dense or inside a larger grid; bf16, fp16 and
fp32; linear layers of 8 to 9216 features over 1 to 16384 rows, bf16 gradients.
"""
import math

import torch

own = False                                 # set by the measuring program: the plain form, or this repository's operators

EPS = 1e-5
MAX_ELEMENTS = 512 * 55 * 55 * 96
MAX_MACS = 8192 * 4096 * 4096
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZES = {"bf16": 2, "fp16": 2, "fp32": 4}


def _norm(kind, n, h, w, c, groups, dtype, activation, padded=False, codes="int8"):
    case = {"kind": kind, "n": n, "h": h, "w": w, "c": c, "groups": groups, "dtype": dtype, "activation": activation, "padded": padded}
    if kind == "norm_train":
        case["codes"] = codes
    return case


def _checkpoint(n, h, w, c, dtype, codes, padded=False):
    return {"kind": "checkpoint", "n": n, "h": h, "w": w, "c": c, "dtype": dtype, "codes": codes, "padded": padded}


def _linear(rows, n_in, n_out, codes):
    return {"kind": "linear_grad", "rows": rows, "in": n_in, "out": n_out, "codes": codes}


def listed():
    return [
        # one picture of an evaluation, behind a 13 x 13 layer of 384 channels: latency
        dict(_norm("norm", 1, 13, 13, 384, 32, "bf16", "relu"), name="norm_1x13x13x384"),
        # the first layer of a minibatch of 128, in the 57 x 57 grid that the convolutions read
        dict(_norm("norm", 128, 55, 55, 96, 32, "bf16", "relu", padded=True), name="norm_128x55x55x96_grid"),
        # full precision, channels that fill neither a vector nor a block
        dict(_norm("norm", 5, 27, 29, 100, 20, "fp32", "silu"), name="norm_5x27x29x100_fp32"),
        # the second layer of a minibatch, trained from 8-bit checkpoints
        dict(_norm("norm_train", 128, 27, 27, 256, 32, "bf16", "silu"), name="norm_train_128x27x27x256_int8"),
        # the first layer of the largest minibatch
        dict(_norm("norm_train", 512, 55, 55, 96, 32, "bf16", "silu", codes="e4m3"), name="norm_train_512x55x55x96_e4m3"),
        # a small minibatch in half precision
        dict(_norm("norm_backward", 2, 13, 13, 256, 32, "fp16", "relu"), name="norm_backward_2x13x13x256_fp16"),
        # one large picture at full resolution: few samples, many positions
        dict(_norm("norm_backward", 1, 256, 256, 128, 32, "bf16", "silu"), name="norm_backward_1x256x256x128"),
        # an activation of the second layer laid away and fetched again
        dict(_checkpoint(128, 27, 27, 256, "bf16", "int8"), name="checkpoint_128x27x27x256_int8"),
        # rows that end inside a block
        dict(_checkpoint(7, 13, 13, 100, "fp32", "e4m3"), name="checkpoint_7x13x13x100_fp32_e4m3"),
        # the first FC layer at the paper's minibatch: bound by writing the gradient
        dict(_linear(128, 9216, 4096, "int8"), name="linear_grad_128x9216x4096_int8"),
        # a 1 x 1 layer between two widths of 4096 over 8192 positions: bound by arithmetic
        dict(_linear(8192, 4096, 4096, "e4m3"), name="linear_grad_8192x4096x4096_e4m3"),
        # the classifier at an odd minibatch
        dict(_linear(173, 4096, 1000, "int8"), name="linear_grad_173x4096x1000_int8"),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("norm", "norm", "norm_backward", "norm_train", "norm_train", "checkpoint", "linear_grad", "linear_grad"))
    codes = rng.choice(("int8", "e4m3"))
    if kind == "linear_grad":
        rows, n_in, n_out = _log_uniform(rng, 1, 16384), _log_uniform(rng, 8, 9216), _log_uniform(rng, 8, 4096)
        if rng.random() < 0.6:              # widths of most layers; the others may be odd
            n_in, n_out = (n_in + 31) // 32 * 32, (n_out + 7) // 8 * 8
        return _linear(max(1, min(rows, MAX_MACS // (n_in * n_out))), n_in, n_out, codes)
    groups = rng.choice((1, 2, 4, 5, 8, 16, 20, 32, 32, 32))
    c = groups * _log_uniform(rng, 1, 64)
    h = _log_uniform(rng, 1, 256)
    w = max(1, min(256, h + rng.choice((0, 0, 0, 1, -1, 5))))
    n = max(1, min(_log_uniform(rng, 1, 512), MAX_ELEMENTS // (h * w * c)))
    dtype = rng.choice(("bf16", "bf16", "bf16", "fp16", "fp32"))
    padded = rng.random() < 0.3
    if kind == "checkpoint":
        return _checkpoint(n, h, w, c, dtype, codes, padded)
    # relu has a jump in its derivative, which only statistics of the same bits put at the same place
    activation = rng.choice(("none", "silu") if kind == "norm_train" else ("none", "relu", "silu"))
    return _norm(kind, n, h, w, c, groups, dtype, activation, padded, codes)


# ---------------------------------------------------------------- inputs
def _activation_tensor(gen, case):
    """[n, h, w, c] with a mean and a spread of its own for each channel, as a convolution leaves it; `padded`: a view of a grid that
    has two more rows and columns."""
    n, h, w, c = case["n"], case["h"], case["w"], case["c"]
    pad = 2 if case["padded"] else 0
    grid = torch.randn((n, h + pad, w + pad, c), device="cuda", generator=gen)
    spread = torch.rand(c, device="cuda", generator=gen) + 0.5
    shift = torch.randn(c, device="cuda", generator=gen) * 0.5
    return grid.mul_(spread).add_(shift).to(DTYPES[case["dtype"]])[:, :h, :w]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    kind = case["kind"]
    state = {"case": case, "kind": kind}
    if kind == "linear_grad":
        rows, n_in, n_out = case["rows"], case["in"], case["out"]
        x = torch.randn((rows, n_in), device="cuda", generator=gen)
        x = torch.relu(x.mul_(torch.rand(n_in, device="cuda", generator=gen) + 0.5).add_(0.2))      # behind a ReLU
        state["codes"], state["scales"] = _plain_encode(x, case["codes"])
        # gradients of a mean over the rows
        state["dy"] = (torch.randn((rows, n_out), device="cuda", generator=gen) / rows).to(torch.bfloat16)
    else:
        state["x"] = _activation_tensor(gen, case)
    if kind.startswith("norm"):
        c = case["c"]
        state["weight"] = torch.rand(c, device="cuda", generator=gen) + 0.5
        state["bias"] = torch.randn(c, device="cuda", generator=gen) * 0.2
    if kind in ("norm_backward", "norm_train"):
        state["dy"] = _activation_tensor(gen, case)
    if kind == "norm_backward":
        state["mean"], state["rstd"] = _plain_statistics(state["x"].float(), case["groups"])
    torch.cuda.synchronize()
    return state


# ---------------------------------------------------------------- the plain forms
def _plain_statistics(x, groups):
    n, c = x.shape[0], x.shape[-1]
    xg = x.reshape(n, -1, groups, c // groups)
    mean = xg.mean(dim=(1, 3))
    var = (xg - mean[:, None, :, None]).square().mean(dim=(1, 3))
    return mean, torch.rsqrt(var + EPS)


def _per_channel(stat, c):
    """[n, groups] -> [n, 1, 1, c]"""
    return stat.repeat_interleave(c // stat.shape[1], dim=1)[:, None, None, :]


def _plain_forward(x, weight, bias, mean, rstd, activation):
    c = x.shape[-1]
    z = (x - _per_channel(mean, c)) * _per_channel(rstd, c) * weight + bias
    if activation == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if activation == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _plain_backward(dy, x, weight, bias, mean, rstd, activation):
    n, c, groups = x.shape[0], x.shape[-1], mean.shape[1]
    rstd_c = _per_channel(rstd, c)
    xhat = (x - _per_channel(mean, c)) * rstd_c
    dz = dy
    if activation == "relu":
        # 64 bits: which side of the jump a value is on
        z = (x.double() - _per_channel(mean, c)) * rstd_c * weight.double() + bias
        dz = torch.where(z > 0, dy, torch.zeros_like(dy))
    elif activation == "silu":
        z = xhat * weight + bias
        s = 1 / (1 + torch.exp(-z))
        dz = dy * (s * (1 + z * (1 - s)))
    dbias = dz.sum(dim=(0, 1, 2))
    dweight = (dz * xhat).sum(dim=(0, 1, 2))
    g = dz * weight
    gg, xg = g.reshape(n, -1, groups, c // groups), xhat.reshape(n, -1, groups, c // groups)
    c1, c2 = gg.mean(dim=(1, 3)), (gg * xg).mean(dim=(1, 3))
    dx = rstd_c * (g - _per_channel(c1, c) - xhat * _per_channel(c2, c))
    return dx, dweight, dbias


def _power_of_two(e):
    """2^(e - 127) as fp32 for e of 0 to 254, by its bits (0: a subnormal)"""
    return torch.where(e > 0, e << 23, torch.full_like(e, 1 << 22)).to(torch.int32).view(torch.float32)


def _plain_encode(x, codes):
    """x fp32 [..., c] -> codes like x, exponents [..., ceil(c / 32)]"""
    c = x.shape[-1]
    blocks = (c + 31) // 32
    xp = torch.nn.functional.pad(x, (0, blocks * 32 - c)).reshape(*x.shape[:-1], blocks, 32)
    amax = xp.abs().amax(dim=-1)
    bits = amax.view(torch.int32)
    # the exponent field, one more where the mantissa is above 127/64 (448/256)
    e = ((bits + 0x1FFFF) >> 23) - 6 if codes == "int8" else ((bits + 0x1FFFFF) >> 23) - 8
    e = torch.where(amax.isfinite(), e.clamp(min=0), torch.full_like(e, 255))
    inverse = _power_of_two(254 - e.clamp(max=253))
    q = (xp * inverse[..., None]).reshape(*x.shape[:-1], blocks * 32)[..., :c]
    # the codes of a block that stands for NaN are zero
    q = torch.where((e == 255).repeat_interleave(32, dim=-1)[..., :c], torch.zeros_like(q), q)
    q = q.round().to(torch.int8) if codes == "int8" else q.to(torch.float8_e4m3fn)
    return q.contiguous(), e.to(torch.uint8)


def _plain_decode(codes, scales):
    """fp32 values"""
    e = scales.int()
    s = torch.where(e == 255, torch.full_like(e, float("nan"), dtype=torch.float32), _power_of_two(e))
    return codes.float() * s.repeat_interleave(32, dim=-1)[..., :codes.shape[-1]]


def _run_plain(state):
    case, kind = state["case"], state["kind"]
    if kind == "linear_grad":
        return state["dy"].float().t() @ _plain_decode(state["codes"], state["scales"])
    x, dtype = state["x"].float(), state["x"].dtype
    if kind == "checkpoint":
        return _plain_decode(*_plain_encode(x, case["codes"])).to(dtype)
    weight, bias, activation = state["weight"], state["bias"], case["activation"]
    if kind == "norm_backward":
        dx, dweight, dbias = _plain_backward(state["dy"].float(), x, weight, bias, state["mean"], state["rstd"], activation)
        return {"dx": dx.to(dtype), "dweight": dweight, "dbias": dbias}
    mean, rstd = _plain_statistics(x, case["groups"])
    y = _plain_forward(x, weight, bias, mean, rstd, activation).to(dtype)
    if kind == "norm":
        return {"y": y, "mean": mean, "rstd": rstd}
    kept = _plain_decode(*_plain_encode(x, case["codes"]))
    del x
    dx, dweight, dbias = _plain_backward(state["dy"].float(), kept, weight, bias, mean, rstd, activation)
    return {"y": y, "dx": dx.to(dtype), "dweight": dweight, "dbias": dbias}


# ---------------------------------------------------------------- the framework's operators
def _run_own(state):
    from paper_1412_2302_b200 import operators as ops
    case, kind = state["case"], state["kind"]
    if kind == "linear_grad":
        return ops.linear_weight_grad(state["dy"], ops.Checkpoint(state["codes"], state["scales"]))
    x = state["x"]
    if kind == "checkpoint":
        return ops.checkpoint_decode(ops.checkpoint_encode(x, case["codes"]), x.dtype)
    groups, weight, bias, activation = case["groups"], state["weight"], state["bias"], case["activation"]
    if kind == "norm_backward":
        dx, dweight, dbias = ops.group_norm_backward(state["dy"], x, state["mean"], state["rstd"], weight, bias, activation=activation)
        return {"dx": dx, "dweight": dweight, "dbias": dbias}
    if kind == "norm":
        r = ops.group_norm(x, groups, weight, bias, eps=EPS, activation=activation)
        return {"y": r.y, "mean": r.mean, "rstd": r.rstd}
    r = ops.group_norm(x, groups, weight, bias, eps=EPS, activation=activation, keep_input=case["codes"])
    dx, dweight, dbias = ops.group_norm_backward(state["dy"], r.input, r.mean, r.rstd, weight, bias, activation=activation)
    return {"y": r.y, "dx": dx, "dweight": dweight, "dbias": dbias}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["kind"] == "linear_grad":
        rows, n_in, n_out = case["rows"], case["in"], case["out"]
        return {"bytes": rows * (n_in + (n_in + 31) // 32) + 2 * rows * n_out + 4 * n_in * n_out, "flops": 2 * rows * n_in * n_out}
    n, positions, c = case["n"], case["n"] * case["h"] * case["w"], case["c"]
    elements, size = positions * c, SIZES[case["dtype"]]
    kept = elements + positions * ((c + 31) // 32)
    if case["kind"] == "checkpoint":
        # laid away, and fetched again
        return {"bytes": 2 * (size * elements + kept), "flops": 4 * elements}
    small = 4 * 2 * (c + n * case["groups"])          # weight and bias (or their gradients), statistics
    act = {"none": 0, "relu": 1, "silu": 4}[case["activation"]]
    forward = {"bytes": 2 * size * elements + small, "flops": (6 + act) * elements}
    if case["kind"] == "norm":
        return forward
    if case["kind"] == "norm_backward":
        return {"bytes": 3 * size * elements + 2 * small, "flops": (12 + 2 * act) * elements}
    return {"bytes": forward["bytes"] + kept + 2 * size * elements + kept + 2 * small, "flops": forward["flops"] + (16 + 2 * act) * elements}


# ---------------------------------------------------------------- the definition in 64 bits
def _exact_kept(x, codes):
    """What a checkpoint of x stands for, from the definition: the smallest power of two s with max|x| <= top * s, then x / s rounded."""
    x = x.double()
    c, top = x.shape[-1], 127.0 if codes == "int8" else 448.0
    out = torch.empty_like(x)
    for b in range(0, c, 32):
        v = x[..., b:b + 32]
        # max = m * 2^k with m in [1/2, 1): max / top <= 2^e holds at e = k - 6 (k - 8) if m / 2^.. is within, else one above
        m, k = torch.frexp(v.abs().amax(dim=-1, keepdim=True))
        lowest = 6 if codes == "int8" else 8
        e = k - lowest - 1
        e = torch.where(torch.ldexp(m, k - e) > top, e + 1, e).clamp(min=-127)
        s = torch.ldexp(torch.ones_like(m), e)
        r = v / s
        if codes == "int8":
            q = torch.round(r)
        else:
            # three bits behind the leading one, and nothing finer than 2^-9
            step = torch.ldexp(torch.ones_like(r), torch.frexp(r)[1].clamp(min=-5) - 4)
            q = torch.round(r / step) * step
        out[..., b:b + 32] = torch.where(v.abs().amax(dim=-1, keepdim=True).isfinite(), q * s, torch.full_like(r, float("nan")))
    return out


def exact(case, seed):
    state = prepare(case, seed)
    kind = case["kind"]
    if kind == "linear_grad":
        codes, scales = state["codes"].double(), state["scales"].double()
        x = torch.empty_like(codes)
        for b in range(scales.shape[-1]):
            x[:, 32 * b:32 * b + 32] = codes[:, 32 * b:32 * b + 32] * 2.0 ** (scales[:, b:b + 1] - 127.0)
        return torch.einsum("ro,ri->oi", state["dy"].double(), x)
    x = state.pop("x")
    if kind == "checkpoint":
        return _exact_kept(x, case["codes"])
    n, groups, c = case["n"], case["groups"], case["c"]
    weight, bias, activation = state["weight"].double(), state["bias"].double(), case["activation"]
    cg = c // groups
    out = {}
    dys = state.pop("dy", None)
    y = torch.empty(x.shape, dtype=torch.float64, device=x.device) if kind != "norm_backward" else None
    dx = torch.empty(x.shape, dtype=torch.float64, device=x.device) if kind != "norm" else None
    dweight, dbias = torch.zeros_like(weight), torch.zeros_like(bias)
    means, rstds = torch.empty((n, groups), dtype=torch.float64, device=x.device), torch.empty((n, groups), dtype=torch.float64, device=x.device)
    step = max(1, n // 32)
    for i in range(0, n, step):                     # a few samples at a time
        xi = x[i:i + step].double()
        if kind == "norm_backward":
            mean, rstd = state["mean"][i:i + step].double(), state["rstd"][i:i + step].double()
        else:
            v = xi.unflatten(-1, (groups, cg))
            mean = v.mean(dim=(1, 2, 4))
            rstd = 1.0 / torch.sqrt(v.var(dim=(1, 2, 4), unbiased=False) + EPS)
            means[i:i + step], rstds[i:i + step] = mean, rstd

        def normal(t):
            return ((t.unflatten(-1, (groups, cg)) - mean[:, None, None, :, None]) * rstd[:, None, None, :, None]).flatten(-2)

        if y is not None:
            z = normal(xi) * weight + bias
            y[i:i + step] = {"none": lambda: z, "relu": lambda: z.clamp(min=0), "silu": lambda: z * torch.sigmoid(z)}[activation]()
        if dx is not None:
            xhat = normal(_exact_kept(xi, case["codes"]) if kind == "norm_train" else xi)
            dz = dys[i:i + step].double()
            z = xhat * weight + bias
            if activation == "relu":
                dz = dz * (z > 0)
            elif activation == "silu":
                s = torch.sigmoid(z)
                dz = dz * (s + z * s * (1 - s))
            dbias += dz.sum(dim=(0, 1, 2))
            dweight += (dz * xhat).sum(dim=(0, 1, 2))
            g = (dz * weight).unflatten(-1, (groups, cg))
            h = xhat.unflatten(-1, (groups, cg))
            t = g - g.mean(dim=(1, 2, 4), keepdim=True) - h * (g * h).mean(dim=(1, 2, 4), keepdim=True)
            dx[i:i + step] = (t * rstd[:, None, None, :, None]).flatten(-2)
    if y is not None:
        out["y"] = y
    if kind == "norm":
        out["mean"], out["rstd"] = means, rstds
    if dx is not None:
        out["dx"], out["dweight"], out["dbias"] = dx, dweight, dbias
    return out
