"""The operators on caller-owned tensors (paper_1412_2302_b200.operators) against their definitions in 64 bits.

Tolerances.  An output is rounded once to its type: half a step, finfo.eps / 2 of the value (below the smallest normal number, half of a
subnormal step).  What is in front of that is fp32: a thread sums at most 192 terms one after another, a block's rows are added in chains of at
most 64 (k alike terms are off by k 2^-25 of their sum: half a step, at most 2^-24 of the running sum, which is half the last one on average), and what is
longer carries the errors of its additions along, so a sum is off by at most 2^-17 of the sum of the magnitudes, a mean of deviations by 2^-17 of their
mean magnitude and a root of a mean square by 2^-17 relative (half of 2^-17 from the root, the rest from the 2^-24s around it).  `FP32`
below is that 2^-17; it multiplies the magnitudes that an expression adds up, not its value.  Codes, exponents and decoded values are whole
numbers of steps by definition and must be equal."""
import itertools

import numpy as np
import pytest
import torch

from paper_1412_2302_b200 import alexnet as A

pytestmark = pytest.mark.gpu

FP32 = 2.0 ** -17
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-5


@pytest.fixture(scope="module")
def ops():
    from paper_1412_2302_b200 import operators
    return operators


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def tensor(g, shape, dtype, pad=0, scale=1.0, shift=0.0, fill=None):
    """a random tensor; pad > 0: a view of a grid with that many more rows and columns, everything else of it being `fill`"""
    n, h, w, c = shape
    v = (torch.randn(shape, device="cuda", generator=g) * (torch.rand(c, device="cuda", generator=g) + 0.5) + torch.randn(c, device="cuda", generator=g)) * scale + shift
    if not pad:
        return v.to(dtype)
    grid = torch.full((n, h + pad, w + pad, c), float("nan") if fill is None else fill, dtype=dtype, device="cuda")
    grid[:, :h, :w] = v.to(dtype)
    return grid[:, :h, :w]


def close(got, want, magnitude, what=""):
    """|got - want| within half a step of the output type and FP32 of `magnitude`; NaN where and only where it is wanted"""
    got64, want = got.double(), want.expand_as(got)
    fi = torch.finfo(got.dtype)
    assert torch.equal(torch.isnan(got64), torch.isnan(want)), what
    # half a step beyond the type's largest number its rounding is an infinity (an fp16 gradient: rstd is 316 where a group has no variance)
    over = want.abs() >= fi.max * (1 + fi.eps / 4)
    want = torch.where(over, torch.copysign(torch.full_like(want, float("inf")), want), want)
    lim = fi.eps / 2 * want.abs() * (1 + 2.0 ** -7) + fi.smallest_normal * fi.eps / 2 + FP32 * magnitude
    bad = ((got64 - want).abs() > lim) & ~over | over & (got64 != want)
    assert not bool(bad.any()), (what, int(bad.sum()), float(((got64 - want).abs() / lim)[bad].max()))


# ---------------------------------------------------------------- definitions in 64 bits
def power(e):
    """2^e exactly, for whole numbers e (pow may be off in the last bit, which decides ties)"""
    return ((e.long() + 1023) << 52).view(torch.float64)


def ref_codes(x, fmt):
    """(codes as numbers, exponent bytes, values) of a checkpoint, from the definition"""
    x = x.double()
    c, top = x.shape[-1], 127.0 if fmt == "int8" else 448.0
    codes, values, exps = torch.empty_like(x), torch.empty_like(x), []
    for b in range(0, c, 32):
        v = x[..., b:b + 32]
        amax = v.abs().amax(-1, keepdim=True)
        finite = amax.isfinite()
        e = torch.full_like(amax, -127.0)
        want = torch.where(finite, amax, torch.zeros_like(amax))
        for k in range(-127, 128):                      # the smallest power of two that is enough
            e = torch.where(want > top * 2.0 ** k, torch.full_like(e, k + 1.0), e)
        r = torch.where(finite, v, torch.zeros_like(v)) / power(e)
        if fmt == "int8":
            q = torch.round(r)
        else:
            lead = torch.floor(torch.log2(r.abs().clamp(min=2.0 ** -30))).clamp(min=-6.0)
            lead = torch.where(power(lead + 1) <= r.abs(), lead + 1, lead)
            lead = torch.where((power(lead) > r.abs()) & (lead > -6), lead - 1, lead)
            step = power(lead - 3)
            q = torch.round(r / step) * step
        codes[..., b:b + 32] = q
        values[..., b:b + 32] = torch.where(finite, q * power(e), torch.full_like(q, float("nan")))
        exps.append(torch.where(finite, e + 127, torch.full_like(e, 255.0)))
    return codes, torch.cat(exps, -1), values


def per_channel(stat, c):
    return stat.repeat_interleave(c // stat.shape[1], 1)[:, None, None, :]


def group_mean(t, groups):
    n, h, w, c = t.shape
    return t.reshape(n, h * w, groups, c // groups).mean((1, 3))


def ref_stats(x, groups):
    x = x.double()
    c = x.shape[-1]
    mean = group_mean(x, groups)
    var = group_mean((x - per_channel(mean, c)) ** 2, groups)
    return mean, (var + EPS).rsqrt()


def ref_act(z, act):
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    return z, torch.ones_like(z)


def ref_forward(x, groups, w, b, act, mean=None, rstd=None):
    """y, mean, rstd and the magnitude that FP32 refers to for y"""
    c = x.shape[-1]
    if mean is None:
        mean, rstd = ref_stats(x, groups)
    w = torch.ones(c, dtype=torch.float64, device=x.device) if w is None else w.double()
    b = torch.zeros(c, dtype=torch.float64, device=x.device) if b is None else b.double()
    M, R = per_channel(mean, c), per_channel(rstd, c)
    xh = (x.double() - M) * R
    z = xh * w + b
    # z: the mean is off by the mean deviation (below one rstd) and by its own rounding, xhat by rstd's error
    mag = (xh.abs() + 1 + 2.0 ** -7 * M.abs() * R) * w.abs() + b.abs()
    return ref_act(z, act)[0], mean, rstd, 1.1 * mag          # |silu'| < 1.1


def ref_backward(dy, x, mean, rstd, w, b, act):
    n, h, ww, c = x.shape
    groups = mean.shape[1]
    w = torch.ones(c, dtype=torch.float64, device=x.device) if w is None else w.double()
    b = torch.zeros(c, dtype=torch.float64, device=x.device) if b is None else b.double()
    M, R = per_channel(mean.double(), c), per_channel(rstd.double(), c)
    xh = (x.double() - M) * R
    z = xh * w + b
    dz = dy.double() * ref_act(z, act)[1]
    g = dz * w
    c1, c2 = group_mean(g, groups), group_mean(g * xh, groups)
    dx = R * (g - per_channel(c1, c) - xh * per_channel(c2, c))
    # errors: of z (through act'', at most 1/2 for silu) on top of those of the sums
    zm = (xh.abs() + 2.0 ** -7 * M.abs() * R) * w.abs() + b.abs() if act == "silu" else torch.zeros_like(z)
    gm = (dz.abs() + dy.double().abs() * zm) * w.abs()
    xm = xh.abs() + 2.0 ** -7 * M.abs() * R
    mag = R * (gm + per_channel(group_mean(gm, groups), c) + 2 * xm * per_channel(group_mean(gm * (1 + xm), groups), c))
    zmag = dz.abs() + dy.double().abs() * zm
    return (dx, (dz * xh).sum((0, 1, 2)), dz.sum((0, 1, 2))), (mag, (zmag * (1 + xm)).sum((0, 1, 2)), zmag.sum((0, 1, 2)))


# ---------------------------------------------------------------- checkpoints
CKPT_SHAPES = [(1, 1, 1, 1), (1, 1, 1, 32), (2, 3, 5, 33), (1, 7, 9, 40), (3, 13, 13, 96), (2, 5, 5, 100), (4, 1, 1, 8), (1, 2, 3, 2056), (2, 27, 29, 48), (600, 1, 1, 24), (1, 64, 65, 7)]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape", CKPT_SHAPES)
def test_checkpoint_codes_are_the_definitions(ops, shape, dtype, fmt):
    g = gen(sum(shape))
    for pad in (0, 2):
        x = tensor(g, shape, TYPES[dtype], pad)
        k = ops.checkpoint_encode(x, fmt)
        codes, exps, values = ref_codes(x, fmt)
        assert torch.equal(k.scales.double(), exps)
        assert torch.equal(k.codes.double(), codes)
        for out_type in TYPES.values():
            assert torch.equal(ops.checkpoint_decode(k, out_type).double(), values.to(out_type).double())
        grid = torch.full((shape[0], shape[1] + pad, shape[2] + pad, shape[3]), 7.0, dtype=TYPES[dtype], device="cuda")
        view = grid[:, :shape[1], :shape[2]]
        assert ops.checkpoint_decode(k, TYPES[dtype], out=view) is view
        assert torch.equal(view.double(), values.to(TYPES[dtype]).double())
        if pad:      # positions outside the view are left as they were
            assert bool((grid[:, shape[1]:] == 7).all()) and bool((grid[:, :, shape[2]:] == 7).all())


@pytest.mark.parametrize("c", [32, 37])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_checkpoint_values_at_the_borders(ops, fmt, c):
    """Largest magnitudes on either side of a power of two and of the largest code, ties between codes, subnormals, the largest numbers
    and blocks that are zero, infinite or NaN."""
    top = 127.0 if fmt == "int8" else 448.0
    one = torch.finfo(torch.float32).eps
    rows = []
    for s in (1.0, 2.0 ** -100, 2.0 ** 100):
        for m in (top, top * (1 + one), top * (1 - one / 2), top * (1 + 2 * one), 2 * top, 1.0, 2.0, 2.0 * (1 - one / 2)):
            row = torch.linspace(-1, 1, c, dtype=torch.float64) * m * s
            row[3] = m * s
            rows.append(row)
        ties = (torch.arange(c, dtype=torch.float64) - 10 + 0.5) * s          # x.5 with a largest magnitude that makes the step one
        ties[0] = -top * s
        rows.append(ties)
    rows += [torch.zeros(c), torch.full((c,), 1e-45), torch.full((c,), 2.0 ** -127), torch.full((c,), -2.0 ** -126), torch.linspace(0, 1, c) * 2.0 ** -120,
             torch.full((c,), torch.finfo(torch.float32).max), torch.linspace(-1, 1, c) * torch.finfo(torch.float32).max]
    for bad in (float("inf"), float("-inf"), float("nan")):
        for at in (0, 31, c - 1):
            row = torch.linspace(-3, 3, c)
            row[at] = bad
            rows.append(row)
    x = torch.stack([r.to(torch.float32) for r in rows]).cuda()
    codes, exps, values = ref_codes(x, fmt)
    k = ops.checkpoint_encode(x, fmt)
    assert torch.equal(k.scales.double(), exps) and torch.equal(k.codes.double(), codes)
    got = ops.checkpoint_decode(k, torch.float32).double()
    # rounded to fp32: the code of its largest number is 64, which stands for 64 * 2^122 = 2^128, an infinity there
    assert torch.equal(values.isnan().any(-1), ~x.isfinite().all(-1))
    values = values.to(torch.float32).double()
    assert torch.equal(got.isnan(), values.isnan()) and torch.equal(got.nan_to_num(), values.nan_to_num())


def test_checkpoint_every_code_is_decoded(ops):
    for fmt, dt in (("int8", torch.int8), ("e4m3", torch.float8_e4m3fn)):
        for c in (256, 255):                                     # vectors and single values
            codes = torch.arange(256, dtype=torch.uint8, device="cuda")[:c].repeat(256, 1).view(dt)
            scales = torch.arange(256, dtype=torch.uint8, device="cuda")[:, None].repeat(1, 8).contiguous()
            got = ops.checkpoint_decode(ops.Checkpoint(codes, scales), torch.float32).double()
            want = codes.double() * power(scales[:, :1].long() - 127)
            want[255] = float("nan")
            want = want.to(torch.float32).double()              # beyond fp32 only with exponents that encode never writes
            assert torch.equal(got.isnan(), want.isnan())
            assert torch.equal(got.nan_to_num(), want.nan_to_num())


# ---------------------------------------------------------------- group norm, forward
# (shape, groups): one position, one channel, one group and as many as channels, groups that straddle vectors, rows longer than a block,
# few and many samples (more than blocks that keep them fit the device), slices of
# several blocks
NORM_SHAPES = [((1, 1, 1, 1), 1), ((1, 1, 1, 64), 8), ((3, 1, 1, 4096), 32), ((2, 3, 5, 12), 4), ((2, 13, 13, 96), 32), ((1, 13, 13, 384), 32), ((2, 27, 27, 40), 5), ((5, 9, 11, 100), 20),
               ((2, 7, 5, 37), 1), ((3, 6, 1, 48), 48), ((1, 1, 50, 2560), 10), ((2, 2, 2, 2064), 3), ((1, 57, 55, 8), 1), ((300, 2, 2, 16), 4), ((7, 1, 1, 6), 3), ((2, 33, 31, 256), 32),
               ((2100, 3, 2, 32), 4), ((700, 9, 9, 64), 8), ((1500, 2, 3, 20), 5), ((1, 96, 90, 64), 32), ((1, 130, 127, 24), 2), ((2, 128, 128, 128), 32)]
ACTS = ["none", "relu", "silu"]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape,groups", NORM_SHAPES)
def test_group_norm_forward(ops, shape, groups, dtype):
    g = gen(groups + sum(shape))
    c = shape[-1]
    for i, act in enumerate(ACTS):
        pad = (0, 2, 0)[i]
        x = tensor(g, shape, TYPES[dtype], pad)
        w = None if i == 0 else torch.randn(c, device="cuda", generator=g)
        b = None if i == 0 else torch.randn(c, device="cuda", generator=g)
        grid = torch.full((shape[0], shape[1] + 1, shape[2] + 1, c), 7.0, dtype=TYPES[dtype], device="cuda")
        out = grid[:, :shape[1], :shape[2]] if pad else None
        r = ops.group_norm(x, groups, w, b, eps=EPS, activation=act, out=out)
        y, mean, rstd, mag = ref_forward(x, groups, w, b, act)
        spread = group_mean((x.double() - per_channel(mean, c)).abs(), groups)
        close(r.mean, mean, spread, "mean")
        close(r.rstd, rstd, rstd, "rstd")
        close(r.y, y, mag, "y")
        if pad:
            assert r.y is out and bool((grid[:, shape[1]:] == 7).all()) and bool((grid[:, :, shape[2]:] == 7).all())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape,groups", [((2, 5, 7, 64), 8), ((1, 9, 9, 36), 6), ((3, 40, 40, 96), 32)])
def test_group_norm_keeps_checkpoints(ops, shape, groups, dtype):
    """The checkpoints written on the way are those of x and of y as it is stored, and the results do not change."""
    g = gen(5)
    x = tensor(g, shape, TYPES[dtype], 1)
    w, b = (torch.randn(shape[-1], device="cuda", generator=g) for _ in range(2))
    plain = ops.group_norm(x, groups, w, b, activation="silu")
    for kx, ky in (("int8", None), (None, "e4m3"), ("e4m3", "int8"), ("int8", "int8")):
        r = ops.group_norm(x, groups, w, b, activation="silu", keep_input=kx, keep_output=ky)
        assert torch.equal(r.y, plain.y) and torch.equal(r.mean, plain.mean) and torch.equal(r.rstd, plain.rstd)
        for k, src, fmt in ((r.input, x, kx), (r.output, r.y, ky)):
            assert (k is None) == (fmt is None)
            if k is not None:
                e = ops.checkpoint_encode(src, fmt)
                assert k.format == fmt and torch.equal(k.codes.view(torch.uint8), e.codes.view(torch.uint8)) and torch.equal(k.scales, e.scales)


@pytest.mark.parametrize("shape,groups", [((2, 20, 20, 64), 4), ((2, 20, 20, 33), 3), ((1, 150, 150, 64), 4)])
def test_group_norm_far_from_zero(ops, shape, groups):
    """A mean of 4000 spreads, in fp32 and 16 bits, and a first position (or any other) that lies far from all others: E[x^2] - mean^2 in
    fp32 would lose the variance."""
    g = gen(8)
    for dtype, shift in (("fp32", 4096.0), ("fp16", 512.0), ("bf16", 0.0)):
        for outlier in (None, 0, -1):
            x = tensor(g, shape, TYPES[dtype], scale=1.0, shift=shift)
            if outlier is not None:
                x[:, outlier, outlier] = -20000.0
            r = ops.group_norm(x, groups, activation="none", eps=EPS)
            y, mean, rstd, mag = ref_forward(x, groups, None, None, "none")
            close(r.mean, mean, group_mean((x.double() - per_channel(mean, shape[-1])).abs(), groups), "mean")
            close(r.rstd, rstd, rstd, "rstd")
            close(r.y, y, mag, "y")


@pytest.mark.parametrize("c,groups", [(64, 8), (36, 6)])
def test_group_norm_bad_values_stay_in_their_group(ops, c, groups):
    g = gen(9)
    x = tensor(g, (3, 6, 6, c), torch.float32)
    w, b = (torch.randn(c, device="cuda", generator=g) for _ in range(2))
    clean = ops.group_norm(x, groups, w, b, activation="relu")
    dy = tensor(g, (3, 6, 6, c), torch.float32)
    gclean = ops.group_norm_backward(dy, x, clean.mean, clean.rstd, w, b, activation="relu")
    for bad in (float("nan"), float("inf")):
        xb = x.clone()
        xb[1, 2, 3, 0] = bad
        r = ops.group_norm(xb, groups, w, b, activation="relu")
        cg = c // groups
        other = torch.ones_like(x, dtype=torch.bool)
        other[1, :, :, :cg] = False
        assert torch.equal(r.y[other], clean.y[other]) and bool(r.y[1, :, :, :cg].isnan().all()) and bool(r.rstd[1, 0].isnan())
        dx, dw, db = ops.group_norm_backward(dy, xb, r.mean, r.rstd, w, b, activation="relu")
        assert torch.equal(dx[other], gclean[0][other]) and bool(dx[1, :, :, :cg].isnan().all())
        assert torch.equal(dw[cg:], gclean[1][cg:]) and torch.equal(db[cg:], gclean[2][cg:]) and bool(dw[:cg].isnan().all())
    constant = torch.full((2, 4, 4, c), 3.0, device="cuda")                 # no variance: y is act(bias)
    r = ops.group_norm(constant, groups, w, b, activation="none")
    assert torch.equal(r.y, b.expand_as(r.y)) and torch.equal(r.mean, torch.full_like(r.mean, 3.0))


# ---------------------------------------------------------------- group norm, backward
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape,groups", NORM_SHAPES)
def test_group_norm_backward(ops, shape, groups, dtype):
    g = gen(3 * groups + sum(shape))
    c = shape[-1]
    for (i, act), src in itertools.product(enumerate(ACTS), ("x", "int8", "e4m3")):
        pad = (0, 0, 2)[i]
        x = tensor(g, shape, TYPES[dtype], pad)
        dy = tensor(g, shape, TYPES[dtype], 3 if i == 1 else 0)
        w = None if i == 0 else torch.randn(c, device="cuda", generator=g)
        b = None if i == 0 else torch.randn(c, device="cuda", generator=g)
        mean, rstd = (t.float() for t in ref_stats(x, groups))
        kept = x if src == "x" else ops.checkpoint_encode(x, src)
        value = x if src == "x" else ref_codes(x, src)[2]
        grid = torch.full((shape[0], shape[1] + 1, shape[2] + 1, c), 7.0, dtype=TYPES[dtype], device="cuda")
        out = grid[:, :shape[1], :shape[2]] if pad else None
        got = ops.group_norm_backward(dy, kept, mean, rstd, w, b, activation=act, out=out)
        want, mag = ref_backward(dy, value, mean, rstd, w, b, act)
        for name, t, v, m in zip(("dx", "dweight", "dbias"), got, want, mag):
            close(t, v, m, (name, act, src))
        if pad:
            assert got[0] is out and bool((grid[:, shape[1]:] == 7).all()) and bool((grid[:, :, shape[2]:] == 7).all())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape,groups", [((3, 6, 6, 64), 8), ((3, 6, 6, 36), 6), ((1, 150, 150, 64), 4), ((1, 150, 150, 33), 3)])
def test_group_norm_backward_of_weights_of_zero(ops, shape, groups, dtype):
    """z is the bias for every x: ReLU passes the gradient on to weight and bias where that is positive, and to x nowhere."""
    g = gen(21 + sum(shape))
    c = shape[-1]
    x, dy = tensor(g, shape, TYPES[dtype]), tensor(g, shape, TYPES[dtype])
    w = torch.randn(c, device="cuda", generator=g)
    w[::2] = 0
    w[:c // groups] = 0                                 # all of a group
    w[1] = -0.0
    b = torch.tensor([0.5, 0.5, -0.5, 0.0, -0.5], device="cuda").repeat(c // 5 + 1)[:c]
    for act, src in itertools.product(ACTS, ("x", "int8", "e4m3")):
        mean, rstd = (t.float() for t in ref_stats(x, groups))
        kept = x if src == "x" else ops.checkpoint_encode(x, src)
        value = x if src == "x" else ref_codes(x, src)[2]
        got = ops.group_norm_backward(dy, kept, mean, rstd, w, b, activation=act)
        want, mag = ref_backward(dy, value, mean, rstd, w, b, act)
        for name, t, v, m in zip(("dx", "dweight", "dbias"), got, want, mag):
            close(t, v, m, (name, act, src))
        assert not bool(got[0][..., :c // groups].any())


def test_reference_gradient_is_the_forward_passes(ops):
    """The formula that the gradients above are held against, against central differences of the definition in 64 bits."""
    g = torch.Generator().manual_seed(4)
    x, dy = (torch.randn((2, 3, 2, 6), dtype=torch.float64, generator=g) for _ in range(2))
    w, b = (torch.randn(6, dtype=torch.float64, generator=g) for _ in range(2))
    for act in ACTS:
        mean, rstd = ref_stats(x, 3)
        grads = ref_backward(dy, x, mean, rstd, w, b, act)[0]
        loss = lambda x, w, b: float((ref_forward(x, 3, w, b, act)[0] * dy).sum())          # noqa: E731
        for k, (t, gr) in enumerate(zip((x, w, b), grads)):
            for j in range(t.numel()):
                h = 1e-5
                d = torch.zeros(t.numel(), dtype=torch.float64)
                d[j] = h
                args = [[x, w, b], [x, w, b]]
                args[0][k], args[1][k] = t + d.view_as(t), t - d.view_as(t)
                # third derivatives of a few units: the difference is off by h^2 of them, the losses by 1e-15 / h
                assert abs((loss(*args[0]) - loss(*args[1])) / (2 * h) - float(gr.reshape(-1)[j])) < 1e-6, (act, k, j)


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("shape,groups", [((2, 5, 4, 32), 4), ((2, 5, 4, 27), 3)])
def test_group_norm_backward_against_differences_of_the_forward(ops, shape, groups, act):
    """Along random directions, the kernels' own forward pass in fp32: the loss is linear in y, so rounding y (2^-24 each, random) costs
    2^-24 |y dy| summed in quadrature over h; h = 2^-6 leaves truncation of h^2 / 6 of the third derivative."""
    g = gen(11)
    x, dy = tensor(g, shape, torch.float32), torch.randn(shape, device="cuda", generator=g)
    c = shape[-1]
    w, b = (torch.randn(c, device="cuda", generator=g) for _ in range(2))
    r = ops.group_norm(x, groups, w, b, activation=act)
    grads = ops.group_norm_backward(dy, x, r.mean, r.rstd, w, b, activation=act)
    h = 2.0 ** -6
    for k in range(3):
        args = [x, w, b]
        v = torch.randn(args[k].shape, device="cuda", generator=g)
        v = v / v.norm()
        loss = []
        for s in (1, -1, 2, -2):
            a = list(args)
            a[k] = args[k] + s * h * v
            loss.append(float((ops.group_norm(a[0], groups, a[1], a[2], activation=act).y.double() * dy.double()).sum()))
        diff = (8 * (loss[0] - loss[1]) - (loss[2] - loss[3])) / (12 * h)       # fourth order: h^4 = 6e-8 of the fifth derivative
        want = float((grads[k].double() * v.double()).sum())
        noise = 2.0 ** -22 * float((r.y.double().abs() * dy.double().abs()).norm()) / h
        assert abs(diff - want) < 20 * noise + 1e-4 * float(grads[k].double().norm()), (k, diff, want)


# ---------------------------------------------------------------- linear weight gradient
LINEAR = [(1, 32, 8), (1, 1, 1), (2, 33, 9), (64, 64, 64), (65, 128, 256), (63, 96, 40), (128, 4096, 72), (173, 500, 1000), (200, 136, 130), (1000, 257, 31), (77, 32, 1000), (4100, 160, 264),
          (300, 1024, 512), (12321, 96, 48), (129, 2080, 2056), (30000, 32, 8)]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("rows,n_in,n_out", LINEAR)
def test_linear_weight_grad(ops, rows, n_in, n_out, fmt):
    """Products of bf16 and decoded values are exact in fp32; a sum of `rows` of them is off by at most (rows + 16) 2^-24 of the sum of
    their magnitudes in any order (16: the joins of a split)."""
    g = gen(rows + n_in + n_out)
    x = torch.relu(torch.randn((rows, n_in), device="cuda", generator=g) + 0.3)
    k = ops.checkpoint_encode(x, fmt)
    value = ref_codes(x, fmt)[2]
    for pad in (0, 8, 3):
        wide = torch.full((rows, n_out + pad), float("nan"), dtype=torch.bfloat16, device="cuda")
        wide[:, :n_out] = torch.randn((rows, n_out), device="cuda", generator=g).to(torch.bfloat16)
        dy = wide[:, :n_out]
        if pad == 8 and n_out % 8 == 0 and rows > 1:
            dy = dy.contiguous()[:, :]                  # the same values, aligned rows
        dw = ops.linear_weight_grad(dy, k)
        want = dy.double().t() @ value
        mag = dy.double().abs().t() @ value.abs()
        bad = (dw.double() - want).abs() > (rows + 16) * 2.0 ** -24 * mag + 2.0 ** -24 * want.abs()
        assert not bool(bad.any()), (pad, int(bad.sum()), float(((dw.double() - want).abs() / mag.clamp(min=1e-30)).max()))
    out = torch.full((n_out, n_in), float("nan"), device="cuda")
    assert ops.linear_weight_grad(dy, k, out=out) is out and torch.equal(out, dw)


@pytest.mark.parametrize("rows,n_in,n_out", [(8192, 2560, 2080), (8192 + 37, 1024, 4096), (16384, 4096, 2000)])
def test_linear_weight_grad_keeps_its_precision_over_many_rows(ops, rows, n_in, n_out):
    """Many tiles, so that none is split.  The tensor cores cut off: 2.2e-10 of the result a row, 4.5e-7 over the 2048 rows that one of their sums
    takes up.  Those sums are added with rounding, at most eight of them, 2^-24 each and random: 1.7e-7 together.  2^-20 is 9.5e-7."""
    g = gen(rows)
    x = torch.randn((rows, n_in), device="cuda", generator=g)
    k = ops.checkpoint_encode(x, "e4m3")
    dy = torch.randn((rows, n_out), device="cuda", generator=g).to(torch.bfloat16)
    dw = ops.linear_weight_grad(dy, k)
    assert torch.equal(dw, ops.linear_weight_grad(dy, k))
    want = dy.double().t() @ ref_codes(x, "e4m3")[2]
    assert float((dw.double() - want).norm() / want.norm()) < 2.0 ** -20
    mag = (rows + 16) * 2.0 ** -24 * (dy.double().abs().t() @ ref_codes(x, "e4m3")[2].abs())
    assert not bool(((dw.double() - want).abs() > mag).any())


def test_linear_weight_grad_of_positions_and_of_nothing(ops):
    g = gen(2)
    x = torch.randn((3, 5, 7, 64), device="cuda", generator=g)
    dy = torch.randn((3, 5, 7, 24), device="cuda", generator=g).to(torch.bfloat16)
    k = ops.checkpoint_encode(x, "int8")
    flat = ops.Checkpoint(k.codes.view(105, 64), k.scales.view(105, 2))
    assert torch.equal(ops.linear_weight_grad(dy, k), ops.linear_weight_grad(dy.view(105, 24), flat))
    none = ops.Checkpoint(torch.empty((0, 64), dtype=torch.int8, device="cuda"), torch.empty((0, 2), dtype=torch.uint8, device="cuda"))
    dw = ops.linear_weight_grad(torch.empty((0, 24), dtype=torch.bfloat16, device="cuda"), none, out=torch.full((24, 64), 5.0, device="cuda"))
    assert bool((dw == 0).all())
    # a block of the checkpoint that stands for NaN, an infinite gradient
    bad = ops.Checkpoint(k.codes.view(105, 64).clone(), k.scales.view(105, 2).clone())
    bad.scales[50, 1] = 255
    got = ops.linear_weight_grad(dy.view(105, 24), bad)
    want = ops.linear_weight_grad(dy.view(105, 24), flat)
    assert bool(got[:, 32:].isnan().all()) and torch.equal(got[:, :32], want[:, :32])


# ---------------------------------------------------------------- together, and around the calls
def test_a_block_of_two_linear_layers_trained_from_checkpoints(ops):
    """h = x0 w1^T, y = silu(norm(h)), o = y w2^T over positions, with x0, h and y kept in 8 bits: gradients of the weights against the
    same block in 64 bits on the values that the checkpoints stand for, and the bias gradient of the layer below by its own entry point."""
    g = gen(21)
    n, s, c0, c1, c2, groups = 2, 9, 64, 96, 40, 32
    x0 = torch.randn((n, s, s, c0), device="cuda", generator=g).to(torch.bfloat16)
    w1 = (torch.randn((c1, c0), device="cuda", generator=g) / 8).to(torch.bfloat16)
    w2 = (torch.randn((c2, c1), device="cuda", generator=g) / 8).to(torch.bfloat16)
    gamma, beta = torch.rand(c1, device="cuda", generator=g) + 0.5, torch.randn(c1, device="cuda", generator=g) * 0.1
    do = torch.randn((n, s, s, c2), device="cuda", generator=g).to(torch.bfloat16)
    k0 = ops.checkpoint_encode(x0, "e4m3")
    h = torch.matmul(x0, w1.t())
    r = ops.group_norm(h, groups, gamma, beta, activation="silu", keep_input="int8", keep_output="int8")
    dw2 = ops.linear_weight_grad(do, r.output)
    dy = torch.matmul(do, w2)
    dh, dgamma, dbeta = ops.group_norm_backward(dy, r.input, r.mean, r.rstd, gamma, beta, activation="silu")
    dw1 = ops.linear_weight_grad(dh, k0)
    db1 = torch.empty(c1, device="cuda")
    A.bias_grad_noalloc(dh.view(-1, c1), db1, stream=torch.cuda.current_stream())
    y64, _, _, ymag = ref_forward(h, groups, gamma, beta, "silu")
    close(r.y, y64, ymag, "y")
    yk, x0k = ref_codes(r.y, "int8")[2].view(-1, c1), ref_codes(x0, "e4m3")[2].view(-1, c0)
    (dh64, dg64, db64), (hm, gm, bm) = ref_backward(dy, ref_codes(h, "int8")[2], r.mean, r.rstd, gamma, beta, "silu")
    close(dh, dh64, hm, "dh"); close(dgamma, dg64, gm, "dgamma"); close(dbeta, db64, bm, "dbeta")      # noqa: E702
    d2, d1 = do.double().view(-1, c2), dh.double().view(-1, c1)
    close(dw2, d2.t() @ yk, d2.abs().t() @ yk.abs(), "dw2")
    close(dw1, d1.t() @ x0k, d1.abs().t() @ x0k.abs(), "dw1")
    close(db1, d1.sum(0), d1.abs().sum(0), "db1")


def all_outputs(ops, x, dy, groups, w, b, dyl, kl):
    r = ops.group_norm(x, groups, w, b, activation="silu", keep_input="int8", keep_output="e4m3")
    back = ops.group_norm_backward(dy, r.input, r.mean, r.rstd, w, b, activation="silu")
    same = ops.group_norm_backward(dy, x, r.mean, r.rstd, w, b, activation="relu")
    k = ops.checkpoint_encode(x, "e4m3")
    return [r.y, r.mean, r.rstd, r.input.codes, r.input.scales, r.output.codes.view(torch.uint8), r.output.scales, *back, *same, k.codes.view(torch.uint8), k.scales,
            ops.checkpoint_decode(k, x.dtype), ops.linear_weight_grad(dyl, kl)]


def inputs(seed, shape=(4, 13, 13, 96), rows=300, n_in=160, n_out=72):
    g = gen(seed)
    from paper_1412_2302_b200 import operators as ops
    c = shape[-1]
    return [tensor(g, shape, torch.bfloat16), tensor(g, shape, torch.bfloat16), 32 if c % 32 == 0 else 3, torch.randn(c, device="cuda", generator=g), torch.randn(c, device="cuda", generator=g),
            torch.randn((rows, n_out), device="cuda", generator=g).to(torch.bfloat16), ops.checkpoint_encode(torch.randn((rows, n_in), device="cuda", generator=g), "int8")]


@pytest.mark.parametrize("shape", [(4, 13, 13, 96), (2, 60, 60, 33), (1, 128, 128, 64)])
def test_results_repeat_on_streams_and_in_graphs(ops, shape):
    """The same bits again, on a stream of the caller's, in two streams at once, captured and replayed with new inputs in place, and twice in
    one graph on branches that run side by side."""
    args, others = inputs(31, shape), inputs(32, shape)
    want, want2 = all_outputs(ops, *args), all_outputs(ops, *others)
    torch.cuda.synchronize()
    same = lambda got, ref: all(torch.equal(a, b) for a, b in zip(got, ref))          # noqa: E731
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    got = {1: [], 2: []}
    for _ in range(20):
        for s, a, k in ((s1, args, 1), (s2, others, 2)):
            with torch.cuda.stream(s):
                got[k].append(all_outputs(ops, *a))
    torch.cuda.synchronize()
    assert all(same(t, want) for t in got[1]) and all(same(t, want2) for t in got[2])
    r = ops.group_norm(args[0], args[2], args[3], args[4], activation="silu", stream=s1)
    s1.synchronize()
    assert torch.equal(r.y, want[0])

    live = inputs(31, shape)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s1):
        fork = torch.cuda.Event()
        fork.record(s1)
        first = all_outputs(ops, *live)
        s2.wait_event(fork)
        with torch.cuda.stream(s2):
            second = all_outputs(ops, *others)
            done = torch.cuda.Event()
            done.record(s2)
        s1.wait_event(done)
    for _ in range(3):
        for t in first + second:
            t.view(torch.uint8).fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert same(first, want) and same(second, want2)
    for dst, src in zip(live, others):
        if torch.is_tensor(dst):
            dst.copy_(src)
    live[-1].codes.copy_(others[-1].codes)
    live[-1].scales.copy_(others[-1].scales)
    graph.replay()
    torch.cuda.synchronize()
    assert same(first, want2) and same(second, want2)
    eager = all_outputs(ops, *args)                    # eager calls beside the captured ones
    torch.cuda.synchronize()
    assert same(eager, want)


def test_orders_and_strides(ops):
    """Positions in another order than their memory, broadcast inputs, samples taken every other one."""
    g = gen(41)
    n, h, w, c, groups = 4, 6, 5, 64, 8
    base = tensor(g, (n, h, w, c), torch.bfloat16)
    want = ops.group_norm(base, groups)
    turned = base.permute(2, 1, 0, 3).contiguous().permute(2, 1, 0, 3)          # memory order w, h, n
    out = torch.empty((h, n, w, c), dtype=torch.bfloat16, device="cuda").permute(1, 0, 2, 3)
    r = ops.group_norm(turned, groups, out=out)
    assert torch.equal(r.y, want.y) and torch.equal(r.mean, want.mean) and r.y is out
    double = torch.zeros((2 * n, h, 2 * w, c), dtype=torch.bfloat16, device="cuda")
    double[::2, :, 1::2] = base
    assert torch.equal(ops.group_norm(double[::2, :, 1::2], groups).y, want.y)
    dy = tensor(g, (1, 1, 1, c), torch.bfloat16).expand(n, h, w, c)
    a = ops.group_norm_backward(dy, base, want.mean, want.rstd)
    b = ops.group_norm_backward(dy.contiguous(), base, want.mean, want.rstd)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    # a slice of channels of a wider tensor: adjacent channels, rows at any alignment
    wide = tensor(g, (n, h, w, c + 8), torch.bfloat16)
    for off in (0, 8, 1, 3):
        part = wide[..., off:off + c]
        assert torch.equal(ops.group_norm(part, groups).mean, ops.group_norm(part.contiguous(), groups).mean) or off in (1, 3)
        x64, mean, rstd, mag = ref_forward(part, groups, None, None, "none")
        close(ops.group_norm(part, groups).y, x64, mag, off)
    # fewer dimensions
    assert torch.equal(ops.group_norm(base.view(n, h * w, c), groups).y.view(n, h, w, c), want.y)
    flat = base.reshape(n * h * w, c)
    assert torch.equal(ops.group_norm(flat, groups).y, ops.group_norm(flat.view(-1, 1, 1, c), groups).y.view(-1, c))


def test_no_samples(ops):
    x = torch.empty((0, 4, 4, 64), device="cuda")
    r = ops.group_norm(x, 8, keep_input="int8")
    assert r.y.shape == x.shape and r.mean.shape == (0, 8) and r.input.shape == x.shape
    dx, dw, db = ops.group_norm_backward(x, r.input, r.mean, r.rstd)
    assert dx.shape == x.shape and bool((dw == 0).all()) and bool((db == 0).all())
    assert ops.checkpoint_decode(ops.checkpoint_encode(x)).shape == x.shape


def test_offsets_beyond_32_bits(ops):
    """Samples that lie more than 2^32 elements apart in one buffer, and a dense tensor of more than 2^32 values."""
    g = gen(51)
    n, c = 3, 64
    buf = torch.empty(2 ** 32 + 2 ** 31 + 4096, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (n, 5, 5, c), (2 ** 31 + 64 * 8, 5 * c, c, 1))
    dense = tensor(g, (n, 5, 5, c), torch.bfloat16)
    x.copy_(dense)
    want = ops.group_norm(dense, 8, activation="silu", keep_input="int8")
    r = ops.group_norm(x, 8, activation="silu", keep_input="int8")
    assert torch.equal(r.y, want.y) and torch.equal(r.input.codes, want.input.codes)
    dy = tensor(g, (n, 5, 5, c), torch.bfloat16)
    out = torch.as_strided(buf, (n, 5, 5, c), (2 ** 31 + 64 * 8, 5 * c, c, 1), 2048)
    a, b = ops.group_norm_backward(dy, x, r.mean, r.rstd, out=out), ops.group_norm_backward(dy, dense, r.mean, r.rstd)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    del x, out
    rows = (2 ** 32 + 2 ** 20) // 4096
    big = buf[:rows * 4096].view(rows, 4096)
    big[:] = 1.0
    big[-1] = torch.linspace(-1, 1, 4096, device="cuda").to(torch.bfloat16)
    k = ops.checkpoint_encode(big, "int8")
    tail = ops.checkpoint_encode(big[-1:].contiguous(), "int8")
    assert torch.equal(k.codes[-1:], tail.codes) and torch.equal(k.scales[-1:], tail.scales) and bool((k.codes[-2] == 64).all())
    back = ops.checkpoint_decode(k, torch.bfloat16)
    assert torch.equal(back[-1], ops.checkpoint_decode(tail, torch.bfloat16)[0]) and bool((back[-2] == 1).all())


def test_numbers_of_other_types(ops):
    x = torch.randn((2, 3, 3, 16), device="cuda")
    want = ops.group_norm(x, 4, eps=1.0)
    assert torch.equal(ops.group_norm(x, np.int64(4), eps=1).y, want.y)
    many = torch.zeros((1, 1, 1, 4), device="cuda").expand(1, 1 << 31, 1, 4)
    for call in (lambda: ops.group_norm(x, 4.0), lambda: ops.group_norm(x, "4"), lambda: ops.group_norm(x, 4, eps="tiny"), lambda: ops.group_norm(x, 1 << 40),
                 lambda: ops.group_norm(x, 4, eps=1e300), lambda: ops.group_norm(many, 4),
                 lambda: ops.group_norm_backward(many, many, torch.ones((1, 4), device="cuda"), torch.ones((1, 4), device="cuda"))):
        with pytest.raises(A.AlexNetError) as e:
            call()
        assert e.value.code == A.ERR_ARG


def test_refusals_on_the_gpu(ops):
    x = torch.zeros((2, 4, 4, 64), device="cuda")

    def refused(word, f, *args, **kw):
        with pytest.raises(A.AlexNetError, match=word) as e:
            f(*args, **kw)
        assert e.value.code == A.ERR_ARG
    refused("groups", ops.group_norm, x, 7)
    refused("dtype", ops.group_norm, x.double(), 8)
    refused("activation", ops.group_norm, x, 8, activation="gelu")
    refused("dtype", ops.checkpoint_decode, ops.checkpoint_encode(x), torch.int8)
    refused("eps", ops.group_norm, x, 8, eps=0.0)
    refused("adjacent", ops.group_norm, x.permute(0, 3, 1, 2), 4)
    refused("dimensions", ops.group_norm, x[0, 0, 0], 8)
    refused("vector", ops.group_norm, x, 8, torch.ones(63, device="cuda"))
    refused("vector", ops.group_norm, x, 8, torch.ones(64, device="cuda", dtype=torch.bfloat16))
    refused("one device", ops.group_norm, x, 8, torch.ones(64))
    refused("out must be", ops.group_norm, x, 8, out=torch.empty_like(x, dtype=torch.bfloat16))
    refused("share", ops.group_norm, x, 8, out=x)
    refused("overlap", ops.group_norm, x, 8, out=torch.empty((1, 4, 4, 64), device="cuda").expand(2, 4, 4, 64))
    refused("format", ops.group_norm, x, 8, keep_input="int4")
    r = ops.group_norm(x, 8)
    refused("differ in shape", ops.group_norm_backward, x[:1], x, r.mean, r.rstd)
    refused("float32", ops.group_norm_backward, x.bfloat16(), x, r.mean, r.rstd)
    refused("mean and rstd", ops.group_norm_backward, x, x, r.mean[:1], r.rstd)
    refused("another shape or format", ops.checkpoint_encode, x, "int8", out=ops.checkpoint_encode(x, "e4m3"))
    refused("differ in their rows", ops.linear_weight_grad, torch.zeros((3, 8), dtype=torch.bfloat16, device="cuda"), ops.checkpoint_encode(x[0, 0]))
