"""The operators on caller-owned tensors over the whole of their ranges: sums as long as a tensor has samples or positions, values and parameters at
the ends of their types, against the definitions in 64 bits.

Tolerances.  Where the terms of a sum are alike, an fp32 running sum of k of them is off by at most k 2^-25 of it (half a step, at most 2^-24 of
the running sum, which is half of the last one on average).  A thread of a backward pass sums at most 192 terms so, the sums of its block's rows
come in four chains of at most 64 each, those of warps in chains of at most 32; everything longer carries the error of its additions along
(2^-24 in all).  192 + 64 of 2^-25 are 2^-17, FP32 below: that times the sum of the magnitudes."""
import subprocess
import sys
import threading

import pytest
import torch

from paper_1412_2302_b200 import alexnet as A

pytestmark = pytest.mark.gpu

FP32 = 2.0 ** -17
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def ops():
    from paper_1412_2302_b200 import operators
    return operators


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def parameter_gradients_of_alike(ops, shape, groups, src):
    """dbias and dweight for a dy that is one number per channel, statistics of 0 and 1 and values of one sign: nothing cancels, so the running sums
    grow and their roundings with them."""
    n, h, w, c = shape
    dy = torch.linspace(0.05, 0.15, c, device="cuda").expand(shape)
    x = (torch.rand((1, h, w, c), device="cuda", generator=gen(n)) + 0.5).expand(shape)
    mean, rstd = torch.zeros((n, groups), device="cuda"), torch.ones((n, groups), device="cuda")
    kept, value = x, x[0]
    if src != "x":
        kept = ops.checkpoint_encode(x, src)
        value = ops.checkpoint_decode(ops.Checkpoint(kept.codes[0], kept.scales[0]), torch.float32)
    _, dw, db = ops.group_norm_backward(dy, kept, mean, rstd)
    dy64 = dy[0, 0, 0].double()
    want_b, want_w = dy64 * (n * h * w), dy64 * value.double().sum((0, 1)) * n
    assert float(((db.double() - want_b).abs() / want_b).max()) < FP32
    assert float(((dw.double() - want_w).abs() / want_w).max()) < FP32


@pytest.mark.parametrize("src", ["x", "int8"])
@pytest.mark.parametrize("shape,groups", [((16384, 9, 9, 64), 8), ((65536, 9, 9, 32), 8), ((65536, 9, 9, 9), 3), ((400000, 3, 2, 32), 4), ((1000000, 1, 1, 32), 4)])
def test_parameter_gradients_of_many_samples(ops, shape, groups, src):
    parameter_gradients_of_alike(ops, shape, groups, src)


@pytest.mark.parametrize("shape,groups", [((1, 4096, 4096, 16), 4), ((1, 16384, 4096, 8), 2), ((1, 16384, 16384, 1), 1), ((444, 256, 256, 8), 1), ((888, 55, 55, 96), 32)])
def test_gradients_of_many_positions(ops, shape, groups):
    """The same of large samples, and what a group's sums do to dx: with an x of 0 and 1 in turn, dx = rstd (dy - mean of dy - xhat mean of dy xhat)."""
    n, h, w, c = shape
    dy = torch.linspace(0.05, 0.15, c, device="cuda").expand(shape)
    x = torch.tensor([0.0, 1.0], device="cuda").view(1, 1, 2, 1).expand(1, 1, 2, c).repeat(1, 1, w // 2 + 1, 1)[:, :, :w].expand(shape)
    mean, rstd = torch.zeros((n, groups), device="cuda"), torch.ones((n, groups), device="cuda")
    dx, dw, db = ops.group_norm_backward(dy, x, mean, rstd)
    dy64, ones = dy[0, 0, 0].double(), w // 2 / w
    want_b, want_w = dy64 * (n * h * w), dy64 * (n * h * (w // 2))
    assert float(((db.double() - want_b).abs() / want_b).max()) < FP32
    assert float(((dw.double() - want_w).abs() / want_w).max()) < FP32
    m = dy64.view(groups, -1).mean(1).repeat_interleave(c // groups)
    for at in (0, 1):
        want = dy64 - m - at * ones * m
        # two means, and the roundings of their difference from dy
        assert float((dx[:, :, at::2].double() - want).abs().max()) < (2 * FP32 + 2.0 ** -21) * 0.15


@pytest.mark.parametrize("dtype,rest", [("bf16", "normal"), ("bf16", 0.37), ("fp16", 0.0), ("fp32", "normal"), ("fp32", 0.37)])
@pytest.mark.parametrize("shape,groups", [((444, 256, 256, 8), 1), ((888, 55, 55, 96), 32), ((128, 55, 55, 96), 32), ((64, 31, 31, 75), 5), ((600, 64, 64, 3), 1), ((1, 4096, 4096, 8), 1)])
def test_statistics_beside_an_outlier(ops, shape, groups, dtype, rest):
    """The first position (or the last) of every sample lies a thousand spreads away from all others, which are alike or normal: squares of the differences
    from it would drown theirs.  A variance is a sum of squares, all positive: chains of at most 192 (about a mean so far that is
    off by an eighth of the outlier for 32 terms, a fortieth for 32 more and so on, half as much again), at most 85 rows, all of 2^-25, and a root halves it: 187 of 2^-25, where 2^-17 is 256."""
    n, h, w, c = shape
    if n * h * w * c > 1 << 27 and dtype == "fp32" and rest == "normal":
        n = n // 2 if n > 1 else n
    g = gen(c)
    x = torch.empty((n, h, w, c), dtype=TYPES[dtype], device="cuda")
    if rest == "normal":
        x.normal_(generator=g)
    else:
        x.fill_(rest)
    for at in (0, -1):
        was = x[:, at, at].clone()
        x[:, at, at] = -1000.0
        r = ops.group_norm(x, groups, activation="none")
        step = max(1, n // 16)
        for i in range(0, n, step):
            v = x[i:i + step].double().view(-1, h * w, groups, c // groups)
            mean = v.mean((1, 3))
            v -= mean[:, None, :, None]
            rstd = (v.square().mean((1, 3)) + 1e-5).rsqrt()
            # and the rounding of the mean itself: half a step, 2^-24 of it (beside one outlier in 2^24 alike values of 0.37 that alone is 1.9e-4 of their mean deviation)
            assert bool(((r.mean[i:i + step].double() - mean).abs() <= FP32 * v.abs().mean((1, 3)) + 2.0 ** -24 * mean.abs()).all()), (at, i)
            assert float(((r.rstd[i:i + step].double() - rstd).abs() / rstd).max()) < FP32, (at, i)
        x[:, at, at] = was


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_linear_weight_grad_of_pairs_repeats(ops, fmt):
    """Both CTAs of a pair decode their half of every step's tile, and one of them multiplies both: the same bits again while another stream keeps the SMs'
    memory busy, and those of the sums taken 64 rows at a time in 64 bits."""
    g = gen(77)
    rows, n_in, n_out = 1536, 2304, 2048
    k = ops.checkpoint_encode(torch.randn((rows, n_in), device="cuda", generator=g), fmt)
    dy = torch.randn((rows, n_out), device="cuda", generator=g).to(torch.bfloat16)
    want = dy.double().t() @ ops.checkpoint_decode(k, torch.float32).double()
    mag = dy.double().abs().t() @ ops.checkpoint_decode(k, torch.float32).double().abs()
    first = ops.linear_weight_grad(dy, k)
    assert bool(((first.double() - want).abs() <= (rows + 16) * 2.0 ** -24 * mag).all())
    side, a = torch.cuda.Stream(), torch.zeros(1 << 26, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    for i in range(200):
        with torch.cuda.stream(side):
            a.add_(1)
        again = ops.linear_weight_grad(dy, k)
        assert torch.equal(again, first), i


@pytest.mark.parametrize("src", ["x", "int8", "e4m3"])
@pytest.mark.parametrize("shape,groups", [((2, 8, 8, 64), 8), ((2, 8, 8, 33), 3), ((1, 150, 150, 64), 4)])
def test_gradients_of_alike_values_with_a_tiny_eps(ops, shape, groups, src):
    """No variance and an eps of 1e-40: rstd is 1e20 and its square no number of fp32, but dx = rstd (dy w - mean) is."""
    g = gen(7)
    x = torch.full(shape, 3.0, device="cuda")
    w = torch.rand(shape[-1], device="cuda", generator=g) + 0.5
    r = ops.group_norm(x, groups, w, eps=1e-40)
    assert torch.equal(r.mean, torch.full_like(r.mean, 3.0))
    dy = torch.randn(shape, device="cuda", generator=g)
    dx, dw, db = ops.group_norm_backward(dy, x if src == "x" else ops.checkpoint_encode(x, src), r.mean, r.rstd, w)
    n, h, ww, c = shape
    gw = (dy.double() * w.double()).view(n, h * ww, groups, -1)
    want = (r.rstd.double()[:, None, :, None] * (gw - gw.mean((1, 3), keepdim=True))).view(shape)
    mag = (r.rstd.double()[:, None, :, None] * (gw.abs() + gw.abs().mean((1, 3), keepdim=True))).view(shape)
    assert bool(((dx.double() - want).abs() <= FP32 * mag).all())
    assert not bool(dw.any()) and bool(((db.double() - dy.double().sum((0, 1, 2))).abs() <= FP32 * dy.double().abs().sum((0, 1, 2))).all())


@pytest.mark.parametrize("src", ["x", "int8"])
@pytest.mark.parametrize("shape,groups", [((2, 8, 8, 64), 8), ((2, 8, 8, 33), 3), ((1, 150, 150, 64), 4), ((1, 150, 150, 33), 3)])
def test_relu_of_weights_too_small_for_products(ops, shape, groups, src):
    """z = xhat w + b is positive where it is, although rstd w, or its product with x - mean, is no number of fp32 any more: dbias counts the positions."""
    g = gen(19)
    n, h, ww, c = shape
    x = torch.randn(shape, device="cuda", generator=g)
    x[:, 0, 0] = 1e-12
    w = torch.tensor([1e-38, -1e-38, 1e-44, -1e-44, 1e-30, -1e-30, 0.0, -0.0, 1.0, -1.0], device="cuda").repeat(c // 10 + 1)[:c]
    b = torch.tensor([0.0, 0.0, 0.0, 1e-45, -1e-45, 1.0, -1.0], device="cuda").repeat(c // 7 + 1)[:c]
    mean, rstd = torch.zeros((n, groups), device="cuda"), torch.full((n, groups), 1e-3, device="cuda")
    kept = x if src == "x" else ops.checkpoint_encode(x, src)
    value = (x if src == "x" else ops.checkpoint_decode(kept, torch.float32)).double()
    dbias = ops.group_norm_backward(torch.ones_like(x), kept, mean, rstd, w, b, activation="relu")[2]
    assert torch.equal(dbias.double(), (value * 1e-3 * w.double() + b.double() > 0).double().sum((0, 1, 2)))


def test_check_waits_for_every_stream(ops):
    """Work on a stream of the caller's, which does not wait for the default stream, has ended when check() returns."""
    side, done = torch.cuda.Stream(), torch.cuda.Event()
    x = torch.randn((4, 8, 8, 64), device="cuda", generator=gen(1))
    want = ops.group_norm(x, 8).y
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)               # about a tenth of a second
        y = ops.group_norm(x, 8).y
        done.record()
    assert not done.query()
    ops.check()
    assert done.query() and torch.equal(y, want)


def test_autograd_is_not_passed_by_in_silence(ops):
    x, w = torch.randn((2, 4, 4, 64), device="cuda", generator=gen(1)), torch.nn.Parameter(torch.ones(64, device="cuda"))
    b = torch.zeros(64, device="cuda")
    plain = ops.group_norm(x, 8, w.detach(), b)
    assert not plain.y.requires_grad
    for args in ((x, 8, w, b), (x.clone().requires_grad_(), 8, None, b), (x, 8, None, b.clone().requires_grad_())):
        r = ops.group_norm(*args)
        assert torch.equal(r.y, ops.group_norm(args[0].detach(), 8, w.detach(), b).y) and r.y.requires_grad
        with pytest.raises(A.AlexNetError, match="group_norm_backward"):
            r.y.square().sum().backward()
        with torch.no_grad():
            assert not ops.group_norm(*args).y.requires_grad
    out = torch.empty_like(x)
    assert ops.group_norm(x, 8, w, b, out=out).y is out and not out.requires_grad

    class Norm(torch.autograd.Function):        # as a caller puts the two together
        @staticmethod
        def forward(ctx, x, weight, bias):
            r = ops.group_norm(x, 8, weight, bias, activation="silu")
            ctx.save_for_backward(x, r.mean, r.rstd, weight, bias)
            return r.y

        @staticmethod
        def backward(ctx, dy):
            x, mean, rstd, weight, bias = ctx.saved_tensors
            return ops.group_norm_backward(dy.contiguous(), x, mean, rstd, weight, bias, activation="silu")
    leaf = x.clone().requires_grad_()
    Norm.apply(leaf, w, b).sum().backward()
    r = ops.group_norm(x, 8, w.detach(), b, activation="silu")
    dx, dw, _ = ops.group_norm_backward(torch.ones_like(x), x, r.mean, r.rstd, w.detach(), b, activation="silu")
    assert torch.equal(leaf.grad, dx) and torch.equal(w.grad, dw)


def test_one_picture_allocates_its_outputs_alone(ops):
    x = torch.randn((1, 13, 13, 384), device="cuda", generator=gen(1)).to(torch.bfloat16)
    allocated = lambda: torch.cuda.memory_stats()["allocation.all.allocated"]      # noqa: E731
    r = ops.group_norm(x, 32)
    before = allocated()
    r = ops.group_norm(x, 32)
    assert allocated() - before == 3                 # y, mean, rstd
    before = allocated()
    ops.group_norm_backward(x, x, r.mean, r.rstd)
    assert allocated() - before == 3                 # dx, dweight, dbias


def test_empty_sizes(ops):
    """Rows may be none, channels and features may not: an AlexNetError like any wrong argument's."""
    def refused(word, f, *args, **kw):
        with pytest.raises(A.AlexNetError, match=word) as e:
            f(*args, **kw)
        assert e.value.code == A.ERR_ARG
    bf16 = dict(dtype=torch.bfloat16, device="cuda")
    codes = lambda *s: ops.Checkpoint(torch.zeros(s, dtype=torch.int8, device="cuda"), torch.zeros((*s[:-1], (s[-1] + 31) // 32), dtype=torch.uint8, device="cuda"))      # noqa: E731
    for lead in ((2,), (2, 3), (2, 1, 1, 3), (0, 3)):
        refused("features", ops.linear_weight_grad, torch.zeros((*lead, 0), **bf16), codes(*lead, 8))
        refused("features", ops.linear_weight_grad, torch.zeros((*lead, 8), **bf16), codes(*lead, 0))
        refused("channels", ops.checkpoint_encode, torch.zeros((*lead, 0), **bf16))
        refused("channels", ops.checkpoint_decode, codes(*lead, 0))
    refused("channels", ops.checkpoint_encode, torch.zeros((2, 1, 1, 1, 0), **bf16))
    refused("channels", ops.group_norm, torch.zeros((2, 3, 3, 0), **bf16), 1)
    refused("at least 1", ops.checkpoint_encode, torch.zeros((2, 0, 3, 8), **bf16))
    for lead in ((0,), (0, 3), (0, 1, 1, 3)):
        assert bool((ops.linear_weight_grad(torch.zeros((*lead, 8), **bf16), codes(*lead, 40)) == 0).all())
        assert ops.checkpoint_decode(ops.checkpoint_encode(torch.zeros((*lead, 8), **bf16))).shape == (*lead, 8)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("rows,n_in,n_out,width", [(173, 500, 1000, 1008), (64, 64, 64, 72), (300, 1024, 512, 520), (129, 40, 13, 16), (77, 33, 1, 8), (2049, 2080, 2056, 2064), (1000, 4096, 1000, 1024)])
def test_linear_weight_grad_of_wider_rows(ops, fmt, rows, n_in, n_out, width):
    """dy as the first columns of rows that are wider and start on 16-byte boundaries: read in place, NaN behind the columns; those before and behind dw stay as
    they were.  Sums are off by (rows + 16) 2^-24 of their magnitudes at most."""
    g = gen(rows + n_out)
    k = ops.checkpoint_encode(torch.randn((rows, n_in), device="cuda", generator=g), fmt)
    wide = torch.full((rows, width), float("nan"), dtype=torch.bfloat16, device="cuda")
    dy = wide[:, :n_out]
    dy.copy_(torch.randn((rows, n_out), device="cuda", generator=g))
    around = torch.full((n_out * n_in + 64,), 7.0, device="cuda")
    dw = around[32:32 + n_out * n_in].view(n_out, n_in)
    assert ops.linear_weight_grad(dy, k, out=dw) is dw
    value = ops.checkpoint_decode(k, torch.float32).double()
    want, mag = dy.double().t() @ value, dy.double().abs().t() @ value.abs()
    assert bool(((dw.double() - want).abs() <= (rows + 16) * 2.0 ** -24 * mag).all())
    assert bool((around[:32] == 7).all()) and bool((around[-32:] == 7).all())
    assert torch.equal(dw, ops.linear_weight_grad(dy.contiguous(), k))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_linear_weight_grad_at_the_ends_of_the_scales(ops, fmt):
    """Blocks of every exponent that encode writes, from subnormal values to the largest, and gradients that bring the products back: what is read is the
    checkpoint's value rounded to bf16 (exact but for e4m3 codes of values below 2^-126)."""
    rows, n_in, n_out = 96, 64, 24
    g = gen(3)
    x = torch.randn((rows, n_in), device="cuda", generator=g) * torch.exp2(torch.linspace(-130, 100, rows, device="cuda").double())[:, None].float()
    x[::7] *= -1
    k = ops.checkpoint_encode(x, fmt)
    value = ops.checkpoint_decode(k, torch.bfloat16).double()
    dy = torch.zeros((rows, n_out), device="cuda", dtype=torch.bfloat16)
    for o in range(n_out):                               # each output sees four rows, so that no sum mixes sizes
        dy[4 * o:4 * o + 4, o] = torch.randn(4, device="cuda", generator=g).bfloat16() * (2.0 ** (100 if o < 4 else 0))
    dw = ops.linear_weight_grad(dy, k)
    want, mag = dy.double().t() @ value, dy.double().abs().t() @ value.abs()
    assert bool(want.abs().amax(1).gt(0).all())
    assert bool(((dw.double() - want).abs() <= 20 * 2.0 ** -24 * mag + 2.0 ** -149).all())


def test_rows_at_any_alignment(ops):
    """Slices of channels of a wider tensor that start between 16-byte boundaries: statistics against the definition."""
    n, h, w, c, groups = 4, 6, 5, 64, 8
    wide = torch.randn((n, h, w, c + 8), device="cuda", generator=gen(41)).to(torch.bfloat16)
    for off in (1, 3, 5):
        part = wide[..., off:off + c]
        r = ops.group_norm(part, groups)
        v = part.double().reshape(n, h * w, groups, c // groups)
        mean = v.mean((1, 3))
        v = v - mean[:, None, :, None]
        rstd = (v.square().mean((1, 3)) + 1e-5).rsqrt()
        assert bool(((r.mean.double() - mean).abs() <= FP32 * v.abs().mean((1, 3)) + 2.0 ** -24 * mean.abs()).all())
        assert bool(((r.rstd.double() - rstd).abs() <= FP32 * rstd).all())
        y = (v * rstd[:, None, :, None]).view(n, h, w, c)
        assert bool(((r.y.double() - y).abs() <= 2.0 ** -8 * y.abs() + 3 * FP32 * (y.abs() + 1)).all())


def test_more_samples_than_a_grid_of_slices_takes(ops):
    n, c = (1 << 25) + 77, 4
    x = torch.randn((n, c), device="cuda", generator=gen(5)).to(torch.float16)
    r = ops.group_norm(x, 2, activation="none", keep_input="int8")
    dy = torch.randn((n, c), device="cuda", generator=gen(6)).to(torch.float16)
    dx, dw, db = ops.group_norm_backward(dy, x, r.mean, r.rstd)
    for at in (slice(0, 1000), slice(n - 1000, n)):
        some = ops.group_norm(x[at].clone(), 2, keep_input="int8")
        assert torch.equal(r.y[at], some.y) and torch.equal(r.mean[at], some.mean) and torch.equal(r.input.codes[at], some.input.codes)
        assert torch.equal(dx[at], ops.group_norm_backward(dy[at].clone(), x[at].clone(), some.mean, some.rstd)[0])
    assert bool(((db.double() - dy.double().sum(0)).abs() <= FP32 * dy.double().abs().sum(0)).all())


FIRST = r"""
import torch
from paper_1412_2302_b200 import operators as ops
g = torch.Generator(device="cuda").manual_seed(1)
x = torch.randn((2, 40, 40, 33), device="cuda", generator=g)
v = torch.randn((4, 13, 13, 64), device="cuda", generator=g).bfloat16()
dy = torch.randn((200, 72), device="cuda", generator=g).bfloat16()
codes = torch.randint(-127, 128, (200, 160), device="cuda", generator=g, dtype=torch.int8)
scales = torch.randint(100, 140, (200, 5), device="cuda", generator=g, dtype=torch.uint8)
def run():
    a, b = ops.group_norm(x, 3, activation="silu", keep_input="int8"), ops.group_norm(v, 8, activation="relu", keep_output="e4m3")
    return [a.y, *ops.group_norm_backward(x, a.input, a.mean, a.rstd, activation="silu"), b.y, *ops.group_norm_backward(v, v, b.mean, b.rstd, activation="relu"),
            ops.checkpoint_decode(b.output), ops.linear_weight_grad(dy, ops.Checkpoint(codes, scales))]
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    got = run()
for t in got:
    t.fill_(5)
graph.replay()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, run()))
print("same")
"""


def test_the_first_calls_of_a_process_are_captured():
    """Nothing has to have run before: a kernel's code, its shared memory and its plan are found while the stream is being captured."""
    r = subprocess.run([sys.executable, "-c", FIRST], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stdout + r.stderr[-2000:]


def test_refusals_name_what_is_wrong(ops):
    x = torch.zeros((2, 4, 4, 64), device="cuda")
    for word, kw in (("groups = .2, 4, 4, 64, 7., eps = 1e-05", dict(groups=7)), ("eps = 0.0", dict(groups=8, eps=0.0)), ("eps = -1.0", dict(groups=8, eps=-1.0))):
        with pytest.raises(A.AlexNetError, match=word) as e:
            ops.group_norm(x, **kw)
        assert e.value.code == A.ERR_ARG


@pytest.mark.parametrize("value", [2.0 ** 75 * 1.1, -2.0 ** 70])
@pytest.mark.parametrize("shape", [(2, 8, 8, 64), (2, 8, 8, 33), (300, 27, 27, 64), (1, 150, 150, 64)])
def test_alike_values_of_any_size(ops, shape, value):
    """Up to 2^76: no sum or square of what is left over passes fp32, the mean is the value and y the bias."""
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.full(shape, value, device="cuda", dtype=dtype)
        bias = torch.arange(shape[-1], device="cuda", dtype=torch.float32)
        r = ops.group_norm(x, 1, None, bias)
        assert torch.equal(r.mean, x[:, 0, 0, :1].float()) and torch.equal(r.y, bias.to(dtype).expand(shape)) and bool(r.rstd.isfinite().all() and (r.rstd > 0).all())


def test_a_group_with_an_infinity_is_nan(ops):
    for shape in ((2, 8, 8, 64), (2, 8, 8, 33), (2, 150, 150, 64)):
        for at in (0, 5, -1):
            x = torch.randn(shape, device="cuda", generator=gen(2))
            x[1, at, at, 0] = float("-inf")
            r = ops.group_norm(x, 1)
            assert bool(r.mean[1].isnan().all() and r.rstd[1].isnan().all() and r.y[1].isnan().all() and r.y[0].isfinite().all())


@pytest.mark.parametrize("c,groups", [(72, 9), (73, 1)])
def test_tensors_of_more_than_2_to_the_32_values(ops, c, groups):
    """The last sample of a dense tensor of 4.8e9 values against the definition, and its codes against those of the sample alone."""
    n, h, w = 64, 1024, 1024
    g = gen(9)
    x = torch.empty((n, h, w, c), dtype=torch.bfloat16, device="cuda")
    dy = torch.empty_like(x)
    for t in (x, dy):
        t[:-1] = 1.0
        t[-1] = torch.randn((h, w, c), device="cuda", generator=g).to(torch.bfloat16) + 0.5
    r = ops.group_norm(x, groups, activation="silu", keep_input="int8")
    alone = ops.checkpoint_encode(x[-1:], "int8")
    assert torch.equal(r.input.codes[-1:], alone.codes) and torch.equal(r.input.scales[-1:], alone.scales)
    v = x[-1].double().view(h * w, groups, c // groups)
    mean = v.mean((0, 2), keepdim=True)
    rstd = ((v - mean).square().mean((0, 2), keepdim=True) + 1e-5).rsqrt()
    z = ((v - mean) * rstd).view(h, w, c)
    assert bool(((r.y[-1].double() - z * torch.sigmoid(z)).abs() <= 2.0 ** -8 * z.abs() + 3 * FP32 * (z.abs() + 1)).all())
    del v, z
    dx, dw, db = ops.group_norm_backward(dy, r.input, r.mean, r.rstd, activation="silu")
    one = ops.group_norm_backward(dy[-1:], alone, r.mean[-1:], r.rstd[-1:], activation="silu")
    assert bool(((dx[-1:].float() - one[0].float()).abs() <= 2.0 ** -7 * one[0].float().abs() + 2 * FP32).all())
    assert bool(dx[:-1].float().abs().max() < 1e-3 * 316 + 1)              # (no variance: rstd is 316 and dy alike)


def test_threads_call_side_by_side(ops):
    """Four threads with streams of their own, each with its own sizes: plans and messages belong to a thread."""
    def work(i, out):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            g = torch.Generator(device="cuda").manual_seed(i)
            for k in range(30):
                c = 32 * (1 + (i + k) % 5)
                x = torch.randn((2 + i, 9, 9 + k, c), device="cuda", generator=g).to(torch.bfloat16)
                r = ops.group_norm(x, 4, activation="silu", keep_input="int8")
                d = ops.group_norm_backward(x, r.input, r.mean, r.rstd, activation="silu")
                dw = ops.linear_weight_grad(x, r.input)
                out.append((x, r, d, dw))
                try:
                    ops.group_norm(x, 5 + i)
                except A.AlexNetError as e:
                    assert f", {5 + i})" in str(e)
        s.synchronize()
    results = [[] for _ in range(4)]
    threads = [threading.Thread(target=work, args=(i, results[i])) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for out in results:
        assert len(out) == 30
        for x, r, d, dw in out:
            again = ops.group_norm(x, 4, activation="silu", keep_input="int8")
            assert torch.equal(again.y, r.y) and torch.equal(again.input.codes, r.input.codes) and torch.equal(dw, ops.linear_weight_grad(x, r.input))
            assert all(torch.equal(a, b) for a, b in zip(d, ops.group_norm_backward(x, r.input, r.mean, r.rstd, activation="silu")))
