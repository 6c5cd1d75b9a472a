"""Refusals of the operators on caller-owned tensors, without a GPU: the binding's own checks and the library's, which come before any
CUDA call.  And the argument blocks that the binding packs."""
import ctypes
import os
import re
import subprocess
import time

import pytest
import torch

from paper_1412_2302_b200 import alexnet as A
from paper_1412_2302_b200 import build as B
from paper_1412_2302_b200 import operators as ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    B.build()
    return A.load_library()


def call(lib, name, block):
    msg = ctypes.create_string_buffer(256)
    return getattr(lib, "alexnet_" + name)(block, None, msg, 256), msg.value.decode()


P = 1 << 20           # stands for a pointer: nothing is launched, nothing follows it
VIEW = lambda h, w, c, p=P: (p, h * w * c, w * c, c)      # noqa: E731
KEPT = (P, P, 1, 0)
NONE = (0, 0, 0, 0)


def test_argument_blocks_have_the_headers_sizes(tmp_path):
    src = tmp_path / "sizes.c"
    src.write_text('#include "%s"\n#include <stdio.h>\nint main(void) { printf("%%zu %%zu %%zu %%zu %%zu\\n", sizeof(alexnet_group_norm_t), '
                   'sizeof(alexnet_checkpoint_args_t), sizeof(alexnet_group_norm_forward_t), sizeof(alexnet_group_norm_backward_t), '
                   'sizeof(alexnet_linear_weight_grad_t)); return 0; }\n' % os.path.join(ROOT, "include", "alexnet.h"))
    exe = str(tmp_path / "sizes")
    subprocess.check_call(["gcc", "-o", exe, str(src)])
    sizes = [int(v) for v in subprocess.check_output([exe], text=True).split()]
    assert sizes == [p.__self__.size for p in (ops._pack_shape, ops._pack_checkpoint, ops._pack_forward, ops._pack_backward, ops._pack_linear)]


def test_enums_match_the_header():
    src = open(os.path.join(ROOT, "include", "alexnet.h")).read()
    value = lambda name: int(re.search(r"\bALEXNET_%s = (\d+)" % name, src).group(1))      # noqa: E731
    assert [value("DTYPE_" + n) for n in ("BF16", "F16", "F32")] == [ops.DTYPES[t] for t in (torch.bfloat16, torch.float16, torch.float32)]
    assert {n: value("ACT_" + n.upper()) for n in ops.ACTIVATIONS} == ops.ACTIVATIONS
    assert {n: value("CODES_" + n.upper()) for n in ops.FORMATS} == ops.FORMATS


def shape(n=2, h=3, w=4, c=64, groups=8, dtype=0, act=0, eps=1e-5):
    return (n, h, w, c, groups, dtype, act, eps, 0)


BAD_SHAPES = [(dict(n=-1), "n must"), (dict(h=0), "at least 1"), (dict(w=0), "at least 1"), (dict(c=0, groups=1), "channels"), (dict(c=(1 << 20) + 8), "channels"),
              (dict(groups=0), "groups"), (dict(groups=7), "groups"), (dict(groups=-8), "groups"), (dict(dtype=3), "dtype"), (dict(dtype=-1), "dtype"),
              (dict(act=3), "activation"), (dict(act=-1), "activation"), (dict(eps=0.0), "eps"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"),
              (dict(h=1 << 16, w=1 << 16), "2^30"), (dict(n=1 << 40), "too large"), (dict(n=1 << 31, c=1 << 20, groups=1), "too large")]


@pytest.mark.parametrize("bad,word", BAD_SHAPES)
def test_group_norm_refuses_shapes(lib, bad, word):
    s = shape(**bad)
    for backward in (0, 1):
        assert lib.alexnet_group_norm_workspace_bytes(ops._pack_shape(*s), backward) == 0
    v = VIEW(3, 4, 64)
    rc, msg = call(lib, "group_norm_forward", ops._pack_forward(*s, *v, *v[:1], *v[1:], P, P, P, P, *NONE, *NONE, P, 1 << 40))
    assert rc == A.ERR_ARG and word in msg, msg
    rc, msg = call(lib, "group_norm_backward", ops._pack_backward(*s, *v, *v, *v, *NONE, P, P, P, P, P, P, P, 1 << 40))
    assert rc == A.ERR_ARG and word in msg, msg


def forward_block(s=shape(), x=VIEW(3, 4, 64), y=VIEW(3, 4, 64, 2 * P), mean=P, rstd=P, kx=NONE, ky=NONE, ws=P, nbytes=1 << 40):
    return ops._pack_forward(*s, *x, *y, P, P, mean, rstd, *kx, *ky, ws, nbytes)


# a sample that no block can keep, so that the call needs its workspace
LARGE = dict(s=shape(h=400, w=400), x=VIEW(400, 400, 64), y=VIEW(400, 400, 64, 2 * P))
LARGE_BACK = dict(s=shape(h=400, w=400), dy=VIEW(400, 400, 64), x=VIEW(400, 400, 64, 2 * P), dx=VIEW(400, 400, 64, 3 * P))
FORWARD = [(dict(x=VIEW(3, 4, 64, 0)), "NULL"), (dict(y=VIEW(3, 4, 64, 0)), "NULL"), (dict(mean=0), "NULL"), (dict(rstd=0), "NULL"), (dict(LARGE, ws=0), "workspace"),
           (dict(x=VIEW(3, 4, 64, P + 1)), "aligned"), (dict(s=shape(dtype=2), x=VIEW(3, 4, 64, P + 2)), "aligned"), (dict(LARGE, ws=P + 8), "workspace"), (dict(LARGE, nbytes=16), "workspace"),
           (dict(y=VIEW(3, 4, 64)), "share"), (dict(x=(P, -768, 256, 64)), "stride"), (dict(x=(P, 768, 1 << 50, 64)), "stride"),
           (dict(y=(2 * P, 768, 256, 63)), "overlap"), (dict(y=(2 * P, 768, 255, 64)), "overlap"), (dict(y=(2 * P, 0, 256, 64)), "overlap"),
           (dict(y=(2 * P, 64, 256, 64)), "overlap"),
           (dict(kx=(P, P, 0, 0)), "format"), (dict(ky=(P, P, 3, 0)), "format"), (dict(kx=(P, 0, 1, 0)), "NULL"), (dict(ky=(0, P, 2, 0)), "NULL")]


@pytest.mark.parametrize("bad,word", FORWARD)
def test_group_norm_forward_refuses(lib, bad, word):
    rc, msg = call(lib, "group_norm_forward", forward_block(**bad))
    assert rc == A.ERR_ARG and word in msg, msg


def backward_block(s=shape(), dy=VIEW(3, 4, 64), x=VIEW(3, 4, 64, 2 * P), dx=VIEW(3, 4, 64, 3 * P), kept=NONE, mean=P, rstd=P, ws=P, nbytes=1 << 40):
    return ops._pack_backward(*s, *dy, *x, *dx, *kept, mean, rstd, P, P, P, P, ws, nbytes)


BACKWARD = [(dict(dy=VIEW(3, 4, 64, 0)), "NULL"), (dict(x=VIEW(3, 4, 64, 0)), "NULL"), (dict(dx=VIEW(3, 4, 64, 0)), "NULL"), (dict(mean=0), "NULL"), (dict(rstd=0), "NULL"),
            (dict(kept=KEPT), "twice"), (dict(x=NONE, kept=(P, P, 9, 0)), "format"), (dict(x=NONE, kept=(P, 0, 1, 0)), "NULL"), (dict(dx=VIEW(3, 4, 64)), "share"),
            (dict(dx=VIEW(3, 4, 64, 2 * P)), "share"), (dict(dx=(3 * P, 768, 0, 64)), "overlap"), (dict(LARGE_BACK, ws=P + 4), "workspace"), (dict(LARGE_BACK, nbytes=0), "workspace"),
            (dict(LARGE_BACK, ws=0), "workspace")]


@pytest.mark.parametrize("bad,word", BACKWARD)
def test_group_norm_backward_refuses(lib, bad, word):
    rc, msg = call(lib, "group_norm_backward", backward_block(**bad))
    assert rc == A.ERR_ARG and word in msg, msg


CHECKPOINT = [(dict(h=0), "at least 1"), (dict(c=0), "channels"), (dict(dtype=7), "dtype"), (dict(x=(0, 1, 1, 1)), "NULL"), (dict(kept=(0, P, 1, 0)), "NULL"), (dict(kept=(P, P, 4, 0)), "format"),
              (dict(x=(P + 1, 768, 256, 64)), "aligned"), (dict(x=(P, 768, 256, -64)), "stride")]


@pytest.mark.parametrize("bad,word", CHECKPOINT)
def test_checkpoint_refuses(lib, bad, word):
    a = dict(dict(n=2, h=3, w=4, c=64, dtype=0, x=VIEW(3, 4, 64), kept=KEPT), **bad)
    block = ops._pack_checkpoint(a["n"], a["h"], a["w"], a["c"], a["dtype"], *a["x"], *a["kept"])
    for name in ("checkpoint_encode", "checkpoint_decode"):
        rc, msg = call(lib, name, block)
        assert rc == A.ERR_ARG and word in msg and msg.startswith(name), msg
    rc, msg = call(lib, "checkpoint_decode", ops._pack_checkpoint(2, 3, 4, 64, 0, P, 768, 0, 64, *KEPT))
    assert rc == A.ERR_ARG and "overlap" in msg


LINEAR = [(dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"), (dict(n_in=0), "features"), (dict(n_out=0), "features"), (dict(n_in=1 << 21), "features"), (dict(dy=0), "NULL"),
          (dict(dy=P + 1), "aligned"), (dict(stride=-8), "stride"), (dict(kept=(P, 0, 1, 0)), "NULL"), (dict(kept=(0, P, 1, 0)), "NULL"), (dict(kept=(P, P, 0, 0)), "format"), (dict(dw=0), "dw"),
          (dict(dw=P + 2), "dw"), (dict(rows=4096, ws=0), "workspace"), (dict(rows=4096, ws=P + 8), "workspace"), (dict(stride=65, nbytes=0), "workspace")]


@pytest.mark.parametrize("bad,word", LINEAR)
def test_linear_weight_grad_refuses(lib, bad, word):
    a = dict(dict(rows=64, n_in=64, n_out=64, dy=P, stride=64, kept=KEPT, dw=P, ws=P, nbytes=1 << 40), **bad)
    rc, msg = call(lib, "linear_weight_grad", ops._pack_linear(a["rows"], a["n_in"], a["n_out"], a["dy"], a["stride"], *a["kept"], a["dw"], a["ws"], a["nbytes"]))
    assert rc == A.ERR_ARG and word in msg, msg
    if word in ("rows", "features", "format", "stride"):
        assert lib.alexnet_linear_weight_grad_workspace_bytes(ops._pack_linear(a["rows"], a["n_in"], a["n_out"], a["dy"], a["stride"], *a["kept"], 0, 0, 0)) == 0


def test_small_calls_need_no_workspace(lib):
    """256 bytes say so; the larger ones name what they need."""
    for backward in (0, 1):
        assert lib.alexnet_group_norm_workspace_bytes(ops._pack_shape(*shape(n=1, h=7, w=7, c=384, groups=32)), backward) == 256
        assert lib.alexnet_group_norm_workspace_bytes(ops._pack_shape(*shape(h=400, w=400)), backward) > 256
    small, large = (ops._pack_linear(rows, 64, 64, P, 64, *KEPT, 0, 0, 0) for rows in (64, 4096))
    assert lib.alexnet_linear_weight_grad_workspace_bytes(small) == 256 and lib.alexnet_linear_weight_grad_workspace_bytes(large) > 4 * 64 * 64 * 4


def test_null_blocks_and_no_samples(lib):
    for name in ("checkpoint_encode", "checkpoint_decode", "group_norm_forward", "group_norm_backward", "linear_weight_grad"):
        rc, msg = call(lib, name, None)
        assert rc == A.ERR_ARG and "NULL" in msg
    # no samples: nothing to read or write, so no pointer is needed and nothing is launched
    s = shape(n=0)
    assert lib.alexnet_group_norm_workspace_bytes(ops._pack_shape(*s), 0) > 0
    assert call(lib, "group_norm_forward", ops._pack_forward(*s, *NONE, *NONE, 0, 0, 0, 0, *NONE, *NONE, 0, 0))[0] == A.OK
    assert call(lib, "checkpoint_encode", ops._pack_checkpoint(0, 3, 4, 64, 0, *NONE, 0, 0, 1, 0))[0] == A.OK


def test_binding_refuses(lib):
    def refused(word, f, *args, **kw):
        with pytest.raises(A.AlexNetError, match=word) as e:
            f(*args, **kw)
        assert e.value.code == A.ERR_ARG
    x = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16)
    codes, scales = torch.zeros(2, 64, dtype=torch.int8), torch.zeros(2, 2, dtype=torch.uint8)
    refused("no CPU fallback", ops.group_norm, x, 8)
    refused("no CPU fallback", ops.checkpoint_encode, x)
    refused("no CPU fallback", ops.checkpoint_decode, ops.Checkpoint(codes, scales))
    refused("no CPU fallback", ops.group_norm_backward, x, x, torch.zeros(2, 8), torch.zeros(2, 8))
    refused("no CPU fallback", ops.linear_weight_grad, torch.zeros(2, 8, dtype=torch.bfloat16), ops.Checkpoint(codes, scales))
    refused("int8", ops.Checkpoint, codes.float(), scales)
    refused("uint8", ops.Checkpoint, codes, scales.int())
    refused("rounded up", ops.Checkpoint, codes, scales[:, :1])
    refused("dense", ops.Checkpoint, torch.zeros(64, 2, dtype=torch.int8).t(), scales)
    refused("Checkpoint", ops.linear_weight_grad, torch.zeros(2, 8, dtype=torch.bfloat16), codes)
    refused("bfloat16", ops.linear_weight_grad, torch.zeros(2, 8), ops.Checkpoint(codes, scales))
    refused("rows", ops.linear_weight_grad, torch.zeros(3, 8, dtype=torch.bfloat16), ops.Checkpoint(codes, scales))


def test_numbers_that_no_argument_block_holds(lib):
    """Refused like any wrong argument, not by an error of the packing; a view may have as many rows as it likes."""
    for bad in (dict(h=1 << 31), dict(groups=1 << 40), dict(n=1 << 64), dict(eps=1e300), dict(groups=8.0)):
        for backward in (0, 1):
            with pytest.raises(A.AlexNetError) as e:
                ops._norm_workspace(shape(**bad), backward)
            assert e.value.code == A.ERR_ARG
    with pytest.raises(A.AlexNetError) as e:
        ops._linear_workspace(64, 1 << 32, 64, 64, 0, 0, 1)
    assert e.value.code == A.ERR_ARG
    with pytest.raises(A.AlexNetError) as e:
        ops._run(lib.alexnet_checkpoint_encode, 0, ops._pack_checkpoint, 1, 1, 1 << 31, 1, 0, P, 0, 0, 0, *KEPT)
    assert e.value.code == A.ERR_ARG


def test_tensors_without_channels_are_refused():
    for shape in ((2, 1, 1, 2, 0), (0, 1, 1, 2, 0)):
        with pytest.raises(A.AlexNetError, match="no channels") as e:
            ops._rows_any(torch.zeros(shape), "x")
        assert e.value.code == A.ERR_ARG


def test_a_result_without_a_gradient_says_so():
    y = torch.ones(3)
    z = ops._without_gradient(y)
    assert z is y and z.requires_grad and not z.is_leaf
    with pytest.raises(A.AlexNetError, match="group_norm_backward"):
        (2 * z).sum().backward()
    with torch.no_grad():
        z += 1                                  # its values are anyone's, as before
    assert torch.equal(z.detach(), torch.full((3,), 2.0))


def test_plans_are_found_once_per_size(lib):
    """How a launch walks a few large samples takes 15 to 60 us to find, several times a call; a call that repeats its sizes does not search again.  The
    best of many calls, each refused for its workspace and so all host: some 2 us, where the searches alone took 120."""
    h = w = 1024
    s = shape(n=1, h=h, w=w, c=64, groups=1, act=2)
    v = lambda p: VIEW(h, w, 64, p)      # noqa: E731
    calls = [lambda: lib.alexnet_group_norm_workspace_bytes(ops._pack_shape(*s), 0), lambda: lib.alexnet_group_norm_workspace_bytes(ops._pack_shape(*s), 1),
             lambda: call(lib, "group_norm_forward", ops._pack_forward(*s, *v(P), *v(2 * P), P, P, P, P, *NONE, *NONE, 0, 0)),
             lambda: call(lib, "group_norm_backward", ops._pack_backward(*s, *v(P), *v(2 * P), *v(3 * P), *NONE, P, P, P, P, P, P, 0, 0))]
    for f in calls:
        best = 1.0
        for _ in range(200):
            t = time.perf_counter()
            f()
            best = min(best, time.perf_counter() - t)
        assert best < 30e-6, best


def test_linear_plans_are_found_once_per_size(lib):
    """The same for the tiles of a linear layer's gradient (11 us at 16384 x 256 x 256); alignment is looked at in each call."""
    block = lambda p, stride, q: ops._pack_linear(16384, 256, 256, p, stride, q, P, 1, 0, 0, 0, 0)      # noqa: E731
    size = lib.alexnet_linear_weight_grad_workspace_bytes
    best = 1.0
    for _ in range(200):
        t = time.perf_counter()
        size(block(P, 256, P))
        best = min(best, time.perf_counter() - t)
    assert best < 5e-6, best
    plain, copied = size(block(P, 256, P)), 16384 * 256
    assert size(block(P + 2, 256, P)) == size(block(P, 257, P)) == plain + 2 * copied
    assert size(block(P, 256, P + 8)) == plain + copied and size(block(P + 2, 256, P + 8)) == plain + 3 * copied


def test_vectors_need_less_workspace(lib):
    """The queries that know a call's tensors: one picture of 13 x 13 x 384 and a minibatch of 27 x 27 x 256 are kept by blocks where they are read in vectors,
    and need none; single channels do, and no call needs more than its sizes' query says."""
    forward, backward = lib.alexnet_group_norm_forward_workspace_bytes, lib.alexnet_group_norm_backward_workspace_bytes
    for n, h, w, c, groups in ((1, 13, 13, 384, 32), (128, 27, 27, 256, 32)):
        s, v = shape(n=n, h=h, w=w, c=c, groups=groups), lambda p: VIEW(h, w, c, p)      # noqa: E731
        most = [lib.alexnet_group_norm_workspace_bytes(ops._pack_shape(*s), b) for b in (0, 1)]
        f = lambda x, y, kx=NONE: forward(ops._pack_forward(*s, *x, *y, 0, 0, 0, 0, *kx, *NONE, 0, 0))      # noqa: E731
        b = lambda dy, x, dx, kept=NONE: backward(ops._pack_backward(*s, *dy, *x, *dx, *kept, 0, 0, 0, 0, 0, 0, 0, 0))      # noqa: E731
        assert f(v(P), v(P)) == f(v(0), v(0), (P, P, 1, 0)) == 256
        assert f(v(P + 2), v(P)) == f(v(P), v(P + 8)) == f(v(P), v(P), (P + 4, P, 1, 0)) == most[0] > 256
        assert (b(v(P), v(P), v(P)) == 256) == (n == 1) and b(v(P), v(P), v(P)) <= most[1]
        assert 256 < b(v(P), NONE, v(P), KEPT) <= most[1] and 256 < b(v(P), v(P), v(P + 8)) <= most[1]
    for bad in (dict(groups=7), dict(eps=0.0), dict(n=-1)):
        s, v = shape(**bad), VIEW(3, 4, 64)
        assert forward(ops._pack_forward(*s, *v, *v, 0, 0, 0, 0, *NONE, *NONE, 0, 0)) == 0
        assert backward(ops._pack_backward(*s, *v, *v, *v, *NONE, 0, 0, 0, 0, 0, 0, 0, 0)) == 0
    assert forward(None) == backward(None) == 0
