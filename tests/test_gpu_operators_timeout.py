"""A wait inside linear_weight_grad that runs out, in a process of its own: the library reports it for the rest of the process."""
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

CHILD = r"""
import ctypes, sys
import torch
from paper_1412_2302_b200 import alexnet as A
from paper_1412_2302_b200 import operators as ops

rows, n_in, n_out, block = map(int, sys.argv[1:])
g = torch.Generator(device="cuda").manual_seed(rows)
k = ops.checkpoint_encode(torch.randn((rows, n_in), device="cuda", generator=g), "int8")
dy = torch.randn((rows, n_out), device="cuda", generator=g).to(torch.bfloat16)
want = ops.linear_weight_grad(dy, k)
ops.check()
dw = torch.zeros_like(want)
nbytes = ops._linear_workspace(rows, n_in, n_out, n_out, 0, 0, 1)
ws = torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda")
msg = ctypes.create_string_buffer(256)
args = ops._pack_linear(rows, n_in, n_out, dy.data_ptr(), n_out, *ops._kept(k), dw.data_ptr(), ws.data_ptr(), nbytes)
L = A.load_library()
assert L.alexnet_operators_debug_expire_wait(args, 2, None, msg, 256) == A.ERR_ARG and b"block" in msg.value
rc = L.alexnet_operators_debug_expire_wait(args, block, torch.cuda.current_stream().cuda_stream, msg, 256)
assert rc == A.OK, msg.value
try:
    ops.check()
except A.AlexNetError as e:
    assert e.code == A.ERR_DEVICE_TIMEOUT
else:
    raise SystemExit("check() did not tell of the wait that ran out")
gone = dw.isnan()
assert bool(gone.any()) and torch.equal(dw[~gone], want[~gone]), int(gone.sum())
assert torch.equal(ops.linear_weight_grad(dy, k), want)              # the GPU is as good as before
x = torch.randn((2, 4, 4, 64), device="cuda")
assert bool(ops.group_norm(x, 8).y.isfinite().all())
print("parts", int(gone.sum()), "of", gone.numel())
"""


@pytest.mark.parametrize("rows,n_in,n_out,block", [(300, 96, 72, 0), (640, 128, 2048, 1), (2048, 4096, 4096, 0), (2048, 4096, 4096, 1)])
def test_a_wait_that_runs_out_is_reported(rows, n_in, n_out, block):
    """Single CTAs, and both CTAs of a pair: the one that issues the products and the one whose decoded half they miss."""
    r = subprocess.run([sys.executable, "-c", CHILD, str(rows), str(n_in), str(n_out), str(block)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "parts" in r.stdout, r.stdout + r.stderr[-2000:]
