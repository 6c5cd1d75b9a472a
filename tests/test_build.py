"""What the library is compiled with."""
from paper_1412_2302_b200 import build as B


def test_kernels_are_compiled_file_by_file(monkeypatch):
    """The code of a kernel follows from its own file and the flags alone: no -split-compile, whose cuts move with the rest of the file and the
    machine's cores (23 of the 47 kernels of a training step got other registers by it)."""
    commands = []
    monkeypatch.setattr(B.subprocess, "check_call", commands.append)
    for timeline in (False, True):
        B.build(force=True, timeline=timeline)
    compiled = [c for c in commands if "-c" in c]
    assert {c[-1].rsplit("/", 1)[-1] for c in compiled} >= {"alexnet_api.cu", "operators.cu"}
    assert not [a for c in commands for a in c if "split-compile" in a]
    assert all("arch=compute_100a,code=sm_100a" in c and "-O3" in c for c in compiled)
