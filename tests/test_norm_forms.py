"""The norm's kernels that are built are those that a call takes, and the calls of the GPU tests take all of them."""
import re
import shutil
import subprocess

import pytest

import norm_forms as nf


def widths():
    return range(8, 32769, 8)


def test_forward_and_backward_calls_of_the_tests_take_every_kernel():
    forward = {nf.forward_kernel(rows, cols, residual, y, fmt) for cols in widths() for rows in (1, 10000) for residual in (False, True) for y in (False, True) for fmt in (0, 1, 2)}
    assert {nf.forward_kernel(*c) for c in nf.FORWARD} == forward and len(forward) == 43
    backward = {nf.backward_kernel(rows, cols, residual) for cols in widths() for rows in (1, 10000) for residual in (False, True)}
    assert {nf.backward_kernel(*c) for c in nf.BACKWARD} == backward and len(backward) == 9


@pytest.mark.skipif(shutil.which("nm") is None, reason="no nm")
def test_nothing_is_built_that_no_call_takes():
    from paper_2602_01410_b200 import build
    names = subprocess.run(["nm", "-C", build.build()], capture_output=True, text=True, check=True).stdout
    # the host's names of the kernels: rmsnorm_kernel<V, threads, stages, residual, format>
    built = {(int(a), int(b), int(c), d == "true", int(e)) for a, b, c, d, e in re.findall(r"rmsnorm_kernel<(\d), (\d+), (\d), (true|false), (\d)>", names)}
    assert built == {nf.forward_kernel(*c) for c in nf.FORWARD}
    built = {(int(a), int(b), int(c), d == "true") for a, b, c, d in re.findall(r"rmsnorm_bwd_kernel<(\d), (\d+), (\d), (true|false)>", names)}
    assert built == {nf.backward_kernel(*c) for c in nf.BACKWARD}
