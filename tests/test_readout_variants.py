"""The GPU tests of `token_logprobs` reach every kernel that its plan can take (host arithmetic: no GPU needed)."""
import os
import subprocess

import pytest

pytest.importorskip("torch")

from test_gpu_logprobs_variants import BATCHES, LONG_LISTS  # noqa: E402
from test_sanitizers import ROOT  # noqa: E402


def plans(tmp_path, cases):
    exe = str(tmp_path / "driver")
    subprocess.check_call(["g++", "-std=c++17", os.path.join(ROOT, "tests", "sanitize", "readout_variants_driver.cpp"), "-o", exe])
    out = subprocess.run([exe] + [str(x) for c in cases for x in c], capture_output=True, text=True, check=True).stdout
    return [tuple(int(x) for x in line.split()) for line in out.splitlines()]


def test_every_kernel_is_reached(tmp_path):
    got = plans(tmp_path, BATCHES)
    kernels = {(threads, stripes, slices > 1) for threads, stripes, slices in got}
    # (a row is cut into no slices of 8192 logits and fewer)
    every = {(256, 4, False), (256, 8, False)} | {(512, s, cut) for s in (8, 16, 32) for cut in (False, True)}
    assert every <= kernels, every - kernels
    assert any(top == 0 and slices > 1 for (_, _, top), (_, _, slices) in zip(BATCHES, got))


def test_the_join_walks_its_lists(tmp_path):
    """It holds 1024 entries at once."""
    for case, (_, _, slices) in zip(LONG_LISTS, plans(tmp_path, LONG_LISTS)):
        assert slices * case[2] > 1024, (case, slices)
