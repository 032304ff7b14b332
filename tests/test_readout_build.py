"""The operators on a step's softmaxes as built: their launch plans under the sanitizers, and the registers of their kernels (host only)."""
import os

import pytest

from test_host_logic import _kernel_resources
from test_sanitizers import ROOT, _build_and_run


def test_launch_planners_under_sanitizers(tmp_path):
    out = _build_and_run(tmp_path, "g++", [os.path.join(ROOT, "tests", "sanitize", "readout_plan_driver.cpp")], ["-std=c++17"])
    assert out.startswith("ok")


@pytest.mark.parametrize("source,occupancy", [
    # keys held in registers: two wavefronts a SIMD with up to 128 channels; streamed: one of 256 fp32 channels at least
    ("kv_weights.hip", {"manyILi64E": 2, "manyILi128E": 2, "manyILi256E": 1, "many_f32": 2, "few": 1, "join": 8}),
    ("kv_evict.hip", {"select": 7, "compact": 7}),
    # 71 KB of LDS for the chunks' maxima of 128k fp32 logits: two workgroups of eight wavefronts a CU
    ("logprobs.hip", {"logprobs_kernel": 4, "join": 8}),
])
def test_kernels_use_no_scratch_memory(source, occupancy):
    for name, scratch, waves in _kernel_resources(source):
        assert scratch == 0, (name, scratch)
        assert any(k in name for k in occupancy), name
        assert all(waves >= least for k, least in occupancy.items() if k in name), (name, waves)
