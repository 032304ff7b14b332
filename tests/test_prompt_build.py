"""The prompt and logits operators as built: their launch plan under the sanitizers, and the registers of their kernels
(host only)."""
import os

import pytest

from test_host_logic import _kernel_resources
from test_sanitizers import ROOT, _build_and_run


def test_launch_planner_of_prompts_under_sanitizers(tmp_path):
    out = _build_and_run(tmp_path, "g++", [os.path.join(ROOT, "tests", "sanitize", "prompt_plan_driver.cpp")], ["-std=c++17"])
    assert out.startswith("ok")


@pytest.mark.parametrize("source,occupancy", [
    # two workgroups of four wavefronts a CU with up to 128 channels, one with 256; the tiled kernel of 64 channels fits three
    ("prompt_mfma.hip", {"kernelILi64E": 3, "kernelILi128E": 2, "kernelILi256E": 1}),
    ("prompt_attn.hip", {"f32_kernelILi64E": 2, "f32_kernelILi128E": 2, "f32_kernelILi256E": 1, "merge": 7}),
    ("logits.hip", {"mark": 8, "penalize": 4}),
    ("page_tables.hip", {"page": 4}),
    ("kv_write.hip", {"kv_write": 8}),
])
def test_kernels_use_no_scratch_memory(source, occupancy):
    """The tiled kernel issues its LDS reads ahead of the products that take them, with waits of its own: a register that
    is spilled or copied in between would hold nothing yet.  The others keep their loads in flight in registers."""
    for name, scratch, waves in _kernel_resources(source):
        assert scratch == 0, (name, scratch)
        assert any(k in name for k in occupancy), name
        assert all(waves >= least for k, least in occupancy.items() if k in name), (name, waves)
