"""CPU: the kernels around the linear layers keep nothing in scratch memory and spill no register (from the compiler's report, which the build writes down)."""
import json
import os

import pytest

from paper_2509_25149_amd import build

KERNELS = ("rmsnorm_forward_kernel", "rmsnorm_backward_kernel", "checkpoint_save_kernel", "checkpoint_load_kernel", "activation_backward_kernel", "colsum_kernel")


@pytest.mark.parametrize("kernel", KERNELS)
def test_streaming_kernels_stay_in_registers(kernel):
    if not os.path.exists(build.RESOURCES):
        pytest.skip("libnvfp4_hip.resources.json is written by build(); run it first")
    reports = {name: r for name, r in json.load(open(build.RESOURCES)).items() if kernel in name}
    assert reports
    for name, r in reports.items():
        assert r["Dynamic Stack"] == "False" and r["ScratchSize"] == 0 and r["VGPRs Spill"] == 0, (name, r)
