"""CPU: the kernels at the ends of a training step keep nothing in scratch memory and spill no register (from the compiler's report, which the build writes down)."""
import json
import os

import pytest

from paper_2509_25149_amd import build

KERNELS = ("embedding_forward_kernel", "rank_kernel", "zero_kernel", "sort_count_kernel", "sort_scan_kernel", "sort_place_kernel", "embedding_sum_kernel", "embedding_join_kernel",
           "embedding_few_kernel", "logprob_forward_kernel", "logprob_join_kernel", "logprob_backward_kernel", "logprob_loss_kernel", "grad_sumsq_kernel", "grad_fold_kernel",
           "grad_clip_kernel")


@pytest.mark.parametrize("kernel", KERNELS)
def test_kernels_stay_in_registers(kernel):
    if not os.path.exists(build.RESOURCES):
        pytest.skip("libnvfp4_hip.resources.json is written by build(); run it first")
    reports = {name: r for name, r in json.load(open(build.RESOURCES)).items() if kernel in name}
    assert reports
    for name, r in reports.items():
        assert r["Dynamic Stack"] == "False" and r["ScratchSize"] == 0 and r["VGPRs Spill"] == 0, (name, r)
