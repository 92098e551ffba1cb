"""No kernel of the paged cache keeps registers in scratch memory: the compiler's own report of every instance (no GPU needed)."""
import os
import re
import subprocess

import pytest

from paper_2604_17397_amd import build


@pytest.mark.parametrize("source,kernels", [("paged_attn.hip", ("paged_attn_kernel", "paged_join_kernel")), ("paged_rows.hip", ("paged_rows_kernel",)),
                                            ("page_plan.hip", ("page_plan_kernel",))])
def test_paged_kernels_do_not_spill(source, kernels):
    cmd = [os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *build.HIPCC_FLAGS, *(build.PRELOAD_FLAGS if source in build.PRELOADED else []),
           "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage",
           "-c", os.path.join(build.CSRC, source), "-o", os.devnull]
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout
    use = re.findall(r"Function Name: (\S+).*?ScratchSize \[bytes/lane\]: (\d+).*?VGPRs Spill: (\d+)", res.stdout, re.S)
    for name in kernels:
        assert any(name in f for f, _, _ in use), name
    assert [u for u in use if u[1:] != ("0", "0")] == []
