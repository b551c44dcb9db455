"""No kernel is compiled that no call reaches (the device assembly of the last build here)."""
import glob
import os
import re

import pytest

from paper_2105_14450_amd import build

ALL_ASM = sorted(glob.glob(os.path.join(build.HERE, "_build", "*-hip-amdgcn-amd-amdhsa-gfx950.s")))


def kernels():
    names = set()
    for path in ALL_ASM:
        with open(path) as f:
            names.update(re.findall(r"\.amdhsa_kernel (\S+)", f.read()))
    return names


@pytest.mark.skipif(not ALL_ASM, reason="no assembly of a build here")
def test_fp8_products_with_fp32_results_and_an_epilogue_are_widened():
    """Neither the tuned kernel, which has the fp8 instructions only, nor the element-wise one in its fp8 form takes them."""
    names = kernels()
    tuned = [n for n in names if "gemm_mfma_kernelI" in n and "EpilogueParams" in n]
    assert sorted(re.search(r"(Fp8|Bf16)E(Li\d+E)", n).group(1) + re.search(r"E([ft])Lb1E", n).group(1) for n in tuned) == \
        ["Bf16f", "Bf16f", "Bf16t", "Bf16t", "Fp8t"]
    generic = [re.search(r"gemm_generic_kernelI([hft])([ft])(?:Lb([01])E)(?:Lb([01])E)(?:Lb([01])E)(?:Lb([01])E)(?:Lb([01])E)", n) for n in names
               if "gemm_generic_kernelI" in n]
    epilogue = sorted(g.group(1) + g.group(2) + g.group(7) for g in generic if g and g.group(6) == "1")
    assert epilogue == ["ff0", "ft0", "hf1", "ht0", "ht1", "tf0", "tt0"]
