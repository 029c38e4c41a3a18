"""No kernel of the w4g products keeps registers in scratch memory: the build refuses one, and the built ones have none."""
import os

import pytest

from tests.test_stage_barriers import OBJDUMP, _kernels


def test_the_build_finds_scratch_memory_in_the_compilers_remarks():
    from paper_2310_09259_amd import build
    remark = ("a.hip:1:1: remark: Function Name: {} [-Rpass-analysis=kernel-resource-usage]\n"
              "a.hip:1:1: remark:     ScratchSize [bytes/lane]: {} [-Rpass-analysis=kernel-resource-usage]\n")
    text = "".join(remark.format(*v) for v in (("_Z16w4g_tiles_kernelv", 0), ("_Z15w4g_rows_kernelv", 12), ("_Z11gemm_kernelv", 8)))
    assert build.scratch_users(text) == [("_Z15w4g_rows_kernelv", 12)]


def test_the_built_kernels_have_none(tmp_path):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    kernels = {k: v for k, v in _kernels(str(tmp_path)).items() if "w4g_" in k}
    assert len(kernels) > 80
    assert not [k for k, code in kernels.items() if any(op.startswith("scratch_") for _, op, _, _ in code)]
