"""The build's look at the kernels' scratch memory leaves no kernel out."""
import glob
import os
import re

from paper_2505_21594_amd import build


def kernels():
    names = set()
    for path in glob.glob(os.path.join(build.CSRC, "*.h*p")):
        for line in open(path):
            m = re.search(r"__global__ .*?(\w+_kernel)\(", line)
            if m:
                names.add(m[1])
    return names


def remarks(name, scratch):
    return f"x.hip:1:1: remark: Function Name: _ZN2ee{len(name)}{name}EPv [-Rpass]\nx.hip:1:1: remark:     ScratchSize [bytes/lane]: {scratch} [-Rpass]\n"


def test_every_kernel_is_looked_at():
    names = kernels()
    assert {"ee_gemm_kernel", "ee_distill_kernel", "ee_norm_grad_kernel", "ee_column_sums_kernel", "ee_score_kernel", "ee_slope_kernel", "ee_gemm16_kernel", "ee_attend_wide_kernel"} <= names
    for name in names:
        accepted = build.ACCEPTED_SCRATCH.get(name, 0)
        assert build.check_resources(remarks(name, accepted)) == []
        found = build.check_resources(remarks(name, accepted + 4))
        assert len(found) == 1 and name in found[0] and str(accepted + 4) in found[0]


def test_what_is_accepted_is_a_kernel_of_the_library():
    assert set(build.ACCEPTED_SCRATCH) <= kernels()
