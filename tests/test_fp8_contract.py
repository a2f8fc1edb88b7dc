"""What can be seen without a GPU of the 8-bit operands' kernels and entry points."""
import os
import re

import pytest

from paper_1905_10759_b200 import build

build.build_lib()


def source(name):
    with open(os.path.join(build.CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


@pytest.mark.parametrize("name,published", [("fp8_gemm.cu", "sfull"), ("fp8_weight_grad.cu", "bfull")])
def test_what_crosses_a_pair_of_ctas_is_released_and_acquired_at_cluster_scope(name, published):
    """The arrival that releases nothing beyond its CTA frees what was read (barriers called ...empty) and announces nothing that was
    written; the barrier that does is completed by st_async_u32 from the other CTA and waited for with an acquire of that scope."""
    code = source(name)
    freed = re.findall(r"mbar_arrive_cluster_read\((.*)\);", code)
    assert freed and all("empty" in a for a in freed), freed
    assert re.search(r"st_async_u32\([^;]*%s" % published, code)
    waits = re.findall(r"\bwait(\.cluster)?\((?:smem_u32\(&%s\[|%s_a)" % (published, published), code)
    assert waits and all(waits), waits
