"""CPU-only, by the sources: the kernels of a block and of a step are launched so that they may begin while the kernel before them in the stream still
writes what they will read.  They wait for it (griddepcontrol.wait), and what they read then must be read by loads that cannot be moved in front of
the wait and that see what was written while the kernel already ran: no __ldg and no ld.global.nc."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_21446_b200", "csrc")


def code(name):
    """The file without comments."""
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


@pytest.mark.parametrize("name", ["kq_common.cuh", "kq_mma16.cuh", "kq_rotary.cuh", "kq_cache.cuh", "kq_cache_attention.cuh", "kq_linear_w4a16.cuh"])
def test_kernels_of_a_step_read_with_plain_loads(name):
    assert "__ldg" not in code(name) and ".nc" not in code(name)


@pytest.mark.parametrize("name", ["kq_linear.cuh", "kq_norm.cuh"])
def test_kernels_of_a_block_read_with_plain_loads(name):
    assert "__ldg" not in code(name) and ".nc" not in code(name)


@pytest.mark.parametrize("name", ["kq_gemm_fp4.cuh", "kq_gemm_fp4_pair.cuh"])
def test_products_read_the_branch_they_add_with_plain_loads(name):
    assert not re.search(r"__ldg\(ap", code(name))


def test_scale_quantizers_read_their_vector_behind_the_wait():
    body = code("kq_stream.cuh")
    assert not re.search(r"__ldg\(sp", body)
    rows = body[body.index("scale_quantize_rows(") :]
    assert rows.index("griddepcontrol.wait") < rows.index("chan_scale", rows.index("{"))
