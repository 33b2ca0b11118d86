"""Kernels launched to set themselves up while the one in front on the stream finishes: in the source of each, nothing of the
caller's memory is read before the wait for that one (visibility is promised to a thread that has waited, to no other)."""
import os
import re

import pytest

from paper_1902_01064_b200 import build

KERNELS = {"hop_norm.cu": ["dropout_kernel", "dropout_askew_kernel", "norm_sums_kernel"], "hop_norm.cuh": ["norm_forward_kernel", "norm_backward_kernel"],
           "hop_linear.cu": ["linear_tc_kernel", "linear_join_kernel", "linear_pack_kernel"]}


def source(name):
    with open(os.path.join(build.CSRC, name)) as f:
        return f.read()


def kernel(file, name):
    """(parameters, body) of a kernel; the set-up that both norm kernels share stands in their bodies."""
    text = source(file)
    m = re.search(r"\n" + name + r"\((.*?)\) \{\n(.*?)\n\}\n", text, re.S)
    setup = re.search(r"#define HOP_TEAM_SETUP\(.*?\n\n", source("hop_norm.cuh"), re.S).group(0)
    return m.group(1), m.group(2).replace("HOP_TEAM_SETUP(", setup + "(")


@pytest.mark.parametrize("file,name", [(f, n) for f, names in KERNELS.items() for n in names])
def test_no_read_before_the_wait(file, name):
    _, body = kernel(file, name)
    waits = [m.start() for m in re.finditer(r"dependency_wait\(\);", body) if "return" not in body[m.end():m.end() + 10] and "if (" not in body[:m.start()].rsplit("\n", 1)[-1]]
    assert waits, "every kernel waits, whatever its arguments"
    before = body[:waits[0]]
    for read in (r"offsets\[", r"op_group_of", r"\b[pq][xy]?\[", r"reinterpret_cast<const u?int", r"reinterpret_cast<const float", r"a\.\w+\["):
        assert not re.search(read, before), read


@pytest.mark.parametrize("file,name", [(f, n) for f, names in KERNELS.items() for n in names])
def test_no_pointer_promises_that_nobody_else_writes(file, name):
    """The kernel in front may still be writing when one of these begins, and dropout's result may be its operand."""
    parameters, body = kernel(file, name)
    assert "__restrict__" not in parameters and "__ldg" not in body and "ld.global.nc" not in body


def test_all_kernels_are_looked_at():
    for file, names in KERNELS.items():
        found = re.findall(r"__global__ void __launch_bounds__\([^)]*\)\n(\w+)\(", source(file))
        assert sorted(n for n in found if "selftest" not in n) == sorted(names)
