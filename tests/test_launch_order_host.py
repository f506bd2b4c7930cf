"""Kernels launched with programmatic stream serialisation may start before what is ahead of them has finished, and see what was written before only behind a
griddepcontrol.wait of their own.  Checked in the source: a program that reads ahead of it gives the right results nearly always."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2304_04237_b200", "csrc")
SOURCES = ["dropout_kernel.cu", "norm_kernel.cu", "select_kernel.cu", "sparse_bwd_kernel.cu", "sparse_kernel.cu"]


def kernels(source):
    """Names and bodies of a file's kernels."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, source)).read())
    for m in re.finditer(r"__global__ void(?: __launch_bounds__\((?:[^()]|\([^()]*\))*\))?\s+(\w+)\(", text):
        start = text.index("{", text.index(")", m.end()))
        depth, at = 0, start
        while True:
            depth += {"{": 1, "}": -1}.get(text[at], 0)
            if depth == 0:
                break
            at += 1
        yield m.group(1), text[start:at]


FOUND = [(s, name, body) for s in SOURCES for name, body in kernels(s)]


def test_all_kernels_are_found():
    found = [name for _, name, _ in FOUND]
    assert len(found) == len(set(found)) and len(found) == sum(open(os.path.join(CSRC, s)).read().count("__global__") for s in SOURCES)


@pytest.mark.parametrize("source,name,body", FOUND, ids=[name for _, name, _ in FOUND])
def test_a_kernel_waits_before_it_reads(source, name, body):
    """The wait stands ahead of every loop, every copy, and every branch that a part of the threads takes."""
    wait = body.index("grid_dependency_wait();")
    reads = re.search(r"\b(for|while|if)\b|\bsend\w*[<(]|\bcopy\w*\(|\bMaps maps\(|\binvert\(|\*reinterpret_cast|\*static_cast", body)
    assert reads is None or wait < reads.start()
