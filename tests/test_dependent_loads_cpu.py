"""Kernels that may be set up while the kernel before them still writes their inputs read them by plain loads: the
read-only path (__ldg, ld.global.nc, const __restrict__ parameters) is specified for data that nothing writes while the
kernel lives, and theirs begins before their producer's ends."""
import glob
import os
import re

import pytest

from paper_1809_10572_gb300 import build

WAIT = "grid_dependency_wait()"


def code(path):
    text = open(path).read()
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))


def dependent_sources():
    files = sorted(glob.glob(os.path.join(build.CSRC, "*.cu*")))
    return [f for f in files if WAIT in re.sub(r"void grid_dependency_wait\(\)", "", code(f))]


def test_the_dependent_kernels_are_found():
    names = {os.path.basename(f) for f in dependent_sources()}
    assert {"conv_kernel.cuh", "matvec4_kernel.cuh", "block8.cu", "ffn.cu"} <= names


@pytest.mark.parametrize("path", dependent_sources(), ids=os.path.basename)
def test_no_read_only_loads(path):
    found = re.findall(r"__ldg\b|\bld\.global\.nc\b|const\s+[\w:]+\s*\*\s*(?:const\s+)?__restrict__\s*\w*", code(path))
    assert not found, found
