"""Kernels that are launched while their predecessor in the stream still runs must not read through the non-coherent path
(__ldg, ld.global.nc, pointers the compiler may take for read-only ones): it asks for memory that nothing writes for as long as the
kernel lives, and these live while the kernel before writes what they read."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_26660_b200", "csrc")
HEADERS = {"tcgen05.cuh", "typed.cuh", "feed_forward.cuh", "lora.cuh"}   # what such kernels are built from


def code(name):
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


OVERLAPPED = sorted(f for f in os.listdir(CSRC) if f in HEADERS or (f.endswith(".cu") and "launch_dependents()" in code(f)))


def test_the_kernels_are_found():
    assert HEADERS | {"product.cu", "product_few.cu", "weight_gradient.cu", "quantize_rows.cu", "feed_forward.cu"} <= set(OVERLAPPED)


@pytest.mark.parametrize("name", OVERLAPPED)
def test_no_non_coherent_loads(name):
    found = re.findall(r"__ldg\b|\.nc\b|__restrict__", code(name))
    assert not found, found
