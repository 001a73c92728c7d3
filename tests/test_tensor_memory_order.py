"""Kernels let their dependents start only once their own CTA has its tensor memory.

A dependent kernel's CTA may become resident as soon as every CTA of the grid has triggered, takes tensor memory and waits
for the grid's end.  If a CTA triggered while its own allocation was still held up (by another stream's kernel on the same
SM), the dependent could win the columns, and each would wait for the other with nothing that ends it.  No run can show
the order, so the sources do: between an allocation and the trigger lies a barrier of the whole CTA.
"""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_27888_gb300", "csrc")
ALLOC = re.compile(r"\b(?:tmem_alloc|tmem_take(?:<\w+>)?)\(saddr|asm volatile\(\"tcgen05\.alloc\b[^\n]*olumns")
BARRIER = re.compile(r"__syncthreads\(\)|\bmake_table\(")  # make_table ends with one


def sources():
    return [p for p in sorted(glob.glob(os.path.join(CSRC, "*.cu*"))) if ALLOC.search(open(p).read())]


def test_the_kernels_that_allocate_are_found():
    assert [os.path.basename(p) for p in sources()] == ["decode_pipe.cuh", "linear.cu", "linear4_mid.cu"]
    linear = open(os.path.join(CSRC, "linear.cu")).read()
    body = re.search(r"void make_table\([^{]*\{\n(.*?)^}", linear, re.M | re.S).group(1)
    assert body.rstrip().endswith("__syncthreads();")


@pytest.mark.parametrize("path", sources(), ids=os.path.basename)
def test_a_barrier_lies_between_the_allocation_and_the_trigger(path):
    text = re.sub(r"//[^\n]*", "", open(path).read())
    for alloc in ALLOC.finditer(text):
        end = re.search(r"^}", text[alloc.end():], re.M)
        rest = text[alloc.end():alloc.end() + end.start()]
        for trigger in re.finditer(r"pdl_trigger\(\)", rest):
            assert BARRIER.search(rest[:trigger.start()]), "a dependent may take the tensor memory that this CTA waits for"
