"""Kernels that load to LDS past the registers: a plain barrier does not say that a wave's own loads have come in, so each of their
barriers is one that waits for them (read from the sources, no GPU)."""

import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2605_29986_amd", "csrc")
LOADS = re.compile(r"global_load_lds|\bRows<|\bTile<|\.load\(|\bmultiply<")


def _functions(text):
    """(name, body) of every kernel"""
    for m in re.finditer(r"__global__[^{;]*?void\s+(\w+)\s*\([^{;]*\)\s*\{", text):
        depth, at = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(text[at], 0)
            at += 1
        yield m.group(1), text[m.end():at]


def _kernels():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.hip"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        if "gemm16.hpp" in text:
            for name, body in _functions(text):
                if LOADS.search(body):
                    yield os.path.basename(path), name, body


def test_the_kernels_are_found():
    assert {"logits_kernel", "grad_kernel", "many_rows_kernel", "many_rows4_kernel", "large16_kernel", "large4_kernel"} <= {k[1] for k in _kernels()}


@pytest.mark.parametrize("path,name,body", [pytest.param(*k, id=k[1]) for k in _kernels()])
def test_barriers_wait_for_the_loads(path, name, body):
    assert "__syncthreads" not in body and "s_barrier" not in body
    assert "wait_for_loads<" in body or "multiply<" in body
