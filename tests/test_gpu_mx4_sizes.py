"""cfgzip_mx4_logits at hidden sizes that each kernel takes in its own way: whole pairs of steps that are read where they lie, many steps,
strides, with the bound of an fp32 sum (tests/test_gpu_mx4.py)."""

import pytest

from test_gpu_mx4 import _check_logits, lib  # noqa: F401

pytestmark = pytest.mark.gpu

pytest.importorskip("torch")


@pytest.mark.parametrize("x_type", ["bf16", "f16", "4"])
@pytest.mark.parametrize("mask", ["none", "class", "token"])
@pytest.mark.parametrize("B,V,K", [(65, 300, 256), (100, 257, 512), (128, 1000, 1024), (200, 515, 256), (256, 256, 768), (300, 700, 2304)])
def test_whole_pairs_of_steps(lib, B, V, K, mask, x_type):  # noqa: F811
    _check_logits(lib, B, V, K, x_type, mask, out="bf16" if V % 2 else "f32", seed=2)


@pytest.mark.parametrize("pad,offset", [(8, 0), (256, 8), (3, 0), (8, 1)])
@pytest.mark.parametrize("B", [20, 70, 256])
def test_rows_of_whole_pairs_some_distance_apart(lib, B, pad, offset):  # noqa: F811
    """Rows that lie at multiples of 16 bytes are read where they are, others through a copy"""
    for x_type in ("bf16", "f16"):
        _check_logits(lib, B, 300, 512, x_type, "class", seed=3, pad=pad, offset=offset)


@pytest.mark.parametrize("x_type", ["bf16", "f16", "4"])
@pytest.mark.parametrize("B,V,K", [(17, 300, 4096), (33, 257, 2560), (40, 140, 4000), (64, 515, 4096), (64, 130, 9000), (10, 300, 8192), (90, 300, 5000)])
def test_many_steps(lib, B, V, K, x_type):  # noqa: F811
    _check_logits(lib, B, V, K, x_type, "class", seed=4)
