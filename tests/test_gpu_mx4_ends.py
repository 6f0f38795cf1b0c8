"""cfgzip_mx4_logits where a row's last block ends inside the step that reads it: what is not finite there stays what it is."""

import numpy as np
import pytest

from head_reference import quantize

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def lib():
    import paper_2605_29986_amd as p
    p.load_library()
    return p


@pytest.mark.parametrize("T", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("K", [1, 31, 33, 64, 96, 130, 200, 288, 512])
@pytest.mark.parametrize("B", [3, 8, 12, 16, 20, 40, 64, 100])
def test_infinity_in_the_last_block(lib, B, K, T):
    """Weights of 1: an infinity makes its row infinite and no other one anything else; a NaN makes its row NaN.  The numbers of rows are
    those of each kernel's range."""
    print(f"case B={B} K={K} {T}", flush=True)
    from gpu_util import dev
    codes, scales = quantize(np.ones((50, K)))
    x = torch.ones((B, K), dtype=T, device="cuda")
    x[0, K - 1], x[1, K - 1], x[2, K // 32 * 32 if K % 32 else K - 32] = float("inf"), float("-inf"), float("nan")
    z = lib.cfgzip_mx4_logits(x, dev(codes), dev(scales))
    assert (z[0] == float("inf")).all() and (z[1] == float("-inf")).all() and z[2].isnan().all() and (z[3:] == K).all()


@pytest.mark.parametrize("K", [33, 96, 200])
@pytest.mark.parametrize("B", [2, 16, 40, 100])
def test_nan_blocks_of_4_bits(lib, B, K):
    """Hidden states in 4 bits whose last block is NaN"""
    print(f"case B={B} K={K}", flush=True)
    from gpu_util import dev
    codes, scales = quantize(np.ones((50, K)))
    x = torch.ones((B, K), device="cuda")
    x[1, K - 1] = float("inf")
    hidden, hidden_scales = lib.cfgzip_mx4_quantize(x)
    z = lib.cfgzip_mx4_logits(hidden, dev(codes), dev(scales), hidden_scales=hidden_scales)
    assert z[1].isnan().all() and (z[0] == K).all() and (z[2:] == K).all()
