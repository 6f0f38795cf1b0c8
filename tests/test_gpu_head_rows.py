"""cfgzip_head_loss_grad around the numbers of rows at which dz changes its form, and weights whose sizes need the power of two that
brings them to fp16, against the definition in 64 bits with the bounds of tests/head_reference.py."""

import numpy as np
import pytest

from head_reference import loss_and_gradients
from test_gpu_head_loss import _check, _close, lib  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("mask", ["none", "class"])
@pytest.mark.parametrize("N,V,D", [(129, 300, 40), (150, 2100, 72), (200, 515, 264), (255, 130, 65), (256, 1000, 128), (257, 515, 80),
                                   (300, 4000, 33), (513, 257, 520)])
def test_rows(lib, N, V, D, mask, dtype):  # noqa: F811
    _check(lib, N, V, D, dtype, mask, seed=N + V + D)


@pytest.mark.parametrize("N", [200, 300])
@pytest.mark.parametrize("scale_w,scale_h", [(1e-20, 1e18), (1e15, 1e-17), (1e-3, 1e-30), (1e-36, 1.0)])
def test_sizes_of_weights_and_hidden_states(lib, N, scale_w, scale_h):  # noqa: F811
    """bf16's range: logits of ordinary size from tiny weights and huge hidden states, and the other way round"""
    print(f"case N={N} {scale_w} {scale_h}", flush=True)
    rng = np.random.default_rng(9)
    V, D = 400, 72
    w = torch.from_numpy(rng.standard_normal((V, D)) * 0.2 * scale_w).bfloat16()
    h = torch.from_numpy(rng.standard_normal((N, D)) * scale_h).bfloat16()
    target = rng.integers(0, V, size=N).astype(np.int32)
    g = (rng.standard_normal(N) / N).astype(np.float32)
    t = torch.from_numpy(target).cuda()
    _, lse = lib.cfgzip_head_loss(h.cuda(), w.cuda(), t)
    gh, gw = lib.cfgzip_head_loss_grad(h.cuda(), w.cuda(), t, lse, torch.from_numpy(g).cuda())
    r = loss_and_gradients(h.double().numpy(), w.double().numpy(), target, np.ones((N, V), bool), g.astype(np.float64), "bf16")
    _close(gh, r["grad_hidden"], r["grad_hidden_err"], "grad_hidden")
    _close(gw, r["grad_weight"], r["grad_weight_err"], "grad_weight")
