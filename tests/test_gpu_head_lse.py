"""cfgzip_head_loss_grad takes the lse that it is given, whatever the number of rows: dz = grad_loss (exp(z - lse) - [v = target]), against
the definition in 64 bits with the bounds of tests/head_rounding.py."""

import numpy as np
import pytest

from head_reference import pack
from head_rounding import few_rows, gradients
from test_gpu_head_range import TYPES, _close, lib  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("N,D", [(1, 64), (9, 72), (40, 64), (128, 65), (200, 64), (256, 72), (257, 72), (400, 65)])
def test_another_lse(lib, dtype, N, D):  # noqa: F811
    print(f"case {dtype} N={N} D={D}", flush=True)
    from gpu_util import dev
    rng = np.random.default_rng(N + D)
    V = 700
    h = torch.from_numpy(rng.standard_normal((N, D))).to(TYPES[dtype])
    w = torch.from_numpy(rng.standard_normal((V, D)) * 0.3).to(TYPES[dtype])
    allowed = rng.random((N, V)) < 0.5
    target = np.array([rng.choice(np.flatnonzero(a)) for a in allowed])
    g = rng.standard_normal(N).astype(np.float32)
    t, bits = dev(target.astype(np.int32)), dev(pack(allowed))
    _, lse = lib.cfgzip_head_loss(h.cuda(), w.cuda(), t, bits=bits)
    # tokens beside these (a sum that is larger), one token less, and the least that is another number
    apart = torch.from_numpy(rng.choice([-0.25, 0.0, 1e-3, 0.5, 4.0, 60.0], size=N).astype(np.float32)).cuda()
    given = lse + apart
    gh, gw = lib.cfgzip_head_loss_grad(h.cuda(), w.cuda(), t, given, dev(g), bits=bits)
    r = gradients(h.double().numpy(), w.double().numpy(), target, allowed, g.astype(np.float64), given.double().cpu().numpy(), dtype,
                  few_rows(N, D, dtype))
    _close(gh, r["grad_hidden"], r["grad_hidden_err"], "grad_hidden")
    _close(gw, r["grad_weight"], r["grad_weight_err"], "grad_weight")


@pytest.mark.parametrize("N", [20, 300])
def test_an_lse_of_infinity_leaves_the_targets(lib, N):  # noqa: F811
    """exp(z - inf) is 0: what remains is -grad_loss weight[target] and -grad_loss hidden at the target"""
    from gpu_util import dev
    rng = np.random.default_rng(3)
    V, D = 400, 64
    h = torch.from_numpy(rng.standard_normal((N, D))).bfloat16()
    w = torch.from_numpy(rng.standard_normal((V, D)) * 0.3).bfloat16()
    target = rng.permutation(V)[:N]
    t = dev(target.astype(np.int32))
    gh, gw = lib.cfgzip_head_loss_grad(h.cuda(), w.cuda(), t, torch.full((N,), float("inf"), device="cuda"), torch.ones(N, device="cuda"))
    assert torch.equal(gh.cpu(), -w[torch.from_numpy(target)])
    want = torch.zeros_like(w)
    want[torch.from_numpy(target)] = -h
    assert torch.equal(gw.cpu(), want)
