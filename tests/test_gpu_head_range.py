"""cfgzip_head_loss_grad where grad_loss lies at the ends of its range, or rows of very different grad_loss stand beside each other, in
each of the forms that dz is kept in, against the definition in 64 bits with the bounds of tests/head_rounding.py."""

import numpy as np
import pytest

from head_reference import pack
from head_rounding import few_rows, gradients

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def lib():
    import paper_2605_29986_amd as p
    p.load_library()
    return p


def _close(got, want, err, name):
    got = got.double().cpu().numpy()
    bad = ~(np.abs(got - want) <= err)
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:5].tolist(), got[bad][:5], want[bad][:5], err[bad][:5])


def _check(lib, h, w, target, allowed, g, dtype):
    from gpu_util import dev
    masks = {} if allowed.all() else {"bits": dev(pack(allowed))}
    t = dev(target.astype(np.int32))
    _, lse = lib.cfgzip_head_loss(h.cuda(), w.cuda(), t, **masks)
    gh, gw = lib.cfgzip_head_loss_grad(h.cuda(), w.cuda(), t, lse, dev(g), **masks)
    r = gradients(h.double().numpy(), w.double().numpy(), target, allowed, g.astype(np.float64), lse.double().cpu().numpy(), dtype,
                  few_rows(*h.shape, dtype))
    _close(gh, r["grad_hidden"], r["grad_hidden_err"], "grad_hidden")
    _close(gw, r["grad_weight"], r["grad_weight_err"], "grad_weight")
    return gh, gw


@pytest.mark.parametrize("scale", [1e-40, 1e-35, 1e-26, 1.0, 1e20, 2.0 ** 115, 2.0 ** 121])
@pytest.mark.parametrize("N,D", [(33, 64), (200, 65), (300, 64)])
def test_ends_of_the_range(lib, N, D, scale):
    """The largest gradient far below and above what fp16 holds"""
    print(f"case N={N} D={D} scale={scale}", flush=True)
    rng = np.random.default_rng(2)
    V = 400
    h = torch.from_numpy(rng.standard_normal((N, D))).bfloat16()
    w = torch.from_numpy(rng.standard_normal((V, D)) * 0.2).bfloat16()
    g = (rng.standard_normal(N) * scale).astype(np.float32)
    _check(lib, h, w, rng.integers(0, V, size=N), np.ones((N, V), bool), g, "bf16")


@pytest.mark.parametrize("dtype,N,D", [("bf16", 40, 72), ("bf16", 200, 65), ("bf16", 300, 72), ("f16", 24, 72), ("f16", 200, 72), ("f16", 300, 72)])
def test_rows_of_very_different_gradients(lib, dtype, N, D):
    """grad_loss over seven powers of ten; weights with a common mean, so that a row's small probabilities make up half of its gradient"""
    print(f"case {dtype} N={N} D={D}", flush=True)
    rng = np.random.default_rng(4)
    V = 30_000
    h = torch.from_numpy(rng.standard_normal((N, D)) * 0.3).to(TYPES[dtype])
    w = torch.from_numpy(rng.standard_normal((V, D)) * 0.2 + 0.25).to(TYPES[dtype])
    g = (16384.0 * 10.0 ** -rng.uniform(0, 7, size=N)).astype(np.float32)
    g[0], g[1] = 16384.0, 16384e-7
    _check(lib, h, w, rng.integers(0, V, size=N), np.ones((N, V), bool), g, dtype)


@pytest.mark.parametrize("dtype,N,D", [("bf16", 300, 72), ("f16", 24, 72), ("f16", 300, 72)])
def test_tokens_of_rows_with_small_gradients(lib, dtype, N, D):
    """A third of the vocabulary is admitted by rows with a ten-thousandth of the others' grad_loss only: nothing covers what is lost there"""
    print(f"case {dtype} N={N} D={D}", flush=True)
    rng = np.random.default_rng(6)
    V = 3_000
    h = torch.from_numpy(rng.standard_normal((N, D)) * 0.3).to(TYPES[dtype])
    w = torch.from_numpy(rng.standard_normal((V, D)) * 0.2).to(TYPES[dtype])
    small = np.arange(N) % 2 == 1
    allowed = np.zeros((N, V), bool)
    allowed[small, :1000], allowed[~small, 1000:] = True, True
    target = np.where(small, rng.integers(0, 1000, size=N), rng.integers(1000, V, size=N))
    g = (rng.standard_normal(N) * np.where(small, 1.0, 1e4)).astype(np.float32)
    gh, gw = _check(lib, h, w, target, allowed, g, dtype)
    assert (gw[:1000] != 0).any(1).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("N", [20, 300])
def test_a_gradient_that_is_not_finite_stays_with_its_row(lib, dtype, N):
    """grad_hidden of the other rows is what it is without it, and nothing hides it in its own"""
    from gpu_util import dev
    rng = np.random.default_rng(8)
    V, D = 500, 64
    h = torch.from_numpy(rng.standard_normal((N, D))).to(TYPES[dtype]).cuda()
    w = torch.from_numpy(rng.standard_normal((V, D)) * 0.2).to(TYPES[dtype]).cuda()
    t = dev(rng.integers(0, V, size=N).astype(np.int32))
    g = rng.standard_normal(N).astype(np.float32)
    _, lse = lib.cfgzip_head_loss(h, w, t)
    want, _ = lib.cfgzip_head_loss_grad(h, w, t, lse, dev(g), want_weight=False)
    for bad in (np.inf, -np.inf, np.nan):
        g[3] = bad
        gh, gw = lib.cfgzip_head_loss_grad(h, w, t, lse, dev(g))
        assert not torch.isfinite(gh[3]).any() and not torch.isfinite(gw).all()
        others = torch.arange(N, device="cuda") != 3
        assert torch.isfinite(gh[others]).all()
        assert ((gh[others].float() - want[others].float()).abs() <= 2e-2 * want[others].float().abs().amax(1, keepdim=True)).all()
