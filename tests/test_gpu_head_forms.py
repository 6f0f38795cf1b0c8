"""cfgzip_head_loss_grad within bounds that know in which form dz is kept (tests/head_rounding.py): two numbers of few rows, one fp16 number
of more, in one piece of the vocabulary and in several."""

import numpy as np
import pytest

from test_gpu_head_range import TYPES, _check, lib  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("mask", [False, True])
@pytest.mark.parametrize("N,V,D", [(1, 300, 40), (17, 257, 72), (40, 130, 128), (64, 2000, 136), (128, 515, 65), (129, 300, 40), (129, 515, 65),
                                   (256, 1000, 128), (257, 515, 80), (300, 4000, 33), (513, 700, 264)])
def test_sizes(lib, N, V, D, mask, dtype):  # noqa: F811
    print(f"case {dtype} N={N} V={V} D={D} mask={mask}", flush=True)
    rng = np.random.default_rng(N + V + D)
    w = torch.from_numpy(rng.standard_normal((V, D)) * (2.0 / np.sqrt(D))).to(TYPES[dtype])
    h = torch.from_numpy(rng.standard_normal((N, D))).to(TYPES[dtype])
    allowed = rng.random((N, V)) < 0.3 if mask else np.ones((N, V), bool)
    target = np.array([rng.choice(np.flatnonzero(a)) for a in allowed])
    if N > 4:
        target[1], target[2], target[3] = -1, V, np.argmin(allowed[3])
    sure = np.arange(N) % 3 == 0  # a certain target here and there
    h[sure] += 3.0 * w[torch.from_numpy(np.clip(target, 0, V - 1))][sure]
    g = (rng.standard_normal(N) / N).astype(np.float32)
    if N > 5:
        g[5] = 0.0
    _check(lib, h, w, target, allowed, g, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_the_gradient_of_a_mean_is_rounded_once(lib, dtype):  # noqa: F811
    """The same grad_loss for all rows, certain and wrong: dz of the target is -grad_loss, which no form of dz rounds, and each token is
    the target of one row, so what is left is the result's own rounding (and the other tokens' e^-17 each)."""
    from gpu_util import dev
    rng = np.random.default_rng(1)
    N, V, D = 300, 301, 64
    w = torch.zeros((V, D))
    w[300] = 5.0  # what all rows are certain of
    h = torch.from_numpy(0.25 + rng.random((N, D))).to(TYPES[dtype])
    h = (h.float() * (20.0 / (5.0 * h.float().sum(1, keepdim=True)))).to(TYPES[dtype])  # a logit of 20
    t = dev(rng.permutation(300).astype(np.int32))
    g = np.full(N, 1.0 / N, dtype=np.float32)
    wd = w.to(TYPES[dtype]).cuda()
    _, lse = lib.cfgzip_head_loss(h.cuda(), wd, t)
    _, gw = lib.cfgzip_head_loss_grad(h.cuda(), wd, t, lse, dev(g))
    want = -(h.double() * float(g[0]))
    half = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}[dtype]
    got = gw.cpu().double()[t.cpu().long()]
    assert ((got - want).abs() <= half * want.abs() + 400 * 2.0 ** -27 / N + 2.0 ** -25).all()


def test_several_pieces(lib):  # noqa: F811
    """dz of several pieces, the last of them ragged, sums carried from piece to piece, against 64 bits on the GPU: dz and grad_weight's
    hidden states off by half a step of fp16 each, weights kept as they are."""
    N, V, D = 2_500, 131_073, 64
    gen = torch.Generator(device="cuda").manual_seed(4)
    h = torch.randn((N, D), device="cuda", generator=gen).bfloat16()
    w = (torch.randn((V, D), device="cuda", generator=gen) * 0.2).bfloat16()
    t = torch.randint(0, V, (N,), device="cuda", generator=gen).int()
    g = torch.randn((N,), device="cuda", generator=gen)
    _, lse = lib.cfgzip_head_loss(h, w, t)
    gh, gw = lib.cfgzip_head_loss_grad(h, w, t, lse, g)
    hd, wd, gd = h.double(), w.double(), g.double()[:, None]
    # of a probability: the logit's D products and exp's argument, |z - lse| below 40
    z_err = (hd.abs() @ wd.abs().amax(0)[:, None]) * (D + 4) * 2.0 ** -24 + (4 * 40 + 8) * 2.0 ** -24
    wgh, egh = torch.zeros_like(hd), torch.zeros_like(hd)
    for v in range(0, V, 16384):
        n = min(16384, V - v)
        p = torch.exp(hd @ wd[v:v + n].t().contiguous() - lse.double()[:, None])
        dz = p.clone()
        here = torch.nonzero((t >= v) & (t < v + n))[:, 0]
        dz[here, t[here].long() - v] -= 1.0
        dz_err = (dz.abs() * (2.0 ** -11 * 1.01) + 2.0 ** -39 + p * z_err + 2.0 ** -23) * gd.abs()
        dz *= gd
        wgh += dz @ wd[v:v + n]
        egh += dz_err @ wd[v:v + n].abs() + (dz.abs() @ wd[v:v + n].abs()) * ((V + 64) * 2.0 ** -24)
        wgw = dz.t().contiguous() @ hd
        share = 2.0 ** -37 * (hd * gd).abs().max()
        egw = dz_err.t().contiguous() @ hd.abs() + dz.abs().t().contiguous() @ hd.abs() * (2.0 ** -11 * 1.01 + (N + 64) * 2.0 ** -24) \
            + ((dz / gd).abs().sum(0) * share)[:, None]
        bound = egw + wgw.abs() * 2.0 ** -8 * 1.01 + 1e-30
        assert ((gw[v:v + n].double() - wgw).abs() <= bound).all(), v
    assert ((gh.double() - wgh).abs() <= egh + wgh.abs() * 2.0 ** -8 * 1.01 + 1e-30).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("N,V,D", [(300, 16384, 1024), (260, 20000, 1000), (40, 16384, 1024), (2048, 6000, 1001), (1030, 4100, 2048)])
def test_sizes_of_the_largest_tiles(lib, N, V, D, dtype):  # noqa: F811
    """Enough tiles of 256 x 256 for all compute units in one of the three products at least, several rows with one target, and tokens that
    are nobody's"""
    print(f"case {dtype} N={N} V={V} D={D}", flush=True)
    rng = np.random.default_rng(N + V + D)
    w = torch.from_numpy(rng.standard_normal((V, D)) * (2.0 / np.sqrt(D))).to(TYPES[dtype])
    h = torch.from_numpy(rng.standard_normal((N, D))).to(TYPES[dtype])
    target = rng.integers(0, V, size=N)
    target[::3] = target[0]
    target[-1], target[5] = -1, V
    g = (rng.standard_normal(N) * 8).astype(np.float32)
    _check(lib, h, w, target, np.ones((N, V), bool), g, dtype)
