"""The vocabulary projection's calls without a GPU: what the C ABI refuses before any device work, the workspace queries, what the
binding refuses, and the references of the GPU tests against themselves."""

import ctypes
import os

import numpy as np
import pytest

from head_reference import VALUES, loss_and_gradients, pack, quantize, unpack, values

P = ctypes.c_void_p


@pytest.fixture(scope="module")
def raw():
    from paper_2605_29986_amd import binding, build
    if not os.path.exists(binding.library_path()):
        build.build()
    return binding.load_library()


@pytest.fixture(scope="module")
def memory():
    buf = ctypes.create_string_buffer(8192)
    return (ctypes.addressof(buf) + 255) // 256 * 256, buf


def _loss(raw, p, **change):
    a = dict(hidden=p, hs=8, weight=p, ws=8, dtype=1, N=4, V=10, D=8, target=p, bits=None, kind=2, c=None, C=0, loss=p, lse=p, work=p,
             size=1 << 30)
    a.update(change)
    return raw.cfgzip_head_loss(*a.values(), None)


def _grad(raw, p, **change):
    a = dict(hidden=p, hs=8, weight=p, ws=8, dtype=1, N=4, V=10, D=8, target=p, bits=None, kind=2, c=None, C=0, lse=p, g=p, gh=p, ghs=8,
             gw=p, gws=8, work=p, size=1 << 30)
    a.update(change)
    return raw.cfgzip_head_loss_grad(*a.values(), None)


def _logits(raw, p, **change):
    a = dict(hidden=p, hd=1, hs=64, hsc=None, codes=p, scales=p, B=40, V=10, K=64, bits=None, kind=2, c=None, C=0, out=p, dtype=0, stride=10,
             work=None, size=0)
    a.update(change)
    return raw.cfgzip_mx4_logits(*a.values(), None)


def test_loss_refuses(raw, memory):
    p = memory[0]
    both = [dict(hidden=None), dict(weight=None), dict(target=None), dict(dtype=0), dict(dtype=3), dict(N=-1), dict(V=0), dict(D=0),
            dict(hs=7), dict(ws=7), dict(hidden=p + 1), dict(weight=p + 1), dict(target=p + 2), dict(kind=3), dict(kind=-1), dict(kind=0),
            dict(kind=1, bits=p), dict(kind=1, bits=p, c=p, C=0), dict(kind=0, bits=p + 2), dict(lse=None), dict(lse=p + 2)]
    for change in both + [dict(loss=None), dict(loss=p + 1)]:
        assert _loss(raw, p, **change) == -1, change
    for change in both + [dict(g=None), dict(gh=None, gw=None), dict(ghs=7), dict(gws=7), dict(gh=p + 1), dict(gw=p + 1), dict(g=p + 2)]:
        assert _grad(raw, p, **change) == -1, change
    for call in (_loss, _grad):
        for change in (dict(work=None), dict(work=p + 16), dict(size=64)):
            assert call(raw, p, **change) == -2, change
        for change in (dict(ws=1 << 22), dict(V=0x7FFFFFFF), dict(D=1 << 22, hs=1 << 22, ws=1 << 22)):
            assert call(raw, p, **change) == -5, change
    assert _loss(raw, p, N=0, hidden=None, target=None) == 0
    assert _grad(raw, p, N=0, hidden=None, target=None, gw=None) == 0


def test_quantize_refuses(raw, memory):
    p = memory[0]
    for bad in ((None, 0, 4, 8, 8, p, p), (p, 3, 4, 8, 8, p, p), (p, -1, 4, 8, 8, p, p), (p, 0, -1, 8, 8, p, p), (p, 0, 4, 0, 8, p, p),
                (p, 0, 4, 8, 7, p, p), (p, 0, 4, 8, 8, None, p), (p, 0, 4, 8, 8, p, None), (p + 2, 0, 4, 8, 8, p, p), (p + 1, 1, 4, 8, 8, p, p),
                (p, 0, 4, 8, 8, p + 8, p)):
        assert raw.cfgzip_mx4_quantize(*bad, None) == -1, bad
        x, dtype, R, K, stride, codes, scales = bad
        assert raw.cfgzip_mx4_values(codes, scales, R, K, x, dtype, stride, None) == -1, bad
    assert raw.cfgzip_mx4_quantize(p, 0, 1, (1 << 22) + 1, 1 << 23, p, p, None) == -5
    assert raw.cfgzip_mx4_quantize(None, 0, 0, 8, 8, None, None, None) == 0
    assert raw.cfgzip_mx4_values(None, None, 0, 8, None, 0, 8, None) == 0


def test_logits_refuse(raw, memory):
    p = memory[0]
    for change in (dict(hidden=None), dict(codes=None), dict(scales=None), dict(out=None), dict(hd=0), dict(hd=4), dict(dtype=2),
                   dict(B=-1), dict(V=0), dict(K=0), dict(stride=9), dict(hs=63), dict(hidden=p + 1), dict(codes=p + 8), dict(out=p + 2),
                   dict(hd=3, hs=32), dict(hd=3, hs=64, hsc=p), dict(hd=3, hs=32, hsc=p, hidden=p + 8), dict(kind=7), dict(kind=0),
                   dict(kind=1, bits=p, c=None, C=5), dict(kind=1, bits=p, c=p, C=0), dict(kind=0, bits=p + 1)):
        assert _logits(raw, p, **change) == -1, change
    # masks over classes become masks over tokens in the workspace, fp16 hidden states sums of two bf16 numbers
    for change in (dict(kind=1, bits=p, c=p, C=5), dict(hd=2)):
        assert _logits(raw, p, **change) == -2, change
        assert _logits(raw, p, work=p, size=16, **change) == -2, change
        assert _logits(raw, p, work=p + 16, size=1 << 20, **change) == -2, change
    assert _logits(raw, p, V=0x7FFFFFFF, stride=0x7FFFFFFF) == -5
    assert _logits(raw, p, B=0, hidden=None) == 0


def test_workspace_queries(raw):
    q, g, l = raw.cfgzip_head_loss_workspace_bytes, raw.cfgzip_head_loss_grad_workspace_bytes, raw.cfgzip_mx4_logits_workspace_bytes
    for f in (q, g):
        assert f(0, 10, 8, 2) == 0 and f(4, 0, 8, 2) == 0 and f(4, 10, 0, 2) == 0 and f(4, 10, 8, 3) == 0
        assert f(4, 1000, 64, 1) >= f(4, 1000, 64, 2) + 4 * 32 * 4  # token masks
    # never the logits: 4,096 rows of 128,256 tokens would be 1 GB of 16 bits; dz of a piece and fp32 sums are kept
    assert q(4096, 128256, 4096, 2) < 80 << 20
    assert g(4096, 128256, 4096, 2) < (256 << 20) + (4096 * 4096 * 6) + (1 << 20)
    assert l(1, 1, 1000, 64, 1) == 0 and l(1, 40, 1000, 64, 2) > 0 and l(3, 40, 1000, 64, 2) == 0
    assert l(3, 40, 1000, 64, 1) >= 40 * 32 * 4 and l(2, 40, 1000, 64, 2) >= 2 * l(1, 40, 1000, 64, 2) - 512
    assert l(0, 4, 10, 8, 2) == 0 and l(1, 0, 10, 8, 2) == 0


def test_binding_refuses_cpu_tensors():
    torch = pytest.importorskip("torch")
    import paper_2605_29986_amd as lib
    w, t = torch.zeros((4, 8), dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(TypeError):
        lib.cfgzip_head_loss(w, w, t)
    with pytest.raises(TypeError):
        lib.cfgzip_head_loss_grad(w, w, t, t, t)
    with pytest.raises(TypeError):
        lib.cfgzip_mx4_quantize(w)
    u = torch.zeros((4, 16), dtype=torch.uint8)
    with pytest.raises(TypeError):
        lib.cfgzip_mx4_values(u, u[:, :1], 8)
    with pytest.raises(TypeError):
        lib.cfgzip_mx4_logits(w, u, u[:, :1])


# ---------------------------------------------------------------- the references


def test_reference_gradients_against_differences():
    rng = np.random.default_rng(0)
    N, V, D = 5, 40, 6
    h, w, g = rng.standard_normal((N, D)), rng.standard_normal((V, D)), rng.standard_normal(N)
    allowed = rng.random((N, V)) < 0.6
    target = np.array([np.flatnonzero(a)[0] for a in allowed])
    r = loss_and_gradients(h, w, target, allowed, g, "bf16")

    def total(x, y):
        return float((loss_and_gradients(x, y, target, allowed, None, "bf16")["loss"] * g).sum())

    e = 1e-5
    for a, grad, which in ((h, r["grad_hidden"], 0), (w, r["grad_weight"], 1)):
        for at in ((0, 0), (1, 3), (4, 5)):
            up, down = a.copy(), a.copy()
            up[at] += e
            down[at] -= e
            slope = (total(up, w) - total(down, w) if which == 0 else total(h, up) - total(h, down)) / (2 * e)
            assert abs(slope - grad[at]) < 1e-7 * (1 + abs(slope)), (which, at)


def test_reference_losses():
    h, w = np.array([[1.0], [1.0], [np.nan], [1.0]]), np.array([[0.0], [1.0], [np.log(2.0)]])
    allowed = np.array([[1, 1, 1], [1, 0, 1], [1, 1, 1], [0, 0, 0]], bool)
    r = loss_and_gradients(h, w, np.array([0, 1, -1, 2]), allowed, np.ones(4), "bf16")
    assert np.allclose(r["lse"][:2], [np.log(3 + np.e), np.log(3.0)]) and r["lse"][3] == -np.inf
    assert np.isclose(r["loss"][0], np.log(3 + np.e)) and r["loss"][1] == np.inf and r["loss"][2] == 0 and r["loss"][3] == np.inf
    assert (r["grad_hidden"][1:] == 0).all() and np.isclose(r["grad_weight"].sum(), 0.0)


def test_reference_codes():
    x = np.zeros((1, 32))
    x[0, :16] = np.concatenate([VALUES, -VALUES])
    c, s = quantize(x)
    assert s[0, 0] == 127 and (values(c, s, 32) == x).all()
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 4.0] + [0.0] * 24)[None]
    c, s = quantize(ties)
    assert values(c, s, 8)[0].tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 4.0]
    c, s = quantize(np.array([[7.9, np.inf, 1e-45]]))
    assert s[0, 0] == 255 and (c == 0).all() and np.isnan(values(c, s, 3)).all()
    rows = np.random.default_rng(0).random((3, 70)) < 0.5
    assert (unpack(pack(rows), 70) == rows).all()
