"""cfgzip_head_layer and its gradient without a GPU: what the C ABI and the binding refuse, the workspace queries, and the tests' reference against
itself."""

import ctypes
import os

import pytest

torch = pytest.importorskip("torch")

from layer_reference import ACTIVATIONS, activation, forward, gradients


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


def _layer(raw, p, **change):
    a = dict(hidden=p, hs=8, weight=p, ws=8, dtype=1, N=40, M=10, D=8, bias=p, act=4, residual=p, rs=10, out=p, out_dtype=1, os=10, slope=p,
             ss=10, work=p, size=1 << 30)
    a.update(change)
    return raw.cfgzip_head_layer(*a.values(), None)


def _grad(raw, p, **change):
    a = dict(hidden=p, hs=8, weight=p, ws=8, dtype=1, N=40, M=10, D=8, g=p, g_dtype=1, gs=10, slope=p, ss=10, gh=p, ghs=8, gw=p, gws=8, gb=p,
             work=p, size=1 << 30)
    a.update(change)
    return raw.cfgzip_head_layer_grad(*a.values(), None)


BOTH = [dict(hidden=None), dict(weight=None), dict(dtype=0), dict(dtype=3), dict(N=-1), dict(M=0), dict(D=0), dict(hs=7), dict(ws=7),
        dict(hidden=257), dict(weight=257), dict(slope=257), dict(ss=9)]


def test_refusals(raw, memory):
    p = memory[0]
    for change in BOTH + [dict(act=-1), dict(act=5), dict(out=None), dict(out=p + 1), dict(out_dtype=2), dict(out_dtype=0, out=p + 2),
                          dict(bias=p + 1), dict(residual=p + 1), dict(rs=9), dict(os=9)]:
        assert _layer(raw, p, **change) == -1, change
    for change in BOTH + [dict(g=None), dict(g=p + 1), dict(g_dtype=2), dict(g_dtype=0, g=p + 2), dict(gs=9), dict(gh=None, gw=None, gb=None),
                          dict(gh=p + 1), dict(gw=p + 1), dict(gb=p + 1), dict(ghs=7), dict(gws=7)]:
        assert _grad(raw, p, **change) == -1, change
    for call in (_layer, _grad):
        for change in (dict(work=None), dict(work=p + 16), dict(size=64)):
            assert call(raw, p, N=70, **change) == -2, change
        for change in (dict(N=(1 << 21) + 1), dict(ws=1 << 22), dict(D=1 << 22, hs=1 << 22, ws=1 << 22),
                       dict(M=1 << 22, rs=1 << 22, os=1 << 22, ss=1 << 22, gs=1 << 22)):
            change = {k: v for k, v in change.items() if k not in (("gs",) if call is _layer else ("rs", "os"))}
            assert call(raw, p, **change) == -5, change
    assert _layer(raw, p, N=0, hidden=None, out=None) == 0
    assert _grad(raw, p, N=0, hidden=None, g=None, gw=None, gb=None) == 0


def test_results_in_the_place_of_inputs(raw, memory):
    p = memory[0]
    apart = dict(hidden=p, weight=p + 256, bias=p + 512, residual=p + 768, out=p + 1024, slope=p + 1280)
    for change in (dict(out=p), dict(out=p + 256), dict(out=p + 512), dict(slope=p), dict(slope=p + 768), dict(slope=p + 1024),
                   dict(out=p + 768, os=12), dict(out=p + 768, out_dtype=0)):
        assert _layer(raw, p, **{**apart, **change}) == -1, change
    apart = dict(hidden=p, weight=p + 256, g=p + 512, slope=p + 768, gh=p + 1024, gw=p + 1280, gb=p + 1536)
    for change in (dict(gh=p), dict(gh=p + 512), dict(gw=p + 256), dict(gw=p), dict(gw=p + 512), dict(gb=p + 768), dict(gh=p + 1280),
                   dict(gb=p + 1024)):
        assert _grad(raw, p, **{**apart, **change}) == -1, change


def test_workspace_queries(raw):
    q, g = raw.cfgzip_head_layer_workspace_bytes, raw.cfgzip_head_layer_grad_workspace_bytes
    for f in (q, g):
        assert f(0, 8, 8) == 0 and f(8, 0, 8) == 0 and f(8, 8, 0) == 0 and f(8, 1 << 22, 8) == 0 and f((1 << 21) + 1, 8, 8) == 0
    assert q(1, 4096, 4096) == 0 and q(32, 4096, 4096) == 0 and q(65, 100, 100) >= 65 * 128 * 2
    # dz, hidden states in whole units, columns' sums; never the weights
    assert 4096 * (16384 + 4096) * 2 <= g(4096, 16384, 4096) < 4096 * (16384 + 4096) * 2 + (8 << 20)


def test_binding_refuses_cpu_tensors():
    import paper_2605_29986_amd as lib
    w = torch.zeros((4, 8), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        lib.cfgzip_head_layer(w, w)
    with pytest.raises(TypeError):
        lib.cfgzip_head_layer_grad(w, w, w[:, :4])


# ---------------------------------------------------------------- the reference


@pytest.mark.parametrize("name", ACTIVATIONS)
def test_reference_activations(name):
    z = torch.linspace(-9.0, 9.0, 4001, dtype=torch.float64) + 1e-4
    y, s = activation(name, z)
    torch_forms = {None: lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu,
                   "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}
    assert torch.allclose(y, torch_forms[name](z), rtol=1e-9, atol=1e-14)
    e = 1e-6
    assert torch.allclose(s, (activation(name, z + e)[0] - activation(name, z - e)[0]) / (2 * e), rtol=1e-6, atol=1e-8)
    assert float(s.abs().max()) < 1.13 and float((activation(name, z + e)[1] - s).abs().max()) / e < 0.85 or name == "relu"


@pytest.mark.parametrize("name", ACTIVATIONS)
def test_reference_gradients_against_differences(name):
    gen = torch.Generator().manual_seed(0)
    x, w, b, r, g = (torch.randn(s, generator=gen, dtype=torch.float64) for s in ((5, 7), (6, 7), (6,), (5, 6), (5, 6)))
    slope = forward(x, w, b, name, r, "f32")[2]
    got = gradients(x, w, g, slope, "f16", False)

    def total(*a):
        return float((forward(*a, name, r, "f32")[0] * g).sum())

    e = 1e-6
    for which, key in ((0, "grad_hidden"), (1, "grad_weight"), (2, "grad_bias")):
        for at in (0, 3, 5):
            args = [[x.clone(), w.clone(), b.clone()] for _ in range(2)]
            args[0][which].view(-1)[at] += e
            args[1][which].view(-1)[at] -= e
            slope_here = (total(*args[0]) - total(*args[1])) / (2 * e)
            assert abs(slope_here - float(got[key][0].reshape(-1)[at])) < 1e-6, (key, at)
