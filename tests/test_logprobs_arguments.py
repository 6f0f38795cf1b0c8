"""cfgzip_token_logprobs and its gradient without a GPU: what the C ABI and the binding refuse, the workspace query, and the tests' references
against themselves."""

import ctypes
import os

import numpy as np
import pytest

from logprobs_reference import gradient, logprobs


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


def _score(raw, p, **change):
    a = dict(logits=p, dtype=1, N=4, V=10, stride=10, tokens=p, n=2, temperature=1.0, bits=None, kind=2, c=None, C=0, logprob=p, entropy=p,
             stats=p, top=3, top_tokens=p, top_logprobs=p, work=p, size=1 << 20)
    a.update(change)
    return raw.cfgzip_token_logprobs(*a.values(), None)


def _grad(raw, p, **change):
    a = dict(logits=p, dtype=1, N=4, V=10, stride=10, tokens=p, n=2, temperature=1.0, bits=None, kind=2, c=None, C=0, logprob=p, stats=p, g=p,
             entropy=p, ge=p, out=p, out_stride=10)
    a.update(change)
    return raw.cfgzip_token_logprobs_grad(*a.values(), None)


BOTH = [dict(logits=None), dict(logits=1), dict(dtype=3), dict(dtype=-1), dict(N=-1), dict(V=0), dict(stride=9), dict(tokens=None),
        dict(n=-1), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")),
        dict(temperature=2.0 ** -21), dict(temperature=2.0 ** 21), dict(kind=3), dict(kind=-1), dict(kind=0), dict(kind=1, bits=256),
        dict(kind=1, bits=256, c=256, C=0), dict(kind=0, bits=258), dict(kind=1, bits=256, c=257, C=4), dict(logprob=None), dict(stats=2)]


def test_score_refuses(raw, memory):
    p = memory[0]
    for change in BOTH + [dict(logprob=p + 2), dict(entropy=p + 1), dict(top=-1), dict(top_tokens=None), dict(top_logprobs=None),
                          dict(top_tokens=p + 2), dict(top_logprobs=p + 1), dict(tokens=p + 2), dict(dtype=0, logits=p + 2)]:
        assert _score(raw, p, **change) == -1, change
    for change in (dict(top=65), dict(n=4097), dict(N=(1 << 22) + 1), dict(V=0x7FFFFFFF, stride=0x7FFFFFFF)):
        assert _score(raw, p, **change) == -5, change
    big = dict(V=100_000, stride=100_000)
    for change in (dict(work=None), dict(work=p + 16), dict(size=64)):
        assert _score(raw, p, **big, **change) == -2, change
    assert _score(raw, p, N=0, logits=None, tokens=None, logprob=None, top_tokens=None) == 0


def test_grad_refuses(raw, memory):
    p = memory[0]
    for change in BOTH + [dict(stats=None), dict(g=None), dict(g=p + 2), dict(entropy=None), dict(ge=p + 2), dict(out=None), dict(out=p + 1),
                          dict(out_stride=9), dict(out_stride=12), dict(dtype=0, out=p + 2)]:
        assert _grad(raw, p, **change) == -1, change
    for change in (dict(n=4097), dict(N=(1 << 22) + 1), dict(N=1 << 22, V=100_000, stride=100_000, out_stride=100_000)):
        assert _grad(raw, p, **change) == -5, change
    assert _grad(raw, p, N=0, logits=None, tokens=None, out=None) == 0


def test_workspace_query(raw):
    q = raw.cfgzip_token_logprobs_workspace_bytes
    assert q(0, 10, 1) == 0 and q(1, 0, 1) == 0 and q(1, 10, -1) == 0 and q(1, 100_000, 65) == 0
    assert q(1, 4096, 8) == 0 and q(600, 100_000, 64) == 0  # one workgroup to a row
    assert q(1, 32_000, 20) == 0 and q(1, 128_256, 0) >= 16 * 2 and q(1, 128_256, 20) >= q(1, 128_256, 0) + 2 * 20 * 8


def test_binding_refuses_cpu_tensors():
    torch = pytest.importorskip("torch")
    import paper_2605_29986_amd as lib
    x, t = torch.zeros((4, 8)), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(TypeError):
        lib.cfgzip_token_logprobs(x, t)
    with pytest.raises(TypeError):
        lib.cfgzip_token_logprobs_grad(x, t, x[:, 0], x[:, :2], x[:, 0])


# ---------------------------------------------------------------- the references


def test_reference_values():
    x = np.log(np.array([[1.0, 2.0, 5.0, 2.0], [1.0, 2.0, 5.0, 2.0], [1.0, 1.0, 1.0, 1.0]]))
    allowed = np.array([[1, 1, 1, 1], [1, 1, 0, 1], [0, 0, 0, 0]], bool)
    tokens = np.array([[1, -1], [2, 3], [0, 4]])
    r = logprobs(x, tokens, allowed, 1.0, 3)
    assert np.allclose(r["logprob"], [[np.log(0.2), 0.0], [-np.inf, np.log(0.4)], [-np.inf, 0.0]])
    assert r["top_tokens"].tolist() == [[2, 1, 3], [1, 3, 0], [-1, -1, -1]]
    assert np.allclose(r["entropy"], [-(0.1 * np.log(0.1) + 0.4 * np.log(0.2) + 0.5 * np.log(0.5)),
                                      -(0.2 * np.log(0.2) + 0.8 * np.log(0.4)), 0.0])
    assert np.allclose(r["stats"][:2], [[np.log(5.0), np.log(2.0)], [np.log(2.0), np.log(2.5)]]) and (r["stats"][2] == -np.inf).all()


@pytest.mark.parametrize("temperature", [1.0, 0.3])
def test_reference_gradient_against_differences(temperature):
    rng = np.random.default_rng(0)
    N, V = 4, 12
    x = rng.standard_normal((N, V))
    allowed = rng.random((N, V)) < 0.7
    x[0, 3] = -np.inf
    tokens = np.array([[0, 5, 0], [1, -1, 2], [11, 12, 3], [7, 7, 7]])
    g, ge = rng.standard_normal((N, 3)), rng.standard_normal(N)
    r = logprobs(x, tokens, allowed, temperature, 0)
    want, _ = gradient(r, tokens, g, ge, temperature, "f32")

    def total(y):
        s = logprobs(y, tokens, allowed, temperature, 0)
        return np.where(s["counts"], np.where(s["counts"], s["logprob"], 0.0) * g, 0.0).sum() + (s["entropy"] * ge).sum()

    for i in range(N):
        for v in range(V):
            up, down = x.copy(), x.copy()
            up[i, v] += 1e-5
            down[i, v] -= 1e-5
            assert abs((total(up) - total(down)) / 2e-5 - want[i, v]) < 1e-7, (i, v)
