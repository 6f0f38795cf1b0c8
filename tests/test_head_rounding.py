"""The bounds of tests/head_rounding.py against emulated kernels, without a GPU: each form of dz that cfgzip_head_loss_grad keeps passes,
and one with fewer bits does not."""

import numpy as np
import pytest

from head_rounding import few_rows, gradients

torch = pytest.importorskip("torch")

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def _round(x, dtype):
    return torch.from_numpy(x).to(TYPES[dtype]).double().numpy()


def _case(N, V, D, dtype, seed):
    rng = np.random.default_rng(seed)
    h = _round(rng.standard_normal((N, D)), dtype)
    w = _round(rng.standard_normal((V, D)) * (2.0 / np.sqrt(D)), dtype)
    target = rng.integers(0, V, size=N)
    g = rng.standard_normal(N).astype(np.float32).astype(np.float64) / N
    z = h @ w.T
    most = z.max(1)
    lse = (most + np.log(np.exp(z - most[:, None]).sum(1))).astype(np.float32).astype(np.float64)
    dz = np.exp(z - lse[:, None])
    dz[np.arange(N), target] -= 1.0
    return h, w, target, g, lse, dz


def _worst(r, gh, gw, dtype):
    return max(float(np.max(np.abs(_round(got, dtype) - r[name]) / r[name + "_err"])) for name, got in (("grad_hidden", gh), ("grad_weight", gw)))


SIZES = [(17, 257, 72), (129, 300, 40), (256, 1000, 128), (300, 4000, 33), (300, 1000, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("N,V,D", SIZES)
def test_the_forms_pass(N, V, D, dtype):
    h, w, target, g, lse, dz = _case(N, V, D, dtype, N + V)
    few = few_rows(N, D, dtype)
    r = gradients(h, w, target, np.ones((N, V), bool), g, lse, dtype, few)
    e = np.floor(np.log2(np.abs(g)))[:, None]
    digits = g[:, None] / 2.0 ** e
    if few and dtype == "bf16":
        x = dz * g[:, None]
        hi = _round(x, "bf16")
        kept = hi + _round(x - hi, "bf16")
        gh, gw = kept @ w, kept.T @ h
    elif few:
        x = dz * digits * 2.0 ** 14
        hi = _round(x, "f16")
        kept = (hi + _round(x - hi, "f16")) * 2.0 ** (e - 14)
        gh, gw = kept @ w, kept.T @ h
    else:
        common = np.abs(digits[np.argmax(np.abs(g))])
        x = dz * digits / common * 2.0 ** 14
        kept = _round(x, "f16")
        if dtype == "f16":  # of the target's element nothing is lost
            kept[np.arange(N), target] = x[np.arange(N), target]
        top = 14 - np.max(np.floor(np.log2(np.abs(h))) + e)
        h16 = _round(h * 2.0 ** (e + top), "f16") * 2.0 ** -top
        gh, gw = (kept @ w) * common * 2.0 ** (e - 14), kept.T @ h16 * common * 2.0 ** -14
    assert _worst(r, gh, gw, dtype) < 1.0


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("N,V,D", SIZES)
def test_dz_in_one_bf16_number_does_not(N, V, D, dtype):
    h, w, target, g, lse, dz = _case(N, V, D, dtype, N + V)
    r = gradients(h, w, target, np.ones((N, V), bool), g, lse, dtype, few_rows(N, D, dtype))
    kept = _round(dz * g[:, None], "bf16")
    assert _worst(r, kept @ w, kept.T @ h, dtype) > 1.0


@pytest.mark.parametrize("N,V,D", [s for s in SIZES if s[0] <= 256])
def test_few_fp16_rows_in_one_number_do_not(N, V, D):
    h, w, target, g, lse, dz = _case(N, V, D, "f16", N + V)
    r = gradients(h, w, target, np.ones((N, V), bool), g, lse, "f16", True)
    kept = _round(dz * g[:, None] / np.abs(g).max() * 2.0 ** 14, "f16") * np.abs(g).max() * 2.0 ** -14
    assert _worst(r, kept @ w, kept.T @ h, "f16") > 1.0


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_one_factor_for_all_rows_does_not(dtype):
    """Rows with 1e-7 of the largest gradient lose their probabilities in fp16"""
    N, V, D = 300, 20_000, 16
    h, w, target, g, lse, dz = _case(N, V, D, dtype, 5)
    w = w + 0.25
    w = _round(w, dtype)
    z = h @ w.T
    most = z.max(1)
    lse = most + np.log(np.exp(z - most[:, None]).sum(1))
    dz = np.exp(z - lse[:, None])
    dz[np.arange(N), target] -= 1.0
    g = np.where(np.arange(N) % 2, 4096.0, 4096e-7)
    r = gradients(h, w, target, np.ones((N, V), bool), g, lse, dtype, False)
    kept = _round(dz * g[:, None] * 4, "f16") / 4
    assert _worst(r, kept @ w, kept.T @ h, dtype) > 1.0


@pytest.mark.parametrize("N,V,D", [s for s in SIZES if s[0] > 256])
def test_many_fp16_rows_without_the_targets_rest_do_not(N, V, D):
    h, w, target, g, lse, dz = _case(N, V, D, "f16", N + V)
    h, target = _round(h * 0.02, "f16"), np.arange(N) % V  # flat probabilities: the target's element is all that counts
    z = h @ w.T
    lse = np.log(np.exp(z).sum(1))
    dz = np.exp(z - lse[:, None])
    dz[np.arange(N), target] -= 1.0
    g = g * 4096
    r = gradients(h, w, target, np.ones((N, V), bool), g, lse, "f16", False)
    most = np.abs(g).max()
    x = dz * g[:, None] / most * 2.0 ** 14
    whole = _round(x, "f16")
    gh, gw = whole @ w * most * 2.0 ** -14, whole.T @ h * most * 2.0 ** -14
    assert _worst(r, gh, gw, "f16") > 1.0
    whole[np.arange(N), target] = x[np.arange(N), target]
    gh, gw = whole @ w * most * 2.0 ** -14, whole.T @ h * most * 2.0 ** -14
    assert _worst(r, gh, gw, "f16") < 1.0
