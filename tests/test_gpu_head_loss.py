"""cfgzip_head_loss and cfgzip_head_loss_grad against their definition in 64 bits, at the sizes, masks, strides and targets where
they can go wrong, with the error bounds of tests/head_reference.py."""

import numpy as np
import pytest

from head_reference import loss_and_gradients, pack
from synthetic_inputs.configs import words_for

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def lib():
    import paper_2605_29986_amd as p
    p.load_library()
    return p


def _masks(rng, N, V, kind):
    """(bool [N][V], arguments of a call); the second row admits nothing, pad bits are set"""
    from gpu_util import dev
    if kind == "none":
        return np.ones((N, V), bool), {}
    share = 2.0 ** -rng.uniform(0, 4, size=(N, 1))
    if kind == "token":
        allowed = rng.random((N, V)) < share
        if N > 1:
            allowed[1] = False
        return allowed, {"bits": dev(pack(allowed))}
    C = max(1, V // 3)
    c = rng.integers(0, C, size=V).astype(np.int32)
    classes = rng.random((N, C)) < share
    if N > 1:
        classes[1] = False
    return classes[:, c], {"bits": dev(pack(classes)), "class_of_token": dev(c), "C": C}


def _placed(x, stride, offset):
    """x as a view `offset` elements into an allocation, rows `stride` apart; what lies between is NaN"""
    R, n = x.shape
    flat = torch.full((offset + R * stride,), float("nan"), dtype=x.dtype, device="cuda")
    view = flat[offset:].view(R, stride)[:, :n]
    view.copy_(x)
    return view


def _close(got, want, err, name):
    got = got.double().cpu().numpy()
    same = np.isnan(want) & np.isnan(got) | (~np.isfinite(want) & (got == want))
    off = np.abs(got - np.where(np.isfinite(want), want, 0.0)) <= err
    good = np.where(np.isfinite(want), off, same)
    assert good.all(), (name, np.argwhere(~good)[:5].tolist(), got[~good][:5], want[~good][:5],
                        np.broadcast_to(err, want.shape)[~good][:5])


def _check(lib, N, V, D, dtype, mask, seed, pad=0, offset=0, w_pad=0):
    print(f"case N={N} V={V} D={D} {dtype} mask={mask} pad={pad} offset={offset} w_pad={w_pad}", flush=True)
    from gpu_util import dev
    rng = np.random.default_rng(seed)
    T = TYPES[dtype]
    allowed, masks = _masks(rng, N, V, mask)
    w = torch.from_numpy(rng.standard_normal((V, D)) * (2.0 / np.sqrt(D))).to(T)
    h = torch.from_numpy(rng.standard_normal((N, D))).to(T)
    target = rng.integers(0, V, size=N)
    for i in range(N):  # mostly tokens that the row admits
        k = np.flatnonzero(allowed[i])
        if len(k) and i % 5:
            target[i] = rng.choice(k)
    h[np.arange(N) % 3 == 0] += 3.0 * w[torch.from_numpy(target)][np.arange(N) % 3 == 0]  # a certain target here and there
    if N > 4:
        target[2], target[3], target[4] = -1, V, -2**31
        h[2] = float("nan")  # a padded position
    grad = rng.standard_normal(N) / N
    if N > 5:
        grad[5] = 0.0
    grad = grad.astype(np.float32)
    hidden, weight = _placed(h, D + pad, offset), _placed(w, D + w_pad, offset)
    t = dev(target.astype(np.int32))
    loss, lse = lib.cfgzip_head_loss(hidden, weight, t, **masks)
    gh, gw = lib.cfgzip_head_loss_grad(hidden, weight, t, lse, dev(grad), **masks)
    torch.cuda.synchronize()
    r = loss_and_gradients(h.double().numpy(), w.double().numpy(), target, allowed, grad.astype(np.float64), dtype)
    for name, got in (("lse", lse), ("loss", loss), ("grad_hidden", gh), ("grad_weight", gw)):
        _close(got, r[name], r[name + "_err"], name)
    return hidden, weight, t, lse, dev(grad), masks, gh, gw


SIZES = [(1, 1, 1), (1, 5, 8), (2, 31, 7), (3, 33, 40), (16, 100, 64), (17, 257, 72), (40, 130, 128), (64, 300, 136), (65, 1000, 200),
         (130, 515, 96), (257, 700, 264), (300, 2048, 65), (20, 3000, 1001), (500, 40, 520), (6, 9000, 328), (129, 5678, 72), (128, 2100, 80)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("mask", ["none", "class", "token"])
@pytest.mark.parametrize("N,V,D", SIZES)
def test_sizes_and_masks(lib, N, V, D, mask, dtype):
    _check(lib, N, V, D, dtype, mask, seed=N * 7 + V + D)


@pytest.mark.parametrize("N", [5, 40, 100, 200])
@pytest.mark.parametrize("pad,offset,w_pad", [(8, 0, 0), (24, 8, 8), (3, 1, 0), (0, 0, 5), (1, 3, 7)])
def test_strides_and_alignment(lib, N, pad, offset, w_pad):
    _check(lib, N, 600, 88, "bf16", "class", seed=3, pad=pad, offset=offset, w_pad=w_pad)


def test_one_gradient_at_a_time_and_given_outputs(lib):
    hidden, weight, t, lse, grad, masks, gh, gw = _check(lib, 70, 900, 104, "f16", "class", seed=5)
    a, none = lib.cfgzip_head_loss_grad(hidden, weight, t, lse, grad, want_weight=False, **masks)
    assert none is None and torch.equal(a, gh)
    none, b = lib.cfgzip_head_loss_grad(hidden, weight, t, lse, grad, want_hidden=False, **masks)
    assert none is None and torch.equal(b, gw)
    wide_h = torch.full((70, 111), 7.0, dtype=gh.dtype, device="cuda")
    wide_w = torch.full((900, 105), 7.0, dtype=gw.dtype, device="cuda")
    lib.cfgzip_head_loss_grad(hidden, weight, t, lse, grad, grad_hidden=wide_h[:, 3:107], grad_weight=wide_w[:, 1:], **masks)
    assert torch.equal(wide_h[:, 3:107], gh) and torch.equal(wide_w[:, 1:], gw)
    assert (wide_h[:, :3] == 7).all() and (wide_h[:, 107:] == 7).all() and (wide_w[:, 0] == 7).all()


def test_masked_weights_may_hold_anything_in_the_loss(lib):
    """Rows of weights that no row admits: logits of infinity and NaN, which do not count."""
    from gpu_util import dev
    rng = np.random.default_rng(11)
    N, V, D = 9, 200, 64
    h, w = rng.standard_normal((N, D)).astype(np.float32), rng.standard_normal((V, D)).astype(np.float32) * 0.2
    allowed = rng.random((N, V)) < 0.5
    allowed[:, 150:] = False
    target = np.array([rng.choice(np.flatnonzero(a)) for a in allowed])
    hb, wb = torch.from_numpy(h).bfloat16(), torch.from_numpy(w).bfloat16()
    dirty = wb.clone()
    dirty[150:160], dirty[160:170], dirty[170:] = float("inf"), float("nan"), 3e38
    args = (dev(target.astype(np.int32)),)
    loss, lse = lib.cfgzip_head_loss(hb.cuda(), dirty.cuda(), *args, bits=dev(pack(allowed)))
    r = loss_and_gradients(hb.double().numpy(), wb.double().numpy(), target, allowed, None, "bf16")
    _close(lse, r["lse"], r["lse_err"], "lse")
    _close(loss, r["loss"], r["loss_err"], "loss")


@pytest.mark.parametrize("scale", [1e-30, 1e-6, 1.0, 1e20])
def test_size_of_the_upstream_gradient(lib, scale):
    """bf16 gradients follow grad_loss over its whole range: they are scaled by powers of two on the way."""
    from gpu_util import dev
    rng = np.random.default_rng(2)
    N, V, D = 33, 400, 64
    h = torch.from_numpy(rng.standard_normal((N, D))).bfloat16()
    w = torch.from_numpy(rng.standard_normal((V, D)) * 0.2).bfloat16()
    t = dev(rng.integers(0, V, size=N).astype(np.int32))
    g = rng.standard_normal(N).astype(np.float32)
    _, lse = lib.cfgzip_head_loss(h.cuda(), w.cuda(), t)
    grad = (g.astype(np.float64) * scale).astype(np.float32)
    gh, gw = lib.cfgzip_head_loss_grad(h.cuda(), w.cuda(), t, lse, dev(grad))
    r = loss_and_gradients(h.double().numpy(), w.double().numpy(), t.cpu().numpy(), np.ones((N, V), bool), grad.astype(np.float64), "bf16")
    _close(gh, r["grad_hidden"], r["grad_hidden_err"], "grad_hidden")
    _close(gw, r["grad_weight"], r["grad_weight_err"], "grad_weight")


def test_several_pieces_of_the_vocabulary(lib):
    """More dz than is kept at a time: pieces, the last of them ragged, sums carried from piece to piece.  The reference is in 64 bits on
    the GPU; the bound is the tests' own with the logits' errors left out, which are below a thousandth of a step here."""
    N, V, D = 2_500, 131_073, 64
    gen = torch.Generator(device="cuda").manual_seed(4)
    h = torch.randn((N, D), device="cuda", generator=gen).bfloat16()
    w = (torch.randn((V, D), device="cuda", generator=gen) * 0.2).bfloat16()
    t = torch.randint(0, V, (N,), device="cuda", generator=gen).int()
    g = torch.randn((N,), device="cuda", generator=gen)
    loss, lse = lib.cfgzip_head_loss(h, w, t)
    gh, gw = lib.cfgzip_head_loss_grad(h, w, t, lse, g)
    hd, wd = h.double(), w.double()
    zt = (hd * wd[t.long()]).sum(1)
    parts = torch.stack([torch.logsumexp(hd @ wd[v:v + 16384].t(), 1) for v in range(0, V, 16384)])
    want = parts.logsumexp(0)
    assert ((lse - want).abs() < 1e-5 * (1 + want.abs())).all() and ((loss - (want - zt)).abs() < 1e-4).all()
    wgh, egh = torch.zeros_like(hd), torch.zeros_like(hd)
    for v in range(0, V, 16384):
        n = min(16384, V - v)
        dz = torch.exp(hd @ wd[v:v + n].t() - want[:, None])
        here = torch.nonzero((t >= v) & (t < v + n))[:, 0]
        dz[here, t[here].long() - v] -= 1.0
        dz *= g.double()[:, None]
        wgh += dz @ wd[v:v + n]
        egh += dz.abs() @ wd[v:v + n].abs()
        wgw, egw = dz.t() @ hd, dz.abs().t() @ hd.abs()
        bound = egw * (2.0 ** -8 * 1.02 + (N + 64) * 2.0 ** -24) + wgw.abs() * 2.0 ** -8 * 1.01 + 1e-30
        assert ((gw[v:v + n].double() - wgw).abs() <= bound).all(), v
    bound = egh * (2.0 ** -8 * 1.02 + (V + 64) * 2.0 ** -24) + wgh.abs() * 2.0 ** -8 * 1.01 + 1e-30
    assert ((gh.double() - wgh).abs() <= bound).all()


def test_gradient_against_differences(lib):
    """Along a direction of hidden states and one of weights, the gradient is the slope of the loss in 64 bits."""
    from gpu_util import dev
    rng = np.random.default_rng(8)
    N, V, D = 24, 500, 48
    allowed, masks = _masks(rng, N, V, "class")
    h = torch.from_numpy(rng.standard_normal((N, D))).half()
    w = torch.from_numpy(rng.standard_normal((V, D)) * 0.3).half()
    target = np.array([rng.choice(np.flatnonzero(a)) if a.any() else -1 for a in allowed])
    g = rng.standard_normal(N).astype(np.float32)
    t = dev(target.astype(np.int32))
    _, lse = lib.cfgzip_head_loss(h.cuda(), w.cuda(), t, **masks)
    gh, gw = lib.cfgzip_head_loss_grad(h.cuda(), w.cuda(), t, lse, dev(g), **masks)
    hd, wd = h.double().numpy(), w.double().numpy()
    dh, dw = rng.standard_normal((N, D)), rng.standard_normal((V, D))

    def total(a, b):
        r = loss_and_gradients(hd + a * dh, wd + b * dw, target, allowed, None, "f16")["loss"]
        return float((np.where(target >= 0, r, 0.0) * g).sum())

    r = loss_and_gradients(hd, wd, target, allowed, g.astype(np.float64), "f16")
    e = 2.0 ** -17  # the third derivative's part, e^2 / 6 of it, and 2^-52 / e of the loss are far below the kernel's roundings
    for got, want, err, d in ((gh, total(e, 0) - total(-e, 0), r["grad_hidden_err"], dh),
                              (gw, total(0, e) - total(0, -e), r["grad_weight_err"], dw)):
        slope = float((got.double().cpu().numpy() * d).sum())
        assert abs(slope - want / (2 * e)) <= (err * np.abs(d)).sum() + 1e-6


def test_same_bits_every_time_on_any_stream_and_in_a_graph(lib):
    hidden, weight, t, lse, grad, masks, gh, gw = _check(lib, 200, 1500, 256, "bf16", "class", seed=21)
    loss, _ = lib.cfgzip_head_loss(hidden, weight, t, **masks)
    raw = lib.load_library()
    ws1 = torch.empty(raw.cfgzip_head_loss_workspace_bytes(200, 1500, 256, 1), dtype=torch.uint8, device="cuda")
    ws2 = torch.empty(raw.cfgzip_head_loss_grad_workspace_bytes(200, 1500, 256, 1), dtype=torch.uint8, device="cuda")
    out = [torch.empty_like(loss), torch.empty_like(lse), torch.empty_like(gh), torch.empty_like(gw)]

    def step():
        lib.cfgzip_head_loss(hidden, weight, t, loss=out[0], lse=out[1], workspace=ws1, **masks)
        lib.cfgzip_head_loss_grad(hidden, weight, t, out[1], grad, grad_hidden=out[2], grad_weight=out[3], workspace=ws2, **masks)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ws1.fill_(0xFF), ws2.fill_(0xFF)
        step()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(out, (loss, lse, gh, gw)):  # bits: there is a NaN among the lse
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for replay in range(3):
        print(f"replay {replay}", flush=True)
        for a in out:
            a.zero_()
        ws1.fill_(replay * 37), ws2.fill_(255 - replay)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, (loss, lse, gh, gw)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), replay


def test_no_rows(lib):
    w = torch.randn((50, 24), device="cuda").bfloat16()
    h, t, f = w[:0], torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    loss, lse = lib.cfgzip_head_loss(h, w, t)
    assert loss.numel() == 0 and lse.numel() == 0
    gh, gw = lib.cfgzip_head_loss_grad(h, w, t, f, f)
    assert gh.shape == (0, 24) and gw.shape == (50, 24) and (gw == 0).all()


def test_refusals(lib):
    w = torch.randn((50, 24), device="cuda").bfloat16()
    h, t = w[:5].clone(), torch.zeros(5, dtype=torch.int32, device="cuda")
    bits = torch.zeros((5, words_for(50)), dtype=torch.int32, device="cuda")
    f = torch.zeros(5, device="cuda")
    for bad in ((h.half(), w, t), (h.float(), w.float(), t), (h.cpu(), w, t), (h, w, t.long())):
        with pytest.raises(TypeError):
            lib.cfgzip_head_loss(*bad)
    for bad, more in (((h[:, :20], w, t), {}), ((h, w, t[:4]), {}), ((h.t(), w, t), {}), ((h, w[:, ::2], t), {}),
                      ((h, w, t), {"bits": bits[:, :1]}), ((h, w, t), {"bits": bits[:4]}), ((h, w, t), {"C": 4}),
                      ((h, w, t), {"bits": bits, "class_of_token": t, "C": 50}), ((h, w, t), {"loss": f[:3]}),
                      ((h[:1].expand(5, 24), w, t), {})):
        with pytest.raises(ValueError):
            lib.cfgzip_head_loss(*bad, **more)
    with pytest.raises(lib.CfgzipError):
        lib.cfgzip_head_loss(h, w, t, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        lib.cfgzip_head_loss_grad(h, w, t, f, f, want_hidden=False, want_weight=False)
    with pytest.raises(ValueError):
        lib.cfgzip_head_loss_grad(h, w, t, f, f[:2])
    with pytest.raises(TypeError):
        lib.cfgzip_head_loss_grad(h, w, t, f, f.double())
