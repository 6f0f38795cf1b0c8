"""Values in 4 bits and logits from them: cfgzip_mx4_quantize and cfgzip_mx4_values bit for bit, cfgzip_mx4_logits against the
definition in 64 bits within the bound of an fp32 sum, masked places exactly."""

import numpy as np
import pytest

from head_reference import F32, HALF_STEP, pack, quantize, values

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(scope="module")
def lib():
    import paper_2605_29986_amd as p
    p.load_library()
    return p


def _check_quantize(lib, x):
    """x: a 2-D GPU tensor, any row stride"""
    K = x.shape[1]
    want_c, want_s = quantize(x.double().cpu().numpy())
    codes, scales = lib.cfgzip_mx4_quantize(x)
    assert (scales.cpu().numpy() == want_s).all(), "scales"
    assert (codes.cpu().numpy() == want_c).all(), "codes"
    want = torch.from_numpy(values(want_c, want_s, K))
    for T in TYPES.values():
        got = lib.cfgzip_mx4_values(codes, scales, K, dtype=T).cpu()
        assert torch.equal(torch.nan_to_num(got.double(), nan=123.0), torch.nan_to_num(want.to(T).double(), nan=123.0)), T
        assert (got.isnan() == want.isnan()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("R,K", [(1, 1), (1, 32), (3, 31), (5, 33), (7, 64), (2, 255), (64, 96), (33, 1000), (9, 2049), (1, 5000), (700, 40)])
def test_quantize(lib, R, K, dtype):
    print(f"case R={R} K={K} {dtype}", flush=True)
    rng = np.random.default_rng(R * 31 + K)
    x = rng.standard_normal((R, K)) * 2.0 ** rng.integers(-10, 10, size=(R, 1))
    x[rng.random((R, K)) < 0.1] = 0.0
    if R > 2:
        x[1] = 0.0
    _check_quantize(lib, torch.from_numpy(x).to(TYPES[dtype]).cuda())


def test_quantize_every_pattern_of_16_bits(lib):
    """Every bf16 and every fp16 number, as a block's largest and next to a larger one: ties, subnormals, infinities, NaN."""
    every = np.arange(65536, dtype=np.uint16)
    for T in (torch.bfloat16, torch.float16):
        x = torch.from_numpy(every.copy()).view(T)
        _check_quantize(lib, x.view(2048, 32).cuda())
        one = torch.zeros((65536, 32), dtype=T)
        one[:, 7] = x
        _check_quantize(lib, one.cuda())
        order = torch.from_numpy(np.random.default_rng(1).permutation(65536))
        _check_quantize(lib, x[order].view(1024, 64).cuda())


def test_quantize_ties_and_ends_of_the_range(lib):
    steps = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.99])
    near = np.concatenate([steps, np.nextafter(steps.astype(np.float32), 0, dtype=np.float32),
                           np.nextafter(steps.astype(np.float32), 99, dtype=np.float32)]).astype(np.float64)
    rows = []
    for e in (-149, -140, -130, -127, -126, -125, -124, -10, 0, 100, 120, 124, 125):
        block = np.zeros(64)
        block[:30], block[32:62] = near, -near
        block[31], block[63] = 4.0, -7.0
        rows.append(np.ldexp(block, e).astype(np.float32))
    rows.append(np.float32([np.inf] + [1.0] * 31 + [np.nan] + [2.0] * 31))
    _check_quantize(lib, torch.from_numpy(np.stack(rows)).cuda())
    bits = np.random.default_rng(5).integers(0, 2**32, size=(500, 96), dtype=np.uint64).astype(np.uint32).view(np.float32)
    _check_quantize(lib, torch.from_numpy(bits.copy()).cuda())


def test_quantize_strides_and_given_outputs(lib):
    x = torch.randn((37, 205), device="cuda")
    for T in TYPES.values():
        _check_quantize(lib, x.to(T)[:, 3:104])
    codes, scales = lib.cfgzip_mx4_quantize(x)
    c = torch.full((39, codes.shape[1]), 0xAB, dtype=torch.uint8, device="cuda")
    s = torch.full((39, scales.shape[1]), 0xCD, dtype=torch.uint8, device="cuda")
    lib.cfgzip_mx4_quantize(x, codes=c[1:38], scales=s[1:38])
    assert torch.equal(c[1:38], codes) and torch.equal(s[1:38], scales)
    assert (c[0] == 0xAB).all() and (c[38] == 0xAB).all() and (s[0] == 0xCD).all() and (s[38] == 0xCD).all()
    wide = torch.full((37, 220), 5.0, device="cuda")
    lib.cfgzip_mx4_values(codes, scales, 205, out=wide[:, 3:208])
    assert torch.equal(wide[:, 3:208], lib.cfgzip_mx4_values(codes, scales, 205))
    assert (wide[:, :3] == 5).all() and (wide[:, 208:] == 5).all()
    c, s = lib.cfgzip_mx4_quantize(x[:0])
    assert c.shape == (0, 112) and s.shape == (0, 7) and lib.cfgzip_mx4_values(c, s, 205).shape == (0, 205)


# ---------------------------------------------------------------- logits


def _masks(rng, B, V, kind):
    from gpu_util import dev
    if kind == "none":
        return np.ones((B, V), bool), {}
    if kind == "token":
        allowed = rng.random((B, V)) < 0.5
        allowed[B // 2] = False
        return allowed, {"bits": dev(pack(allowed))}
    C = max(1, V // 3)
    c = rng.integers(0, C, size=V).astype(np.int32)
    classes = rng.random((B, C)) < 0.3
    classes[B // 2] = False
    return classes[:, c], {"bits": dev(pack(classes)), "class_of_token": dev(c), "C": C}


def _weights(rng, V, K):
    w = rng.standard_normal((V, K)) * 2.0 ** rng.integers(-6, 3, size=(V, 1))
    return quantize(w)


def _check_logits(lib, B, V, K, x_type, mask, out="f32", seed=0, pad=0, offset=0, out_pad=0):
    print(f"case B={B} V={V} K={K} x={x_type} mask={mask} out={out} pad={pad} offset={offset} out_pad={out_pad}", flush=True)
    from gpu_util import dev
    rng = np.random.default_rng(seed + B * 13 + V * 7 + K)
    codes, scales = _weights(rng, V, K)
    allowed, masks = _masks(rng, B, V, mask)
    w = values(codes, scales, K)
    dirty_c, dirty_s = codes.copy(), scales.copy()
    dirty_s[~allowed.any(0)] = 255  # weights of tokens that no row admits are NaN
    x = torch.from_numpy(rng.standard_normal((B, K)) * 2.0 ** rng.integers(-4, 4, size=(B, 1)))
    if x_type == "4":
        xc, xs = quantize(x.numpy())
        xd, args = values(xc, xs, K), {"hidden_scales": dev(xs)}
        hidden = dev(xc)
    else:
        x = x.to(TYPES[x_type])
        flat = torch.full((offset + B * (K + pad),), float("nan"), dtype=x.dtype, device="cuda")
        hidden = flat[offset:].view(B, K + pad)[:, :K]
        hidden.copy_(x)
        xd, args = x.double().numpy(), {}
    T = TYPES[out]
    buffer = torch.full((B, V + out_pad), 3.0, dtype=T, device="cuda")
    got = lib.cfgzip_mx4_logits(hidden, dev(dirty_c), dev(dirty_s), logits=buffer[:, out_pad // 2:out_pad // 2 + V], **masks, **args)
    torch.cuda.synchronize()
    if out_pad:
        left, right = buffer[:, :out_pad // 2], buffer[:, out_pad // 2 + V:]
        assert (left == 3).all() and (right == 3).all(), "columns beside the logits"
    got = got.double().cpu().numpy()
    want = xd @ w.T
    bound = (np.abs(xd) @ np.abs(w).T) * (K * (2 if x_type == "f16" else 1) + 8) * F32 + HALF_STEP[out] * np.abs(want) * 1.01
    assert (got[~allowed] == -np.inf).all(), "masked places"
    bad = allowed & ~(np.abs(got - want) <= bound)
    assert not bad.any(), (np.argwhere(bad)[:5].tolist(), got[bad][:5], want[bad][:5], bound[bad][:5])


@pytest.mark.parametrize("x_type", ["bf16", "f16", "4"])
@pytest.mark.parametrize("mask", ["none", "class", "token"])
@pytest.mark.parametrize("B,V,K", [
    (1, 1, 1), (1, 17, 33), (1, 1000, 500), (2, 15, 32), (3, 100, 64), (7, 257, 128), (8, 640, 1000), (9, 33, 2048), (12, 500, 96),
    (16, 300, 256), (17, 130, 100), (25, 200, 512), (32, 77, 160), (33, 515, 288), (64, 129, 480), (65, 300, 1001), (130, 257, 320),
    (200, 1030, 72), (300, 40, 544)])
def test_logits(lib, B, V, K, x_type, mask):
    _check_logits(lib, B, V, K, x_type, mask, out="bf16" if (B + V) % 3 == 0 else "f32")


@pytest.mark.parametrize("x_type", ["bf16", "f16", "4"])
@pytest.mark.parametrize("B", [1, 5, 16])
def test_logits_of_more_tokens_than_waves(lib, B, x_type):
    """Waves that go around several times, whole tiles of 16 tokens each"""
    _check_logits(lib, B, 140_007, 40, x_type, "class")


@pytest.mark.parametrize("x_type", ["bf16", "f16", "4"])
@pytest.mark.parametrize("B", [4, 10])
def test_logits_of_long_rows(lib, B, x_type):
    """Shares of a token's blocks in several waves; hidden states beyond what LDS holds (10 rows of 16 bits)"""
    _check_logits(lib, B, 50, 9_000, x_type, "none")


@pytest.mark.parametrize("B", [3, 20, 70])
@pytest.mark.parametrize("x_type,pad,offset,out_pad", [("bf16", 8, 0, 0), ("bf16", 5, 1, 3), ("f16", 8, 8, 8), ("f16", 1, 3, 7), ("4", 0, 0, 5)])
def test_logits_strides_and_alignment(lib, B, x_type, pad, offset, out_pad):
    for out in ("f32", "bf16"):
        _check_logits(lib, B, 203, 136, x_type, "class", out=out, pad=pad, offset=offset, out_pad=out_pad)


def test_logits_of_infinite_hidden_states(lib):
    """What is not finite stays so: infinity in fp16 is split into infinity and 0, not into infinity and NaN."""
    from gpu_util import dev
    codes, scales = quantize(np.ones((20, 64)))
    for B in (2, 40):
        for T in (torch.bfloat16, torch.float16):
            x = torch.ones((B, 64), dtype=T, device="cuda")
            x[0, 3], x[1, 5] = float("inf"), float("nan")
            z = lib.cfgzip_mx4_logits(x, dev(codes), dev(scales))
            assert (z[0] == float("inf")).all() and z[1].isnan().all() and (z[2:] == 64).all()


def test_logits_same_bits_every_time_on_any_stream_and_in_a_graph(lib):
    from gpu_util import dev
    rng = np.random.default_rng(6)
    for B, x_type in ((4, "bf16"), (40, "f16"), (100, "4")):
        codes, scales = (dev(a) for a in _weights(rng, 3000, 512))
        _, masks = _masks(rng, B, 3000, "class")
        x = torch.randn((B, 512), device="cuda")
        hidden, more = (x.to(TYPES[x_type]), {}) if x_type != "4" else (None, {})
        if x_type == "4":
            hidden, hs = lib.cfgzip_mx4_quantize(x)
            more = {"hidden_scales": hs}
        want = lib.cfgzip_mx4_logits(hidden, codes, scales, **masks, **more)
        kind = {"bf16": 1, "f16": 2, "4": 3}[x_type]
        ws = torch.full((max(256, lib.load_library().cfgzip_mx4_logits_workspace_bytes(kind, B, 3000, 512, 1)),), 255, dtype=torch.uint8,
                        device="cuda")
        out = torch.zeros_like(want)

        def step():
            lib.cfgzip_mx4_logits(hidden, codes, scales, logits=out, workspace=ws, **masks, **more)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for replay in range(3):
            out.zero_(), ws.fill_(replay)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want), (B, replay)


def test_no_rows(lib):
    codes, scales = lib.cfgzip_mx4_quantize(torch.randn((40, 64), device="cuda"))
    x = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    assert lib.cfgzip_mx4_logits(x, codes, scales).shape == (0, 40)


def test_refusals(lib):
    x = torch.randn((5, 70), device="cuda")
    codes, scales = lib.cfgzip_mx4_quantize(torch.randn((40, 70), device="cuda"))
    h = x.bfloat16()
    bits = torch.zeros((5, 2), dtype=torch.int32, device="cuda")
    for call in (lambda: lib.cfgzip_mx4_quantize(x.cpu()), lambda: lib.cfgzip_mx4_quantize(x.double()),
                 lambda: lib.cfgzip_mx4_logits(x, codes, scales), lambda: lib.cfgzip_mx4_logits(h, codes.int(), scales),
                 lambda: lib.cfgzip_mx4_logits(h, codes, scales, dtype=torch.float16)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: lib.cfgzip_mx4_quantize(x.t()), lambda: lib.cfgzip_mx4_quantize(x, codes=codes),
                 lambda: lib.cfgzip_mx4_values(codes, scales, 64), lambda: lib.cfgzip_mx4_values(codes[:3], scales, 70),
                 lambda: lib.cfgzip_mx4_logits(h[:, :64], codes, scales), lambda: lib.cfgzip_mx4_logits(h, codes, scales, bits=bits[:3]),
                 lambda: lib.cfgzip_mx4_logits(h, codes, scales, bits=bits[:, :1]),
                 lambda: lib.cfgzip_mx4_logits(h, codes, scales, logits=torch.empty((5, 41), device="cuda"))):
        with pytest.raises(ValueError):
            call()
