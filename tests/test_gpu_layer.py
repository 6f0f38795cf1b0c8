"""cfgzip_head_layer and cfgzip_head_layer_grad against their definition in 64 bits."""

import pytest

torch = pytest.importorskip("torch")

from layer_reference import ACTIVATIONS, forward, gradients, slopes

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(scope="module")
def lib():
    import paper_2605_29986_amd as cz
    return cz


def rows(gen, n, columns, dtype, offset=0, gap=0, size=1.0):
    """A slice of a wider tensor, NaN around it"""
    wide = torch.full((n, columns + offset + gap), float("nan"), dtype=dtype, device="cuda")
    wide[:, offset:offset + columns] = torch.randn((n, columns), device="cuda", generator=gen) * size
    return wide[:, offset:offset + columns]


def make(seed, N, M, D, dtype, bias=True, residual=True, offset=0, gap=0, w_offset=0, w_gap=0, size=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    T = TYPES[dtype]
    s = {"x": rows(gen, N, D, T, offset, gap), "w": rows(gen, M, D, T, w_offset, w_gap, 1.5 / D ** 0.5),
         "b": torch.randn(M, device="cuda", generator=gen).to(T) if bias else None,
         "r": rows(gen, N, M, T, offset, gap) if residual else None, "g": rows(gen, N, M, T, gap, offset, size)}
    return s


def within(got, want, err, what):
    # (what rounds to more than fp16's largest number, 65504 and half a step of 32, is infinite there)
    beyond = got.isinf() & ((got.dtype == torch.float16) & (got.sign().double() * want + err >= 65520.0))
    got = got.double()
    bad = ~((got == want) | ((got - want).abs() <= err) | beyond)
    assert not bool(bad.any()), (what, torch.nonzero(bad)[:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist(), err[bad][:4].tolist())


def double(t):
    return None if t is None else t.double()


def check(lib, s, dtype, name, f32=False, g=None):
    out, slope = lib.cfgzip_head_layer(s["x"], s["w"], s["b"], activation=name, residual=s["r"], want_slope=True,
                                       dtype=torch.float32 if f32 else None)
    y, y_err, sl, sl_err = forward(s["x"].double(), s["w"].double(), double(s["b"]), name, double(s["r"]), "f32" if f32 else dtype)
    assert out.dtype == TYPES["f32" if f32 else dtype] and slope.dtype == torch.int16
    within(out, y, y_err, "out")
    within(slopes(slope), sl, sl_err, "slope")
    g = s["g"] if g is None else g
    slope = None if name is None else slope
    got = lib.cfgzip_head_layer_grad(s["x"], s["w"], g, slope=slope, want_bias=True)
    exact = name is None and g.dtype == TYPES[dtype] and dtype == "bf16"
    want = gradients(s["x"].double(), s["w"].double(), g.double(), None if slope is None else slopes(slope), dtype, exact)
    for t, key in zip(got, ("grad_hidden", "grad_weight", "grad_bias")):
        assert t.dtype == TYPES[dtype]
        within(t, *want[key], key)
    return out, got


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("N", [1, 2, 15, 16, 17, 33, 64, 65, 129, 300])
@pytest.mark.parametrize("M,D", [(1, 1), (8, 64), (7, 72), (129, 100), (64, 63), (500, 256), (1001, 1000), (96, 2048)])
def test_sizes(lib, N, M, D, dtype):
    print(f"case N={N} M={M} D={D} {dtype}", flush=True)
    check(lib, make(N + M + D, N, M, D, dtype), dtype, ACTIVATIONS[(N + M + D) % 5])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("name", ACTIVATIONS)
@pytest.mark.parametrize("N", [5, 200])
def test_activations(lib, N, name, dtype):
    print(f"case N={N} {name} {dtype}", flush=True)
    for bias, residual, f32 in ((True, True, False), (True, False, True), (False, True, True), (False, False, False)):
        check(lib, make(N, N, 320, 192, dtype, bias=bias, residual=residual), dtype, name, f32=f32)


@pytest.mark.parametrize("name", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("size", [8.0, 60.0])
def test_large_arguments(lib, name, size):
    """Activations' tails"""
    s = make(1, 100, 256, 128, "bf16")
    s["w"].mul_(size)
    check(lib, s, "bf16", name, f32=True)


@pytest.mark.parametrize("N", [5, 200])
@pytest.mark.parametrize("name", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("size", [1e5, 1e12, 1e17])
def test_arguments_whose_squares_are_no_numbers(lib, size, name, N):
    """z of 1e10 to 1e34: z or 0, with slopes of 1 or 0"""
    s = make(17, N, 72, 24, "bf16", bias=False, residual=False)
    s["x"].mul_(size)
    s["w"].mul_(size)
    out, slope = lib.cfgzip_head_layer(s["x"], s["w"], activation=name, want_slope=True)
    z, z_err = forward(s["x"].double(), s["w"].double(), None, None, None, "bf16")[:2]
    assert float(z.abs().min()) > 1e3
    within(out, z.clamp(min=0.0), z_err, "out")
    assert (slope == torch.where(z > 0, 1 << 14, 0)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("N", [7, 150])
@pytest.mark.parametrize("offset,gap,w_offset,w_gap", [(0, 8, 0, 8), (1, 0, 0, 0), (0, 3, 1, 0), (8, 8, 4, 4), (3, 6, 3, 2), (0, 0, 0, 5)])
def test_rows_anywhere(lib, N, offset, gap, w_offset, w_gap, dtype):
    print(f"case N={N} {offset} {gap} {w_offset} {w_gap} {dtype}", flush=True)
    for M, D in ((328, 192), (333, 250)):
        check(lib, make(2, N, M, D, dtype, offset=offset, gap=gap, w_offset=w_offset, w_gap=w_gap), dtype, "silu")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("N,M,D", [(2000, 2048, 512), (2048, 8200, 128), (4096, 8192, 64), (700, 128, 8192), (64, 16384, 512)])
def test_many_tiles(lib, N, M, D, dtype):
    """All sizes of tiles, workgroups that make more than one, sums that are split"""
    print(f"case N={N} M={M} D={D} {dtype}", flush=True)
    check(lib, make(3, N, M, D, dtype), dtype, "gelu_tanh")
    check(lib, make(4, N, M, D, dtype, bias=False, residual=False), dtype, None)


@pytest.mark.parametrize("N,M,D", [(4000, 4100, 4104), (12, 8200, 2100), (20, 10000, 2000), (50, 1030, 4000)])
def test_largest_tiles_and_few_rows(lib, N, M, D):
    """The largest tiles in all three products; rows on either side of where every workgroup reads all of them"""
    print(f"case N={N} M={M} D={D}", flush=True)
    check(lib, make(11, N, M, D, "bf16"), "bf16", "silu")


@pytest.mark.parametrize("N,M,D", [(4000, 4100, 8256), (4000, 8256, 4104), (8256, 4000, 4104)])
def test_long_sums_of_the_largest_tiles(lib, N, M, D):
    """Equal rows have equal results, whatever step their tiles begin with"""
    print(f"case N={N} M={M} D={D}", flush=True)
    s = make(20, N, M, D, "bf16", residual=False)
    s["x"][N - 7] = s["x"][1]
    out, _ = check(lib, s, "bf16", "gelu")
    assert torch.equal(out[N - 7], out[1])


def test_offsets_beyond_32_bits(lib):
    """Results that begin more than 2^31 elements behind the first one"""
    N, M, D = 140_000, 16_384, 64
    s = make(12, N, M, D, "bf16", bias=True, residual=False)
    out, slope = lib.cfgzip_head_layer(s["x"], s["w"], s["b"], activation="silu", want_slope=True)
    y, y_err, sl, sl_err = forward(s["x"][-200:].double(), s["w"].double(), s["b"].double(), "silu", None, "bf16")
    within(out[-200:], y, y_err, "out")
    within(slopes(slope[-200:]), sl, sl_err, "slope")
    gh = lib.cfgzip_head_layer_grad(s["x"], s["w"], s["g"], slope=slope, want_weight=False)[0]
    want = gradients(s["x"][-200:].double(), s["w"].double(), s["g"][-200:].double(), slopes(slope[-200:]), "bf16", False)
    within(gh[-200:], *want["grad_hidden"], "grad_hidden")


def test_offsets_beyond_32_bits_in_the_weights_gradient(lib):
    """Only the last rows have gradients"""
    N, M, D = 140_000, 16_384, 64
    s = make(13, N, M, D, "bf16", bias=True, residual=False)
    s["g"][:-200] = 0
    slope = lib.cfgzip_head_layer(s["x"], s["w"], s["b"], activation="gelu", want_slope=True)[1]
    _, gw, gb = lib.cfgzip_head_layer_grad(s["x"], s["w"], s["g"], slope=slope, want_hidden=False, want_bias=True)
    want = gradients(s["x"][-200:].double(), s["w"].double(), s["g"][-200:].double(), slopes(slope[-200:]), "bf16", False)
    within(gw, *want["grad_weight"], "grad_weight")
    within(gb, *want["grad_bias"], "grad_bias")


def test_many_odd_rows_are_copied(lib):
    """More units than a copy has threads"""
    N, M, D = 21_000, 24, 7_001
    s = make(14, N, M, D, "bf16", bias=True, residual=False)
    out = lib.cfgzip_head_layer(s["x"], s["w"], s["b"])[0]
    gw = lib.cfgzip_head_layer_grad(s["x"], s["w"], s["g"], want_hidden=False)[1]
    x, w, b, g = (s[k].double() for k in "xwbg")
    within(out, *forward(x, w, b, None, None, "bf16")[:2], "out")
    within(gw, *gradients(x, w, g, None, "bf16", True)["grad_weight"], "grad_weight")


def test_odd_weights_in_large_tiles(lib):
    check(lib, make(5, 1000, 1111, 777, "bf16", w_offset=1), "bf16", "relu")
    check(lib, make(5, 1000, 1111, 777, "f16", w_gap=2), "f16", "relu")


@pytest.mark.parametrize("size", [1e-7, 3e-5, 1.0, 3e4])
def test_gradients_of_any_size_in_half_precision(lib, size):
    s = make(6, 120, 200, 96, "f16", size=size)
    s["g"].clamp_(-60000.0, 60000.0)
    check(lib, s, "f16", "silu")
    check(lib, s, "f16", None)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("size", [1e-20, 1.0, 1e6])
def test_gradients_in_single_precision(lib, size, dtype):
    s = make(7, 90, 130, 64, dtype)
    if dtype == "f16" and size != 1.0:  # results that the type holds
        s["x"].mul_(1e-3), s["w"].mul_(1e-3)
        size = {1e-20: 1e-2, 1e6: 1e6}[size]
    gen = torch.Generator(device="cuda").manual_seed(1)
    check(lib, s, dtype, "gelu", g=rows(gen, 90, 130, torch.float32, 3, 4, size))
    check(lib, s, dtype, None, g=rows(gen, 90, 130, torch.float32, 0, 0, size))


def test_given_outputs_and_a_residual_in_place(lib):
    for N in (9, 40, 300):
        s = make(8, N, 136, 128, "bf16")
        want, slope = lib.cfgzip_head_layer(s["x"], s["w"], s["b"], activation="silu", residual=s["r"], want_slope=True)
        assert lib.cfgzip_head_layer(s["x"], s["w"], s["b"], activation="silu", residual=s["r"])[1] is None
        given = torch.zeros((N, 150), dtype=torch.int16, device="cuda")
        place = s["r"].clone()
        work = torch.empty(lib.load_library().cfgzip_head_layer_workspace_bytes(N, 136, 128) + 256, dtype=torch.uint8, device="cuda")
        out, sl = lib.cfgzip_head_layer(s["x"], s["w"], s["b"], activation="silu", residual=place, out=place, slope=given[:, 3:139], workspace=work)
        assert out is place and torch.equal(place, want) and torch.equal(given[:, 3:139], slope) and not given[:, :3].any() and not given[:, 139:].any()
        gh, gw, gb = lib.cfgzip_head_layer_grad(s["x"], s["w"], s["g"], slope=slope, want_bias=True)
        wide = torch.zeros((136, 131), dtype=torch.bfloat16, device="cuda")
        a = lib.cfgzip_head_layer_grad(s["x"], s["w"], s["g"], slope=slope, want_hidden=False, grad_weight=wide[:, 2:130])
        assert a[0] is None and a[2] is None and torch.equal(wide[:, 2:130], gw) and not wide[:, :2].any() and not wide[:, 130:].any()
        assert torch.equal(lib.cfgzip_head_layer_grad(s["x"], s["w"], s["g"], slope=slope, want_weight=False)[0], gh)
        b = lib.cfgzip_head_layer_grad(s["x"], s["w"], s["g"], slope=slope, want_hidden=False, want_weight=False, want_bias=True)
        assert b[0] is None and b[1] is None and torch.equal(b[2], gb)


def test_no_rows_and_refusals(lib):
    x, w = torch.zeros((0, 8), dtype=torch.float16, device="cuda"), torch.ones((4, 8), dtype=torch.float16, device="cuda")
    out, slope = lib.cfgzip_head_layer(x, w, want_slope=True)
    assert out.shape == slope.shape == (0, 4)
    gh, gw, gb = lib.cfgzip_head_layer_grad(x, w, out, slope=slope, want_bias=True)
    assert gh.shape == (0, 8) and not gw.any() and not gb.any()
    x = torch.zeros((3, 8), dtype=torch.float16, device="cuda")
    for bad in (lambda: lib.cfgzip_head_layer(x[:, :7], w), lambda: lib.cfgzip_head_layer(x, w, w[0]), lambda: lib.cfgzip_head_layer(x, w, residual=x),
                lambda: lib.cfgzip_head_layer(x, w, activation="tanh"), lambda: lib.cfgzip_head_layer(x, w.t()),
                lambda: lib.cfgzip_head_layer(x, w, out=w), lambda: lib.cfgzip_head_layer_grad(x, w, x),
                lambda: lib.cfgzip_head_layer_grad(x, w, x[:, :4], want_hidden=False, want_weight=False)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: lib.cfgzip_head_layer(x.bfloat16(), w), lambda: lib.cfgzip_head_layer(x.float(), w.float()),
                lambda: lib.cfgzip_head_layer(x, w, dtype=torch.bfloat16), lambda: lib.cfgzip_head_layer(x, w, slope=x[:, :4]),
                lambda: lib.cfgzip_head_layer_grad(x, w, x[:, :4].bfloat16())):
        with pytest.raises(TypeError):
            bad()


@pytest.mark.parametrize("N", [12, 70, 600])
def test_streams_and_graphs(lib, N):
    """On a side stream, captured, and replayed with other inputs between eager calls that have workspaces of their own"""
    s = make(9, N, 520, 384, "f16")

    def call(stream=None):
        out, slope = lib.cfgzip_head_layer(s["x"], s["w"], s["b"], activation="gelu", residual=s["r"], want_slope=True, stream=stream)
        return (out, slope, *lib.cfgzip_head_layer_grad(s["x"], s["w"], s["g"], slope=slope, want_bias=True, stream=stream))

    want = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = call(side)
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for seed in range(4):
        other = make(20 + seed, N, 520, 384, "f16")
        s["x"].copy_(other["x"]), s["w"].copy_(other["w"]), s["g"].copy_(other["g"])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, call()):
            assert torch.equal(a, b), seed


def test_gradients_against_differences(lib):
    s = make(10, 20, 24, 16, "f16", size=1.0)
    out, slope = lib.cfgzip_head_layer(s["x"], s["w"], s["b"], activation="silu", want_slope=True, dtype=torch.float32)
    gh, gw, gb = lib.cfgzip_head_layer_grad(s["x"], s["w"], s["g"], slope=slope, want_bias=True)

    def total(**change):
        t = {**s, **change}
        return float((lib.cfgzip_head_layer(t["x"], t["w"], t["b"], activation="silu", dtype=torch.float32)[0].double() * s["g"].double()).sum())

    for key, grad in (("x", gh), ("w", gw), ("b", gb)):
        for at in (0, 5, 11):
            up, down = s[key].contiguous().clone(), s[key].contiguous().clone()
            value = float(up.view(-1)[at])
            up.view(-1)[at] = value + 0.03
            down.view(-1)[at] = value - 0.03
            step = float(up.view(-1)[at]) - float(down.view(-1)[at])
            # a difference is off by step^2 / 24 of the third derivative: of each of 24 (20) outputs at most 0.25 |other operand|^3, and by the
            # rounding of outputs of at most 10; the gradient by dz's rounding, slope's and its own
            size = float(s["g"].abs().double().sum()) * 4.0 ** 3
            allowed = step ** 2 / 24 * 0.25 * size + 500 * 10 * 2.0 ** -24 / step + 3 * 2.0 ** -11 * size / 16
            assert abs((total(**{key: up}) - total(**{key: down})) / step - float(grad.view(-1)[at])) < allowed, (key, at)
