"""cfgzip_token_logprobs and cfgzip_token_logprobs_grad against their definition in 64 bits."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from head_reference import F32, pack
from logprobs_reference import gradient, logprobs

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(scope="module")
def lib():
    import paper_2605_29986_amd as cz
    return cz


def make(seed, N, V, dtype, mask="none", n=1, C=None, values="normal", offset=0, gap=0):
    """What a call takes: logits a slice of a wider tensor, masks, tokens and gradients; NaN and infinities in masked places"""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((N, V)) * 3
    if values == "ties":
        x = np.round(x)
    if values == "equal":
        x[:] = 1.5
    if values == "rising":
        x = np.sort(x, axis=1)
    if values == "peaked":
        x[np.arange(N), rng.integers(0, V, N)] += 40.0
    if values == "large":
        x = x * 100 - 20000.0
    if values == "lowest":  # masks of the type's lowest value, one row of nothing else
        low = torch.finfo(TYPES[dtype]).min
        x[rng.random((N, V)) < 0.5] = low
        x[0] = low
    if values == "infinite":
        x[rng.random((N, V)) < 0.5] = -np.inf
        x[0] = -np.inf
    if values == "zeros":
        x = np.where(rng.random((N, V)) < 0.5, 0.0, -0.0)
    t = torch.from_numpy(x).to(TYPES[dtype])
    allowed = np.ones((N, V), bool)
    how = {}
    if mask != "none":
        C = C or max(1, V // 5)
        c = rng.integers(0, C, V).astype(np.int32)
        share = rng.random((N, 1)) ** 2
        bits = rng.random((N, C if mask == "class" else V)) < share
        if N > 1:
            bits[1] = False
        if N > 2:
            bits[2] = False
            bits[2, rng.integers(0, bits.shape[1])] = True
        allowed = bits[:, c] if mask == "class" else bits
        wild = torch.tensor([float("nan"), float("inf"), -float("inf")], dtype=TYPES[dtype])
        at = torch.from_numpy(~allowed)
        t[at] = wild[torch.from_numpy(rng.integers(0, 3, int(at.sum())))]
        how["bits"] = torch.from_numpy(pack(bits)).cuda()
        if mask == "class":
            how.update(class_of_token=torch.from_numpy(c).cuda(), C=C)
    wide = torch.full((N, V + offset + gap), float("nan"), dtype=TYPES[dtype], device="cuda")
    wide[:, offset:offset + V] = t.cuda()
    tokens = rng.integers(-2, V + 2, (N, n)).astype(np.int32)
    if n > 1:
        tokens[:, 1] = tokens[:, 0]
    for i in range(0, N, 2):  # admitted ones too
        here = np.flatnonzero(allowed[i])
        if len(here) and n:
            tokens[i] = rng.choice(here, n)
    g, ge = rng.standard_normal((N, n)).astype(np.float32), (0.3 * rng.standard_normal(N)).astype(np.float32)
    return {"x": t.double().numpy(), "logits": wide[:, offset:offset + V], "wide": wide, "tokens": tokens, "allowed": allowed, "how": how, "g": g, "ge": ge}


def within(got, want, err, what):
    got = got.double().cpu().numpy() if isinstance(got, torch.Tensor) else got
    got = got.reshape(want.shape)
    same = got == want  # infinities
    with np.errstate(invalid="ignore"):
        bad = ~(same | (np.abs(got - want) <= err))
    assert not bad.any(), (what, np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4], np.broadcast_to(err, want.shape)[bad][:4])


def check(lib, s, dtype, top=0, temperature=1.0, entropy_too=True, rows=None):
    tokens = torch.from_numpy(s["tokens"]).cuda()
    before = s["wide"].clone()
    how = {**s["how"], "temperature": temperature}
    lp, h, st, tt, tl = lib.cfgzip_token_logprobs(s["logits"], tokens, top=top, **how)
    grad = lib.cfgzip_token_logprobs_grad(s["logits"], tokens, lp, st, torch.from_numpy(s["g"]).cuda(), entropy=h if entropy_too else None,
                                          grad_entropy=torch.from_numpy(s["ge"]).cuda() if entropy_too else None, **how)
    assert torch.equal(before.view(torch.uint8), s["wide"].view(torch.uint8))
    pick = np.arange(len(s["x"])) if rows is None else np.asarray(rows)
    r = logprobs(s["x"][pick], s["tokens"][pick], s["allowed"][pick], temperature, top)
    at = torch.from_numpy(pick)
    lp, h, st = lp.cpu()[at], h.cpu()[at], st.cpu()[at]
    within(lp, r["logprob"], r["logprob_err"], "logprob")
    within(h, r["entropy"], r["entropy_err"], "entropy")
    assert (st[:, 0].double().numpy() == r["stats"][:, 0]).all()
    within(st[:, 1], r["stats"][:, 1], r["log_sum_err"], "log of the sum")
    if top:
        assert (tt.cpu()[at].numpy() == r["top_tokens"]).all(), np.argwhere(tt.cpu()[at].numpy() != r["top_tokens"])[:4]
        within(tl.cpu()[at], r["top_logprobs"], r["top_err"], "top_logprobs")
    else:
        assert tt is None and tl is None
    want, err = gradient(r, s["tokens"][pick], s["g"][pick].astype(np.float64), s["ge"][pick].astype(np.float64) if entropy_too else None,
                         temperature, dtype)
    within(grad.cpu()[at], want, err, "grad_logits")
    return lp, h, st, tt, tl, grad


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 63, 65, 513, 4095, 4096, 4097, 9001, 70001])
def test_lengths(lib, V, dtype):
    print(f"case V={V} {dtype}", flush=True)
    check(lib, make(V, 3, V, dtype, n=2), dtype, top=min(64, V + 3))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("mask", ["none", "token", "class"])
@pytest.mark.parametrize("N,V,n,top", [(1, 5000, 1, 20), (5, 12345, 3, 1), (70, 9000, 1, 64), (300, 1500, 5, 7), (600, 4100, 0, 0)])
def test_masks(lib, N, V, n, top, mask, dtype):
    print(f"case N={N} V={V} n={n} top={top} mask={mask} {dtype}", flush=True)
    check(lib, make(N + V, N, V, dtype, mask=mask, n=n), dtype, top=top, temperature=0.7)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("N,V", [(769, 3001), (801, 9000), (131, 200_001)])
def test_two_rows_to_a_workgroup(lib, N, V, dtype):
    """Many rows under masks over classes, whole and in pieces; an odd one out"""
    print(f"case N={N} V={V} {dtype}", flush=True)
    check(lib, make(N, N, V, dtype, mask="class", n=2, C=700), dtype, rows=[0, 1, 2, 3, N // 2, N - 2, N - 1])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("values", ["ties", "equal", "rising", "peaked", "large", "lowest", "infinite", "zeros"])
def test_values(lib, values, dtype):
    print(f"case {values} {dtype}", flush=True)
    for N, V, top in ((2, 20000, 64), (3, 700, 33), (520, 9000, 12)):
        check(lib, make(1, N, V, dtype, n=2, values=values), dtype, top=top, rows=[0, 1, N - 1])


@pytest.mark.parametrize("temperature", [0.05, 0.2, 1.5, 30.0])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_temperatures(lib, dtype, temperature):
    print(f"case {temperature} {dtype}", flush=True)
    check(lib, make(2, 9, 6001, dtype, mask="class", n=2), dtype, top=10, temperature=temperature, entropy_too=dtype != "f16")


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("offset,gap", [(0, 1), (1, 0), (3, 2), (8, 8), (5, 11)])
def test_rows_anywhere(lib, offset, gap, dtype):
    print(f"case {offset} {gap} {dtype}", flush=True)
    check(lib, make(3, 4, 5003, dtype, mask="token", n=1, offset=offset, gap=gap), dtype, top=5)


@pytest.mark.parametrize("N,V,mask", [(1, 128_256, "none"), (3, 5001, "class"), (4, 70_001, "token"), (800, 4000, "class")])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_certain_rows(lib, N, V, mask, dtype):
    """Rows of which one token has nearly all: what is left of 1 is their log probability, entropy and gradient, and is as exact relative to itself"""
    print(f"case {N} {V} {mask} {dtype}", flush=True)
    s = make(15, N, V, dtype, mask=mask, n=1)
    rng = np.random.default_rng(1)
    rows = [0, N - 1] if N < 5 else [0, 5, N - 1]
    for i in rows:
        if s["allowed"][i].any():
            best = rng.choice(np.flatnonzero(s["allowed"][i]))
            s["tokens"][i] = best
            s["logits"][i, int(best)] = 24.0 + 6 * rng.random()
    s["x"] = s["logits"].double().cpu().numpy()
    lp, h, st, _, _, grad = check(lib, s, dtype, rows=rows)
    r = logprobs(s["x"][rows], s["tokens"][rows], s["allowed"][rows], 1.0, 0)
    for k, i in enumerate(rows):
        if not s["allowed"][i].any():
            continue
        # exactly, by the largest logit's token: its log p is log(1 - all others), and theirs are apart from it by d
        others, d, t = r["p"][k].copy(), r["d"][k], int(s["tokens"][i, 0])
        best = int(np.argmax(others))
        others[best] = 0.0
        top = np.log1p(-others.sum()) if others.sum() < 0.5 else r["log_p"][k, best]
        want = top + d[t]
        # the sum of all others is off relative to itself: terms as in logprobs(), d up to 40 here; its logarithm by two steps more
        rounds = -(-V // (8 * 512))
        rel = F32 * (6 * 60 + 6 * (rounds + 2) + 4 + 8 * rounds + 24 + 8)
        assert abs(float(lp[k, 0]) - want) <= rel * (abs(top) + abs(d[t])) + 2.0 ** -126, (i, float(lp[k, 0]), want)
        with np.errstate(all="ignore"):
            entropy = -top * r["p"][k, best] - np.where(others > 0, others * (np.where(others > 0, d, 0.0) + top), 0.0).sum()
        assert abs(float(h[k]) - entropy) <= 3 * rel * entropy + 2.0 ** -120, (i, float(h[k]), entropy)
        left = others.sum() if t == best else 1.0 - r["p"][k, t]
        if dtype == "f32":  # with an entropy bonus in it: what both give to the token, each as exact
            g, ge = float(s["g"][i, 0]), float(s["ge"][i])
            parts = abs(g) * left + abs(ge) * entropy + abs(ge * want)
            exact = g * left - ge * (1 - left) * (want + entropy)
            assert abs(float(grad[i, t]) - exact) <= 8 * rel * parts + 2.0 ** -120, (i, float(grad[i, t]), exact)


def test_offsets_beyond_32_bits(lib):
    """Rows that begin more than 2^31 elements behind the first one"""
    N, V = 17_000, 128_256
    x = torch.zeros((N, V), dtype=torch.bfloat16, device="cuda")
    s = make(16, 2, V, "bf16", n=1)
    x[N - 2:] = s["logits"]
    tokens = torch.zeros((N, 1), dtype=torch.int32, device="cuda")
    tokens[N - 2:] = torch.from_numpy(s["tokens"]).cuda()
    g = torch.zeros((N, 1), device="cuda")
    g[N - 2:] = torch.from_numpy(s["g"]).cuda()
    lp, h, st, tt, tl = lib.cfgzip_token_logprobs(x, tokens, top=5)
    lib.cfgzip_token_logprobs_grad(x, tokens, lp, st, g, grad_logits=x)
    r = logprobs(s["x"], s["tokens"], s["allowed"], 1.0, 5)
    within(lp[N - 2:], r["logprob"], r["logprob_err"], "logprob")
    within(h[N - 2:], r["entropy"], r["entropy_err"], "entropy")
    assert (tt[N - 2:].cpu().numpy() == r["top_tokens"]).all()
    within(x[N - 2:], *gradient(r, s["tokens"], s["g"].astype(np.float64), None, 1.0, "bf16"), "grad_logits")
    assert not x[:N - 2].any()


def test_many_classes(lib):
    """Masks over more classes than LDS holds"""
    check(lib, make(4, 3, 300_000, "bf16", mask="class", C=280_000, n=2), "bf16", top=9)


@pytest.mark.parametrize("dtype,mask,top,C", [("bf16", "none", 64, 0), ("f16", "token", 33, 0), ("f32", "class", 20, 3000), ("bf16", "class", 50, 131_072)])
def test_alternatives_of_long_rows(lib, dtype, mask, top, C):
    """A thread has more units than slots, some of them behind the row's end"""
    print(f"case {dtype} {mask} top={top}", flush=True)
    check(lib, make(18, 200, 270_001, dtype, mask, n=1, C=C), dtype, top=top, rows=[0, 1, 2, 101, 199])


@pytest.mark.parametrize("N,V", [(260, 131_000), (3, 20_000)])
@pytest.mark.parametrize("top", [5, 24, 64])
def test_alternatives_that_differ_in_their_last_bits(lib, N, V, top):
    """Of fp32 logits that are one value in fewer bits, all slots look as if they had one of the best"""
    s = make(19, N, V, "f32", n=1)
    s["logits"].mul_(2.0 ** -12).add_(1.0 if top != 24 else -1.0)
    s["x"] = s["logits"].double().cpu().numpy()
    check(lib, s, "f32", top=top, rows=[0, 1, N - 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_logits_in_a_few_threads(lib, dtype):
    """The best logits lie in units that the same few threads take: more of them than there is room to put together"""
    N, V = 300, 65_536
    s = make(5, N, V, dtype, n=1)
    rng = np.random.default_rng(6)
    unit = np.arange(V) // 8 % 512
    for i in range(2):
        few = np.isin(unit, rng.choice(64, 40, replace=False))
        s["x"][i, few] += 100.0
    s["logits"].copy_(torch.from_numpy(s["x"]).to(TYPES[dtype]))
    s["x"] = s["logits"].double().cpu().numpy()
    check(lib, s, dtype, top=64, rows=[0, 1, 2, N - 1])


def test_many_tokens(lib):
    """Every token of the vocabulary given, some twice; and the most that a call takes"""
    s = make(7, 3, 300, "f32", n=700)
    s["tokens"][0] = np.arange(700) % 300
    check(lib, s, "f32")
    check(lib, make(8, 2, 5000, "bf16", mask="class", n=4096), "bf16", top=3)


def test_without_tokens(lib):
    s = make(9, 5, 1000, "f32")
    lp, h, st, tt, tl = lib.cfgzip_token_logprobs(s["logits"])
    assert lp is None and tt is None and tl is None
    ge = torch.from_numpy(s["ge"]).cuda()
    grad = lib.cfgzip_token_logprobs_grad(s["logits"], None, None, st, None, entropy=h, grad_entropy=ge)
    none = np.zeros((5, 0), np.int32)
    r = logprobs(s["x"], none, s["allowed"], 1.0, 0)
    within(h, r["entropy"], r["entropy_err"], "entropy")
    within(grad, *gradient(r, none, np.zeros((5, 0)), s["ge"].astype(np.float64), 1.0, "f32"), "grad_logits")


def test_one_token_a_row_and_given_outputs(lib):
    s = make(10, 6, 3000, "bf16", mask="class")
    tokens = torch.from_numpy(s["tokens"][:, 0].copy()).cuda()
    want = lib.cfgzip_token_logprobs(s["logits"], tokens, top=4, **s["how"])
    assert want[0].shape == (6,)
    out = {"logprob": torch.zeros(6, device="cuda"), "entropy": torch.zeros(6, device="cuda"), "stats": torch.zeros((6, 2), device="cuda"),
           "top_tokens": torch.zeros((6, 4), dtype=torch.int32, device="cuda"), "top_logprobs": torch.zeros((6, 4), device="cuda"),
           "workspace": torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")}
    got = lib.cfgzip_token_logprobs(s["logits"], tokens, top=4, **s["how"], **out)
    for a, b, name in zip(want, got, out):
        assert b is out[name] and torch.equal(a, b)
    g = torch.from_numpy(s["g"][:, 0].copy()).cuda()
    grad = lib.cfgzip_token_logprobs_grad(s["logits"], tokens, want[0], want[2], g, **s["how"])
    wide = torch.zeros((6, 3011), dtype=torch.bfloat16, device="cuda")
    lib.cfgzip_token_logprobs_grad(s["logits"], tokens, want[0], want[2], g, grad_logits=wide[:, 5:3005], **s["how"])
    assert torch.equal(wide[:, 5:3005], grad) and not wide[:, :5].any() and not wide[:, 3005:].any()


@pytest.mark.parametrize("dtype", list(TYPES))
def test_gradient_in_place(lib, dtype):
    s = make(11, 40, 33_001, dtype, mask="class", n=6, gap=7)
    tokens, g, ge = torch.from_numpy(s["tokens"]).cuda(), torch.from_numpy(s["g"]).cuda(), torch.from_numpy(s["ge"]).cuda()
    lp, h, st, _, _ = lib.cfgzip_token_logprobs(s["logits"], tokens, **s["how"])
    want = lib.cfgzip_token_logprobs_grad(s["logits"], tokens, lp, st, g, entropy=h, grad_entropy=ge, **s["how"])
    got = lib.cfgzip_token_logprobs_grad(s["logits"], tokens, lp, st, g, entropy=h, grad_entropy=ge, grad_logits=s["logits"], **s["how"])
    assert got.data_ptr() == s["logits"].data_ptr() and torch.equal(got, want)
    assert torch.isnan(s["wide"][:, 33_001:]).all()


def test_rows_without_gradients(lib):
    """Gradients of 0, tokens that are none: zeros, whatever the logits hold"""
    x = torch.full((4, 5000), float("nan"), device="cuda")
    x[3] = torch.randn(5000, device="cuda")
    tokens = torch.tensor([3, -1, 5000, 7], dtype=torch.int32, device="cuda")
    lp, h, st, _, _ = lib.cfgzip_token_logprobs(x, tokens)
    g = torch.tensor([0.0, 1.0, 1.0, 1.0], device="cuda")
    grad = lib.cfgzip_token_logprobs_grad(x, tokens, lp, st, g)
    assert not grad[:3].any() and grad[3].all() and torch.isnan(lp[0]) and lp[1] == 0 and lp[2] == 0


def test_masked_in_the_logits_or_by_the_mask(lib):
    """Logits that cfgzip_apply_mask masked need no mask: the same bits"""
    s = make(12, 20, 9000, "bf16", n=3)
    rng = np.random.default_rng(3)
    c = torch.from_numpy(rng.integers(0, 400, 9000).astype(np.int32)).cuda()
    bits = torch.from_numpy(pack(rng.random((20, 400)) < 0.4)).cuda()
    tokens, g = torch.from_numpy(s["tokens"]).cuda(), torch.from_numpy(s["g"]).cuda()
    how = {"bits": bits, "class_of_token": c, "C": 400}
    a = lib.cfgzip_token_logprobs(s["logits"], tokens, top=30, **how)
    ga = lib.cfgzip_token_logprobs_grad(s["logits"], tokens, a[0], a[2], g, **how)
    masked = s["logits"].contiguous().clone()
    lib.cfgzip_apply_mask(masked, bits, class_of_token=c, C=400)
    b = lib.cfgzip_token_logprobs(masked, tokens, top=30)
    gb = lib.cfgzip_token_logprobs_grad(masked, tokens, b[0], b[2], g)
    for x, y in zip((*a, ga), (*b, gb)):
        assert torch.equal(x, y)


def test_gradient_against_differences(lib):
    s = make(13, 2, 400, "f32", mask="class", n=3)
    tokens, g, ge = torch.from_numpy(s["tokens"]).cuda(), torch.from_numpy(s["g"]).cuda().double(), torch.from_numpy(s["ge"]).cuda().double()

    def total(x):
        lp, h, _, _, _ = lib.cfgzip_token_logprobs(x, tokens, **s["how"])
        return float((torch.where(torch.isfinite(lp), lp, 0.0).double() * torch.where(torch.isfinite(lp), g, 0.0)).sum() + (h.double() * ge).sum())

    lp, h, st, _, _ = lib.cfgzip_token_logprobs(s["logits"], tokens, **s["how"])
    grad = lib.cfgzip_token_logprobs_grad(s["logits"], tokens, lp, st, g.float(), entropy=h, grad_entropy=ge.float(), **s["how"])
    for v in np.flatnonzero(s["allowed"][0])[:20]:
        up, down = s["logits"].contiguous().clone(), s["logits"].contiguous().clone()
        up[0, v] += 0.02
        down[0, v] -= 0.02
        # the difference's own error: 0.02^2 / 6 of the third derivative, at most 2 (|g| + |ge| (entropy + 6)) here; totals rounded to fp32
        size = float(g.abs().sum() + ge.abs().sum() * 15)
        assert abs((total(up) - total(down)) / 0.04 - float(grad[0, v])) < 0.02 ** 2 / 3 * size + 64 * 2.0 ** -24 * size / 0.04


def test_streams_and_graphs(lib):
    """On a side stream, captured, and replayed with other logits between eager calls that use workspaces of their own"""
    s = make(14, 8, 40_000, "bf16", mask="class", n=2)
    tokens, g = torch.from_numpy(s["tokens"]).cuda(), torch.from_numpy(s["g"]).cuda()
    x = s["logits"].contiguous().clone()
    side = torch.cuda.Stream()

    def call(stream=None):
        out = lib.cfgzip_token_logprobs(x, tokens, top=12, stream=stream, **s["how"])
        return (*out, lib.cfgzip_token_logprobs_grad(x, tokens, out[0], out[2], g, stream=stream, **s["how"]))

    want = call()
    torch.cuda.synchronize()
    got = call(side)
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for seed in range(4):
        x.copy_(make(20 + seed, 8, 40_000, "bf16", n=2)["logits"])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, call()):
            assert torch.equal(a, b), seed


def test_no_rows_and_refusals(lib):
    x = torch.zeros((0, 50), device="cuda")
    t = torch.zeros(0, dtype=torch.int32, device="cuda")
    lp, h, st, tt, tl = lib.cfgzip_token_logprobs(x, t, top=3)
    assert lp.shape == (0,) and st.shape == (0, 2) and tt.shape == (0, 3)
    assert lib.cfgzip_token_logprobs_grad(x, t, lp, st, lp).shape == (0, 50)
    x = torch.zeros((4, 50), device="cuda")
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (lambda: lib.cfgzip_token_logprobs(x, t[:3]), lambda: lib.cfgzip_token_logprobs(x.t(), t), lambda: lib.cfgzip_token_logprobs(x, t.view(1, 4)),
                lambda: lib.cfgzip_token_logprobs(x, t, bits=t.view(4, 1)), lambda: lib.cfgzip_token_logprobs(x, t, class_of_token=t, C=4),
                lambda: lib.cfgzip_token_logprobs(x, t, logprob=x[:3, 0].contiguous())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: lib.cfgzip_token_logprobs(x.double(), t), lambda: lib.cfgzip_token_logprobs(x, t.long())):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: lib.cfgzip_token_logprobs(x, t, top=65), lambda: lib.cfgzip_token_logprobs(x, t, top=-1),
                lambda: lib.cfgzip_token_logprobs(x, t, temperature=0.0)):
        with pytest.raises(lib.CfgzipError):
            bad()
    lp, h, st, _, _ = lib.cfgzip_token_logprobs(x, t)
    for bad in (lambda: lib.cfgzip_token_logprobs_grad(x, t, lp, st, lp[:3]), lambda: lib.cfgzip_token_logprobs_grad(x, t, None, st, lp),
                lambda: lib.cfgzip_token_logprobs_grad(x, t, lp, st, lp, grad_entropy=lp),
                lambda: lib.cfgzip_token_logprobs_grad(x, t, lp, st, lp, grad_logits=x[:3])):
        with pytest.raises(ValueError):
            bad()
