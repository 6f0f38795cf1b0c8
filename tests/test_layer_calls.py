"""Log probabilities and the layer in front of the vocabulary projection through the binding's extension: what is not plain tensors in GPU
memory is left to the general way, and what it takes gives the same bits as the calls through ctypes."""

import os

import pytest

torch = pytest.importorskip("torch")

CALLS = {"token_logprobs": 7, "token_logprobs_grad": 11, "head_layer": 7, "head_layer_grad": 7}


@pytest.fixture()
def binding():
    from paper_2605_29986_amd import binding, build
    if not (os.path.exists(binding.library_path()) and os.path.exists(binding.stepcall_path())):
        build.build()
    binding.load_library()
    return binding


def test_what_is_not_plain_is_left_alone(binding):
    assert list(CALLS) == list(binding._LAYER_CALLS)
    t = torch.zeros((4, 4))
    for name, n in CALLS.items():
        call = getattr(binding, "_" + name)
        assert call.__module__ == "cfgzip_stepcall"
        assert call(*range(n)) is None and call(*[t] * n) is None and call() is None and call(*[None] * n) is None


def test_without_the_extension(binding, monkeypatch, tmp_path):
    for name in ("_lib", *("_" + c for c in (*binding._CALLS, *binding._HEAD_CALLS, *CALLS))):  # (put back behind the test)
        monkeypatch.setattr(binding, name, None)
    monkeypatch.setattr(binding, "_STEPCALL_PATH", str(tmp_path / "cfgzip_stepcall.so"))
    with pytest.warns(RuntimeWarning, match="through ctypes"):
        binding.load_library()
    for name, n in CALLS.items():
        assert getattr(binding, "_" + name) is binding._by_ctypes


@pytest.mark.gpu
@pytest.mark.parametrize("mask", ["none", "token", "class"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_the_same_as_through_ctypes(binding, monkeypatch, dtype, mask):
    print(f"case {dtype} mask={mask}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(3)
    N, M, D, C = 21, 6000, 72, 40
    hidden = torch.randn((N, D + 8), device="cuda", generator=gen).to(dtype)[:, 3:3 + D]
    weight = torch.randn((M, D), device="cuda", generator=gen).to(dtype)
    bias = torch.randn((M,), device="cuda", generator=gen).to(dtype)
    residual = torch.randn((N, M + 3), device="cuda", generator=gen).to(dtype)[:, 1:1 + M]
    tokens = torch.randint(-1, M + 1, (N, 3), device="cuda", generator=gen).int()
    masks = {}
    if mask == "token":
        masks = {"bits": torch.randint(-2**31, 2**31 - 1, (N, (M + 31) // 32), device="cuda", generator=gen).int()}
    if mask == "class":
        masks = {"bits": torch.randint(-2**31, 2**31 - 1, (N, (C + 31) // 32), device="cuda", generator=gen).int(),
                 "class_of_token": torch.randint(0, C, (M,), device="cuda", generator=gen).int(), "C": C}
    g = torch.randn((N, 3), device="cuda", generator=gen)
    ge = torch.randn((N,), device="cuda", generator=gen)

    def results():
        out = []
        for t in (None, torch.float32, dtype):
            out += binding.cfgzip_head_layer(hidden, weight, bias, activation="gelu", residual=residual, dtype=t, want_slope=True)
        slope = out[-1]
        out.append(binding.cfgzip_head_layer(hidden, weight)[0])
        for logits in (out[0], out[2]):
            for one in (tokens, tokens[:, 0].contiguous()):
                score = binding.cfgzip_token_logprobs(logits, one, top=5, temperature=0.5, **masks)
                out += score
                g1 = g.view(-1)[:one.numel()].view(one.shape)
                out.append(binding.cfgzip_token_logprobs_grad(logits, one, score[0], score[2], g1, temperature=0.5, **masks))
                out.append(binding.cfgzip_token_logprobs_grad(logits, one, score[0], score[2], g1, entropy=score[1], grad_entropy=ge,
                                                              temperature=0.5, **masks))
            out += binding.cfgzip_head_layer_grad(hidden, weight, out[-1], slope=slope, want_bias=True)
            out += binding.cfgzip_token_logprobs(logits, **masks)[1:3]
        out += binding.cfgzip_head_layer_grad(hidden, weight, residual, want_weight=False)[:1]
        return out

    quick = results()
    for name in CALLS:
        monkeypatch.setattr(binding, "_" + name, binding._by_ctypes)
    for i, (a, b) in enumerate(zip(quick, results())):
        assert a.shape == b.shape and a.dtype == b.dtype and a.stride() == b.stride(), i
        assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)), i
