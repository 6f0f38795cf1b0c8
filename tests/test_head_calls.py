"""The vocabulary projection's calls through the binding's extension: what is not plain tensors in GPU memory is left to the general
way, and what it takes gives the same bits as the calls through ctypes."""

import os

import pytest

torch = pytest.importorskip("torch")

CALLS = {"head_loss": 6, "head_loss_grad": 10, "mx4_quantize": 1, "mx4_values": 4, "mx4_logits": 8}


@pytest.fixture()
def binding():
    from paper_2605_29986_amd import binding, build
    if not (os.path.exists(binding.library_path()) and os.path.exists(binding.stepcall_path())):
        build.build()
    binding.load_library()
    return binding


def test_what_is_not_plain_is_left_alone(binding):
    assert list(CALLS) == list(binding._HEAD_CALLS)
    t = torch.zeros((4, 4))
    for name, n in CALLS.items():
        call = getattr(binding, "_" + name)
        assert call.__module__ == "cfgzip_stepcall"
        assert call(*range(n)) is None and call(*[t] * n) is None and call() is None and call(*[None] * n) is None


def test_refusals_without_a_gpu(binding):
    w = torch.zeros((50, 24), dtype=torch.bfloat16)
    t = torch.zeros(5, dtype=torch.int32)
    for call in (lambda: binding.cfgzip_head_loss(w[:5], w, t), lambda: binding.cfgzip_head_loss_grad(w[:5], w, t, t.float(), t.float()),
                 lambda: binding.cfgzip_mx4_quantize(w), lambda: binding.cfgzip_mx4_values(w.byte(), w.byte(), 24),
                 lambda: binding.cfgzip_mx4_logits(w, w.byte(), w.byte())):
        with pytest.raises(TypeError):
            call()


@pytest.mark.gpu
@pytest.mark.parametrize("mask", ["none", "token", "class"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_the_same_as_through_ctypes(binding, monkeypatch, dtype, mask):
    print(f"case {dtype} mask={mask}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(3)
    N, V, D, C = 21, 300, 72, 40
    hidden = torch.randn((N, D + 8), device="cuda", generator=gen).to(dtype)[:, 3:3 + D]
    weight = torch.randn((V, D), device="cuda", generator=gen).to(dtype)
    target = torch.randint(0, V, (N,), device="cuda", generator=gen).int()
    grad = torch.randn((N,), device="cuda", generator=gen)
    masks = {}
    if mask == "token":
        masks = {"bits": torch.randint(-2**31, 2**31 - 1, (N, (V + 31) // 32), device="cuda", generator=gen).int()}
    if mask == "class":
        masks = {"bits": torch.randint(-2**31, 2**31 - 1, (N, (C + 31) // 32), device="cuda", generator=gen).int(),
                 "class_of_token": torch.randint(0, C, (V,), device="cuda", generator=gen).int(), "C": C}

    def results():
        loss, lse = binding.cfgzip_head_loss(hidden, weight, target, **masks)
        out = [loss, lse, *binding.cfgzip_head_loss_grad(hidden, weight, target, lse, grad, **masks)]
        out.append(binding.cfgzip_head_loss_grad(hidden, weight, target, lse, grad, want_hidden=False, **masks)[1])
        out += binding.cfgzip_mx4_quantize(weight)
        codes, scales = out[-2:]
        out += [binding.cfgzip_mx4_values(codes, scales, D, dtype=t) for t in (torch.float32, torch.bfloat16, torch.float16)]
        for rows in (1, N):
            few = {**masks, "bits": masks["bits"][:rows].contiguous()} if masks else {}
            out += [binding.cfgzip_mx4_logits(hidden[:rows], codes, scales, dtype=t, **few) for t in (torch.float32, torch.bfloat16)]
        hc, hs = binding.cfgzip_mx4_quantize(hidden)
        out.append(binding.cfgzip_mx4_logits(hc, codes, scales, hidden_scales=hs, **masks))
        return out

    quick = results()
    for name in CALLS:
        monkeypatch.setattr(binding, "_" + name, binding._by_ctypes)
    for i, (a, b) in enumerate(zip(quick, results())):
        assert a.shape == b.shape and a.dtype == b.dtype and a.stride() == b.stride(), i
        assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)), i
