"""The layer, the projection, log probabilities and their gradients one after the other, as a program has them: a drafting head under a
grammar's masks, served with weights in 4 bits and trained.  Every call is held to its definition on what the call before it gave."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from head_reference import pack
from layer_reference import forward, gradients, slopes
from logprobs_reference import gradient, logprobs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    import paper_2605_29986_amd as cz
    return cz


def near(got, want, err, what):
    got, want, err = (t.double().cpu().numpy() if isinstance(t, torch.Tensor) else t for t in (got, want, err))
    with np.errstate(invalid="ignore"):
        assert ((got == want) | (np.abs(got - want) <= err)).all(), what


def setting(N, V, D, dtype):
    gen = torch.Generator(device="cuda").manual_seed(N)
    rng = np.random.default_rng(N)
    C = 90
    c, bits = rng.integers(0, C, V).astype(np.int32), rng.random((N, C)) < 0.3
    bits[1] = False
    allowed = bits[:, c]
    s = {"hidden": torch.randn((N, D), device="cuda", generator=gen).to(dtype), "w": (torch.randn((D, D), device="cuda", generator=gen) / D ** 0.5).to(dtype),
         "b": torch.randn((D,), device="cuda", generator=gen).to(dtype), "head": (1.5 * torch.randn((V, D), device="cuda", generator=gen) / D ** 0.5).to(dtype),
         "allowed": allowed, "how": {"bits": torch.from_numpy(pack(bits)).cuda(), "class_of_token": torch.from_numpy(c).cuda(), "C": C}}
    return s, rng


def test_serving(lib):
    """One block of a drafting head, its masked logits from weights in 4 bits, the candidates of a draft"""
    s, rng = setting(6, 5003, 256, torch.bfloat16)
    codes, scales = lib.cfgzip_mx4_quantize(s["head"])
    states, _ = lib.cfgzip_head_layer(s["hidden"], s["w"], s["b"], activation="silu", residual=s["hidden"])
    y, err, _, _ = forward(s["hidden"].double(), s["w"].double(), s["b"].double(), "silu", s["hidden"].double(), "bf16")
    near(states, y, err, "states")
    logits = lib.cfgzip_mx4_logits(states, codes, scales, **s["how"])
    sampled = logits.argmax(1).int()
    lp, h, st, tokens, tlp = lib.cfgzip_token_logprobs(logits, sampled, top=8, temperature=0.2)
    r = logprobs(logits.double().cpu().numpy(), sampled.cpu().numpy()[:, None], s["allowed"], 0.2, 8)
    near(lp[:, None], r["logprob"], r["logprob_err"], "logprob")
    near(h, r["entropy"], r["entropy_err"], "entropy")
    assert (tokens.cpu().numpy() == r["top_tokens"]).all() and (tokens[1] == -1).all()
    near(tlp, r["top_logprobs"], r["top_err"], "top_logprobs")
    live = np.arange(6) != 1
    assert (tokens[:, 0] == sampled).cpu().numpy()[live].all() and torch.equal(tlp[live, 0], lp[live])
    for i in np.flatnonzero(live):  # whatever is a candidate is admitted
        there = tokens[i][tokens[i] >= 0].cpu().numpy()
        assert s["allowed"][i, there].all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_training(lib, dtype):
    """The same head in 16 bits: log probabilities of taken tokens with an entropy bonus, and gradients back to the layer's inputs"""
    N, V, D = 90, 3001, 192
    s, rng = setting(N, V, D, torch.bfloat16 if dtype == "bf16" else torch.float16)
    states, slope = lib.cfgzip_head_layer(s["hidden"], s["w"], s["b"], activation="gelu", residual=s["hidden"], want_slope=True)
    logits, _ = lib.cfgzip_head_layer(states, s["head"])
    z, z_err, _, _ = forward(states.double(), s["head"].double(), None, None, None, dtype)
    near(logits, z, z_err, "logits")
    taken = rng.integers(0, V, (N, 1)).astype(np.int32)
    for i in range(0, N, 2):
        if s["allowed"][i].any():
            taken[i] = rng.choice(np.flatnonzero(s["allowed"][i]))
    g, ge = rng.standard_normal((N, 1)).astype(np.float32), np.full(N, 0.01, np.float32)
    tokens = torch.from_numpy(taken).cuda()
    lp, h, st, _, _ = lib.cfgzip_token_logprobs(logits, tokens, **s["how"])
    grad_logits = lib.cfgzip_token_logprobs_grad(logits, tokens, lp, st, torch.from_numpy(g).cuda(), entropy=h, grad_entropy=torch.from_numpy(ge).cuda(),
                                                 **s["how"])
    r = logprobs(logits.double().cpu().numpy(), taken, s["allowed"], 1.0, 0)
    near(lp, r["logprob"], r["logprob_err"], "logprob")
    near(grad_logits, *gradient(r, taken, g.astype(np.float64), ge.astype(np.float64), 1.0, dtype), "grad_logits")
    assert not grad_logits[1].any()
    grad_states, grad_head, _ = lib.cfgzip_head_layer_grad(states, s["head"], grad_logits)
    want = gradients(states.double(), s["head"].double(), grad_logits.double(), None, dtype, dtype == "bf16")
    near(grad_states, *want["grad_hidden"], "grad_states")
    near(grad_head, *want["grad_weight"], "grad_head")
    grad_hidden, grad_w, grad_b = lib.cfgzip_head_layer_grad(s["hidden"], s["w"], grad_states, slope=slope, want_bias=True)
    want = gradients(s["hidden"].double(), s["w"].double(), grad_states.double(), slopes(slope), dtype, False)
    for got, key in ((grad_hidden, "grad_hidden"), (grad_w, "grad_weight"), (grad_b, "grad_bias")):
        near(got, *want[key], key)
