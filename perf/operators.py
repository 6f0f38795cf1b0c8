"""The vocabulary projection at the end of a language model, as measurable cases: trained under a grammar's masks in 16 bits,
kept in 4, and served under the grammar's masks.

Four kinds, each through the public entry points of ``paper_2605_29986_amd``:

  loss      cross entropy of hidden states against target tokens over the tokens that each row's mask admits, without the
            logits in memory (``cfgzip_head_loss``)
  train     the same and its gradients of hidden states and weights (``cfgzip_head_loss``, ``cfgzip_head_loss_grad``)
  quantize  weights to blocks of 32 values of 4 bits with a shared power of two, and back (``cfgzip_mx4_quantize``,
            ``cfgzip_mx4_values``)
  logits    logits of such weights, -inf where the row's mask does not admit the token (``cfgzip_mx4_logits``); hidden states in
            16 bits, or quantised on the way in like the weights

The definitions.  z[i][v] = sum_d hidden[i][d] weight[v][d].  Row i admits token v if bit class_of_token[v] of cls_bits[i] is
set (every token without a mask).  lse[i] = log sum over admitted v of exp z[i][v], -inf if there are none.  A target outside
[0, V) counts for nothing: loss 0.  A target that the row does not admit has loss +inf.  Else loss[i] = lse[i] - z[i][target[i]],
and dz[i][v] = grad_loss[i] (exp(z[i][v] - lse[i]) - [v = target[i]]) for admitted v; dz is 0 everywhere else and in all rows of the
first two sorts; grad_hidden = dz weight, grad_weight = dz^T hidden.

A block of 32 values x along a row has the scale 2^e, e = floor(log2 max|x|) - 2, at least -127, kept as the byte e + 127 (0 for
a block of zeros); a value is the nearest of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} to x / 2^e, ties to the even code, at most 6.  Codes
are sign * 8 + index, the earlier value in a byte's low half, 16 bytes a block; the last block of a row is filled up with 0.

Vocabularies, class counts and the density of single-step masks are those of the repository's workloads; hidden sizes and rows are
generic.  Inputs are made on the GPU from the seed.
"""

from __future__ import annotations

import math

import torch

own = False

NINF = float("-inf")
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
STATES = 64  # automaton states that the rows of a training batch are in


def _words(n):
    return (n + 31) // 32


def _blocks(n):
    return (n + 31) // 32


def listed():
    return [
        # scoring one continuation of a prompt: one row, a medium vocabulary; the weights are read once
        {"name": "loss_n1", "kind": "loss", "N": 1, "V": 32_000, "D": 2_048, "C": 683, "dtype": "bf16", "pad": 0},
        # evaluation of a corpus: many rows, a large vocabulary, no grammar
        {"name": "loss_n2048", "kind": "loss", "N": 2_048, "V": 128_256, "D": 2_048, "C": 0, "dtype": "bf16", "pad": 0},
        # a small model learning a small grammar's language: launches count as much as products
        {"name": "train_n64", "kind": "train", "N": 64, "V": 4_096, "D": 256, "C": 683, "dtype": "bf16", "pad": 0},
        # a ragged batch in half precision: odd vocabulary, hidden states that are a slice of a wider tensor
        {"name": "train_n777_odd", "kind": "train", "N": 777, "V": 50_003, "D": 1_000, "C": 3_001, "dtype": "f16", "pad": 24},
        # a training batch of a large model under the masks of its grammar
        {"name": "train_n4096", "kind": "train", "N": 4_096, "V": 128_256, "D": 4_096, "C": 8_000, "dtype": "bf16", "pad": 0},
        # a medium head on its way into 4 bits, from the master copy
        {"name": "quantize_32k", "kind": "quantize", "V": 32_000, "D": 1_999, "dtype": "f32"},
        # a large head
        {"name": "quantize_128k", "kind": "quantize", "V": 128_256, "D": 4_096, "dtype": "bf16"},
        # interactive decoding under a grammar: one sequence, a large vocabulary of which the mask leaves half
        {"name": "logits_b1", "kind": "logits", "B": 1, "V": 128_256, "D": 4_096, "C": 8_000, "dtype": "bf16", "x": "16",
         "out": "f32"},
        # a small batch without a grammar, half precision
        {"name": "logits_b12", "kind": "logits", "B": 12, "V": 50_003, "D": 2_048, "C": 0, "dtype": "f16", "x": "16",
         "out": "f32"},
        # the serving batch
        {"name": "logits_b256", "kind": "logits", "B": 256, "V": 128_256, "D": 4_096, "C": 8_000, "dtype": "bf16", "x": "16",
         "out": "bf16"},
        # a small batch with both sides in 4 bits
        {"name": "logits4_b8", "kind": "logits", "B": 8, "V": 32_000, "D": 2_048, "C": 683, "dtype": "bf16", "x": "4",
         "out": "f32"},
        # prompts of a whole batch with both sides in 4 bits
        {"name": "logits4_b1024", "kind": "logits", "B": 1_024, "V": 128_256, "D": 4_096, "C": 8_000, "dtype": "bf16", "x": "4",
         "out": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_hidden_size(rng):
    """Mostly whole multiples of 64 or 8, as hidden sizes are; now and then any number."""
    D = _log_int(rng, 64, 4_096)
    step = rng.choice((64, 64, 64, 8, 8, 1))
    return max(step, D // step * step)


def draw(rng):
    kind = rng.choice(("loss", "train", "train", "quantize", "logits", "logits", "logits"))
    V = _log_int(rng, 1_000, 151_936)
    D = _draw_hidden_size(rng)
    C = _log_int(rng, 24, min(V // 4, 16_000)) if rng.random() < 0.6 else 0
    if kind in ("loss", "train"):
        most = 4_096 * 4_096 * 128_256 // (D * V)
        return {"kind": kind, "N": _log_int(rng, 1, min(4_096, most)), "V": V, "D": D, "C": C,
                "dtype": rng.choice(("bf16", "bf16", "f16")), "pad": rng.choice((0, 0, 8, 64, 5))}
    if kind == "quantize":
        return {"kind": kind, "V": min(V, 128_256), "D": D, "dtype": rng.choice(("bf16", "f16", "f32"))}
    return {"kind": kind, "B": _log_int(rng, 1, 1_024), "V": min(V, 128_256), "D": D, "C": C,
            "dtype": rng.choice(("bf16", "bf16", "f16")), "x": rng.choice(("16", "16", "4")),
            "out": rng.choice(("bf16", "f32"))}


# ---------------------------------------------------------------- inputs


def _randn(gen, *shape):
    return torch.randn(shape, device="cuda", generator=gen)


def _class_map(gen, V, C):
    """A class map with heavy-tailed class sizes, every class used."""
    u = torch.rand((V,), device="cuda", generator=gen)
    cls = (torch.pow(C + 1.0, u) - 1.0).long().clamp_(0, C - 1)  # density ~ 1 / (1 + class)
    at = torch.randperm(V, device="cuda", generator=gen)[:C]
    cls[at] = torch.arange(C, device="cuda")
    return cls.to(torch.int32)


def _pack_bits(bits):
    """bool [R][32 * W] to int32 [R][W]"""
    R, n = bits.shape
    shift = torch.arange(32, device=bits.device)
    word = (bits.view(R, n // 32, 32).long() << shift).sum(-1)
    return torch.where(word >= 2**31, word - 2**32, word).to(torch.int32)


def _admits(cls_bits, class_of_token, rows=None):
    """bool [rows][V]: the tokens that each row admits, from the masks over classes"""
    c = class_of_token.long()
    bits = cls_bits if rows is None else cls_bits[rows]
    return ((bits[:, c // 32] >> (c % 32).to(torch.int32)) & 1).bool()


def _state_masks(gen, N, V, C):
    """Masks of rows that are in one of a grammar's states each: the states leave very different shares of the classes, one of
    them (no live state any more) nothing."""
    c = _class_map(gen, V, C)
    share = torch.pow(2.0, -8.0 * torch.rand((STATES, 1), device="cuda", generator=gen))
    share[0], share[1] = 0.0, 0.5
    bits = torch.rand((STATES, 32 * _words(C)), device="cuda", generator=gen) < share
    masks = _pack_bits(bits)
    state = torch.randint(0, STATES, (N,), device="cuda", generator=gen)
    state[0] = 1
    return masks[state].contiguous(), c


def _targets(gen, N, V, cls_bits, c):
    """Tokens that the rows admit, if one is found in 512 tries; some rows are prompt and have none, a few are mistakes in the data."""
    if cls_bits is None:
        target = torch.randint(0, V, (N,), device="cuda", generator=gen)
    else:
        tries = torch.randint(0, V, (N, 512), device="cuda", generator=gen)
        k = c.long()[tries]
        good = (torch.gather(cls_bits, 1, k // 32) >> (k % 32).to(torch.int32)) & 1
        target = torch.gather(tries, 1, good.argmax(1, keepdim=True))[:, 0]
    u = torch.rand((N,), device="cuda", generator=gen)
    any_token = torch.randint(0, V, (N,), device="cuda", generator=gen)
    u[0] = 0.5
    target = torch.where(u < 0.02, any_token, target)
    target = torch.where(u > 0.95, torch.full_like(target, -1), target)
    return target.to(torch.int32)


def _prepare_loss(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    N, V, D, C, T = case["N"], case["V"], case["D"], case["C"], TYPES[case["dtype"]]
    weight = torch.empty((V, D), dtype=T, device="cuda")
    for v in range(0, V, 16_384):  # logits of hidden states of unit size have a spread of 1.5
        weight[v:v + 16_384] = (_randn(gen, min(16_384, V - v), D) * (1.5 / math.sqrt(D))).to(T)
    cls_bits, c = _state_masks(gen, N, V, C) if C else (None, None)
    target = _targets(gen, N, V, cls_bits, c)
    # a model that has learned something: the target's logit is anything from an accident to a certainty
    sure = 16.0 * torch.rand((N, 1), device="cuda", generator=gen) / (1.5 * math.sqrt(D))
    toward = weight[target.long().clamp(min=0)].float() * (math.sqrt(D) / 1.5)
    hidden = torch.zeros((N, D + case["pad"]), dtype=T, device="cuda")
    hidden[:, :D] = (_randn(gen, N, D) + sure * math.sqrt(D) / 1.5 * toward).to(T)
    s = {"hidden": hidden[:, :D], "weight": weight, "target": target, "cls_bits": cls_bits, "c": c}
    if case["kind"] == "train":  # rows weighted by advantages of both signs, divided by their number; half precision scales its losses
        s["grad_loss"] = _randn(gen, N) * ((1_024.0 if case["dtype"] == "f16" else 1.0) / N)
    return s


def _prepare_logits(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B, V, D, C, T = case["B"], case["V"], case["D"], case["C"], TYPES[case["dtype"]]
    codes = torch.empty((V, 16 * _blocks(D)), dtype=torch.uint8, device="cuda")
    scales = torch.empty((V, _blocks(D)), dtype=torch.uint8, device="cuda")
    for v in range(0, V, 16_384):
        n = min(16_384, V - v)
        size = torch.exp(0.5 * _randn(gen, n, 1)) * (1.5 / math.sqrt(D))
        codes[v:v + n], scales[v:v + n] = _plain_quantize(_randn(gen, n, D) * size)
    hidden = _randn(gen, B, D)
    hidden[:, :: max(1, D // 6)] *= 20.0  # a few channels stand out, as they do behind a model's last layer
    s = {"hidden": hidden.to(T), "codes": codes, "scales": scales, "cls_bits": None, "c": None}
    if C:
        s["c"] = _class_map(gen, V, C)
        s["cls_bits"] = _pack_bits(torch.rand((B, 32 * _words(C)), device="cuda", generator=gen) < 0.5)
    return s


def _prepare_quantize(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    V, D = case["V"], case["D"]
    x = torch.empty((V, D), dtype=TYPES[case["dtype"]], device="cuda")
    for v in range(0, V, 16_384):
        n = min(16_384, V - v)
        x[v:v + n] = (_randn(gen, n, D) * torch.exp(_randn(gen, n, 1)) * (1.5 / math.sqrt(D))).to(x.dtype)
    x[:: 97] = 0.0  # tokens that were never trained
    return {"x": x}


def prepare(case, seed):
    make = {"loss": _prepare_loss, "train": _prepare_loss, "quantize": _prepare_quantize, "logits": _prepare_logits}
    s = make[case["kind"]](case, seed)
    s["case"] = case
    return s


# ---------------------------------------------------------------- the plain forms


def _plain_blocks(x):
    """fp32 [R][nb][32], filled up with 0"""
    R, D = x.shape
    x = x.float()
    if D % 32:
        x = torch.cat([x, x.new_zeros((R, 32 - D % 32))], 1)
    return x.view(R, -1, 32)


def _plain_quantize(x):
    blocks = _plain_blocks(x)
    R, nb = blocks.shape[:2]
    most = blocks.abs().amax(-1)
    e = (torch.frexp(most).exponent - 3).clamp(min=-127)
    e = torch.where(most > 0, e, torch.full_like(e, -127))
    y = torch.ldexp(blocks.abs(), -e[..., None])
    # steps of 1/2 up to 2, of 1 up to 4, of 2 up to 6; round() takes ties to the even multiple, which has the even code
    index = torch.where(y < 2, torch.round(2 * y), torch.where(y < 4, torch.round(y) + 2, torch.round(y / 2) + 4))
    code = index.clamp(max=7).to(torch.uint8) | (torch.signbit(blocks).to(torch.uint8) << 3)
    codes = code[..., 0::2] | (code[..., 1::2] << 4)
    return codes.reshape(R, nb * 16), (e + 127).to(torch.uint8)


def _plain_values(codes, scales, D):
    """fp32 [R][D]"""
    R, nb = scales.shape
    code = torch.stack([codes & 15, codes >> 4], -1).view(R, nb, 32)
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    value = torch.ldexp(table[code.int()], (scales.int() - 127)[..., None])
    return value.reshape(R, nb * 32)[:, :D]


def _plain_loss(s):
    hidden, weight, target = s["hidden"].float(), s["weight"].float(), s["target"].long()
    V = weight.shape[0]
    z = hidden @ weight.t()
    if s["cls_bits"] is not None:
        z = z.masked_fill(~_admits(s["cls_bits"], s["c"]), NINF)
    most = z.amax(1)
    shift = torch.where(most > NINF, most, torch.zeros_like(most))
    e = torch.exp(z - shift[:, None])
    total = e.sum(1)
    lse = torch.log(total) + shift
    there = (target >= 0) & (target < V)
    at = target.clamp(0, V - 1)
    z_target = torch.gather(z, 1, at[:, None])[:, 0]
    counts = there & (z_target > NINF)
    loss = torch.where(counts, lse - z_target, torch.where(there, torch.full_like(lse, math.inf), torch.zeros_like(lse)))
    return hidden, weight, e, total, at, counts, loss, lse


def _plain_train(s):
    hidden, weight, e, total, at, counts, loss, lse = _plain_loss(s)
    p = e / total[:, None]
    dz = p - torch.zeros_like(p).scatter_(1, at[:, None], 1.0)
    dz = torch.where(counts[:, None], dz * s["grad_loss"][:, None], torch.zeros_like(dz))
    T = s["hidden"].dtype
    return loss, lse, (dz @ weight).to(T), (dz.t() @ hidden).to(T)


def _plain_logits(s):
    case = s["case"]
    x = s["hidden"].float()
    if case["x"] == "4":
        x = _plain_values(*_plain_quantize(x), x.shape[1])
    z = x @ _plain_values(s["codes"], s["scales"], x.shape[1]).t()
    if s["cls_bits"] is not None:
        z = z.masked_fill(~_admits(s["cls_bits"], s["c"]), NINF)
    return z.to(TYPES[case["out"]])


# ---------------------------------------------------------------- one pass


def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        if kind == "loss":
            loss, lse = _plain_loss(s)[-2:]
            return {"loss": loss, "lse": lse}
        if kind == "train":
            loss, lse, gh, gw = _plain_train(s)
            return {"loss": loss, "lse": lse, "grad_hidden": gh, "grad_weight": gw}
        if kind == "quantize":
            return {"values": _plain_values(*_plain_quantize(s["x"]), s["x"].shape[1]).to(s["x"].dtype)}
        return {"logits": _plain_logits(s)}

    import paper_2605_29986_amd as cfgzip
    masks = {"bits": s["cls_bits"], "class_of_token": s["c"], "C": case["C"]} if case.get("C") else {}
    if kind in ("loss", "train"):
        loss, lse = cfgzip.cfgzip_head_loss(s["hidden"], s["weight"], s["target"], **masks)
        if kind == "loss":
            return {"loss": loss, "lse": lse}
        gh, gw = cfgzip.cfgzip_head_loss_grad(s["hidden"], s["weight"], s["target"], lse, s["grad_loss"], **masks)
        return {"loss": loss, "lse": lse, "grad_hidden": gh, "grad_weight": gw}
    if kind == "quantize":
        codes, scales = cfgzip.cfgzip_mx4_quantize(s["x"])
        return {"values": cfgzip.cfgzip_mx4_values(codes, scales, s["x"].shape[1], dtype=s["x"].dtype)}
    hidden, hidden_scales = s["hidden"], None
    if case["x"] == "4":
        hidden, hidden_scales = cfgzip.cfgzip_mx4_quantize(hidden)
    return {"logits": cfgzip.cfgzip_mx4_logits(hidden, s["codes"], s["scales"], hidden_scales=hidden_scales,
                                               dtype=TYPES[case["out"]], **masks)}


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    """Bytes: every input read once, every output written once.  Operations: one product for the logits, one for each gradient.
    Weights of tokens that no row of the batch admits need not be read: that counts where rows are few (each row of the decoding
    cases admits half of the classes)."""
    kind, V, D = case["kind"], case["V"], case["D"]
    if kind == "quantize":
        size = 4 if case["dtype"] == "f32" else 2
        return {"bytes": 2 * size * V * D, "flops": 0}
    mask = 4 * V if case["C"] else 0
    if kind == "logits":
        B, nb = case["B"], _blocks(D)
        read = 1.0 - 0.5 ** B if case["C"] else 1.0
        out = 2 if case["out"] == "bf16" else 4
        n = read * V * nb * 17 + B * D * 2 + B * V * out + mask + (4 * B * _words(case["C"]) if case["C"] else 0)
        return {"bytes": n, "flops": 2 * read * B * V * D}
    N = case["N"]
    n = 2 * (V + N) * D + 12 * N + mask + (4 * N * _words(case["C"]) if case["C"] else 0)
    if kind == "loss":
        return {"bytes": n, "flops": 2 * N * V * D}
    return {"bytes": n + 2 * (V + N) * D + 4 * N, "flops": 6 * N * V * D}


# ---------------------------------------------------------------- the definition in 64 bits


def _exact_allowed(s, lo, hi):
    """Which of the tokens lo..hi each row admits, from the bytes of the masks."""
    B = s["cls_bits"].shape[0]
    octets = s["cls_bits"].contiguous().view(torch.uint8).view(B, -1).short()
    k = s["c"][lo:hi].long()
    return (octets[:, k // 8].bitwise_right_shift((k % 8).short()) & 1) == 1


def _exact_train(case, s):
    h = s["hidden"].double()
    N, V = case["N"], case["V"]
    t = s["target"].long()
    step = max(1_024, 2**27 // N)
    parts = [(v, min(V, v + step)) for v in range(0, V, step)]

    def z_of(lo, hi):
        z = torch.mm(h, s["weight"][lo:hi].double().t().contiguous())
        return z if s["cls_bits"] is None else torch.where(_exact_allowed(s, lo, hi), z, NINF)

    lse = torch.stack([torch.logsumexp(z_of(*p), 1) for p in parts]).logsumexp(0)
    has = (t > -1) & (t < V)
    row = torch.nonzero(has)[:, 0]
    zt = torch.full((N,), NINF, dtype=torch.float64, device="cuda")
    zt[row] = (h[row] * s["weight"][t[row]].double()).sum(1)
    if s["cls_bits"] is not None:
        k = s["c"].long()[t[row]]
        bit = (s["cls_bits"][row, k // 32].long() >> (k % 32)) & 1
        zt[row[bit == 0]] = NINF
    loss = torch.zeros_like(lse)
    loss[has] = lse[has] - zt[has]
    loss[has & (zt == NINF)] = math.inf
    if case["kind"] == "loss":
        return {"loss": loss, "lse": lse}
    live = torch.nonzero(has & (zt > NINF))[:, 0]
    g = s["grad_loss"].double()
    gh, gw = torch.zeros_like(h), torch.zeros((V, case["D"]), dtype=torch.float64, device="cuda")
    for lo, hi in parts:
        d = torch.exp(z_of(lo, hi)[live] - lse[live, None])
        inside = torch.nonzero((t[live] >= lo) & (t[live] < hi))[:, 0]
        d[inside, t[live][inside] - lo] -= 1.0
        d *= g[live, None]
        gh[live] += torch.mm(d, s["weight"][lo:hi].double())
        gw[lo:hi] = torch.mm(d.t().contiguous(), h[live])
    return {"loss": loss, "lse": lse, "grad_hidden": gh, "grad_weight": gw}


def _exact_rounded(x):
    """The nearest values that 4 bits and a scale of 2^e to each 32 values can stand for, in 64 bits, by comparison with the
    midpoints of neighbouring values."""
    R, D = x.shape
    x = torch.nn.functional.pad(x.double(), (0, -D % 32)).view(R, -1, 32)
    most = x.abs().max(-1, keepdim=True).values
    scale = torch.exp2((torch.floor(torch.log2(most)) - 2).clamp(min=-127.0))
    y = x.abs() / scale
    up = torch.zeros_like(y)
    # (midpoint, step to the upper neighbour, whether a value on the midpoint goes up: to the even code)
    for mid, gap, tie in ((0.25, 0.5, False), (0.75, 0.5, True), (1.25, 0.5, False), (1.75, 0.5, True), (2.5, 1.0, False),
                          (3.5, 1.0, True), (5.0, 2.0, False)):
        up += gap * ((y >= mid) if tie else (y > mid)).double()
    return (torch.sign(x) * up * scale).view(R, -1)[:, :D]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("loss", "train"):
        return _exact_train(case, s)
    if case["kind"] == "quantize":
        return {"values": torch.cat([_exact_rounded(x) for x in s["x"].split(16_384)])}
    x = s["hidden"].double()
    if case["x"] == "4":
        x = _exact_rounded(x)
    V, nb = s["scales"].shape
    sizes = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device="cuda")
    z = torch.empty((x.shape[0], V), dtype=torch.float64, device="cuda")
    for lo in range(0, V, 16_384):
        hi = min(V, lo + 16_384)
        octets = s["codes"][lo:hi].int()
        w = torch.empty((hi - lo, nb * 32), dtype=torch.float64, device="cuda")
        for half in (0, 1):
            nibble = octets // 16 if half else octets % 16
            w[:, half::2] = torch.where(nibble > 7, -1.0, 1.0) * sizes[(nibble % 8).long()]
        w = w.view(hi - lo, nb, 32) * torch.exp2(s["scales"][lo:hi].double() - 127.0)[..., None]
        z[:, lo:hi] = torch.mm(x, w.view(hi - lo, -1)[:, : x.shape[1]].t().contiguous())
        if s["cls_bits"] is not None:
            z[:, lo:hi] = torch.where(_exact_allowed(s, lo, hi), z[:, lo:hi], NINF)
    return {"logits": z}
