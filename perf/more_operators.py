"""What stands around the vocabulary projection of a language model, as measurable cases: the layer in front of it, and what is
read from its logits under a grammar's masks, each forwards and backwards.

Four kinds, each through the public entry points of ``paper_2605_29986_amd``:

  score   log probabilities of given tokens over the tokens that each row's mask admits, entropy, what the gradient
          needs of a row, and the best alternatives (``cfgzip_token_logprobs``)
  policy  the same with the gradient of the logits, of log probabilities and entropy (``cfgzip_token_logprobs``,
          ``cfgzip_token_logprobs_grad``)
  layer   matrix product with bias, activation and residual (``cfgzip_head_layer``)
  train   the same with the gradients of its inputs (``cfgzip_head_layer``, ``cfgzip_head_layer_grad``)

The definitions.  Row i admits token v if bit class_of_token[v] of bits[i] is set (every token without a mask) and its logit is
not -inf.  z[i][v] = logits[i][v] / temperature.  lse[i] = log sum over admitted v of exp z[i][v], -inf if there are none.  For a given
token t: logprob = z[i][t] - lse[i]; 0 if t lies outside [0, V), which makes it none; -inf if the row does not admit it.  stats[i] is the largest
admitted logit, and lse[i] less that one's z (both -inf if there are none).  With p = exp(z - lse): entropy[i] = -sum over admitted v of p log p, 0 if there are none.  Alternatives: the admitted tokens with the largest logits, largest
first, of equal ones the lowest; token -1 with -inf where there are no more.  With gradients g of the log probabilities and e of the entropy, over
admitted v:

    grad_logits[i][v] = (sum_j g[i][j] [v = t[i][j]] - p[v] (G + e[i] (log p[v] + entropy[i]))) / temperature,

G the sum of g[i][j] over the tokens that are admitted; 0 elsewhere.

    out = act(hidden weight^T + bias) + residual;   with dz = grad_out act'(.):
    grad_hidden = dz weight,   grad_weight = dz^T hidden,   grad_bias = the sum of dz over the rows

gelu(x) = x (1 + erf(x / sqrt 2)) / 2; gelu_tanh(x) = x (1 + tanh(sqrt(2 / pi) (x + 0.044715 x^3))) / 2; silu(x) = x / (1 + exp(-x)).

Vocabularies, class counts and masks are those of the repository's workloads; hidden sizes and rows are generic.  Inputs are made on the GPU
from the seed.
"""

from __future__ import annotations

import math

import torch

own = False

NINF = float("-inf")
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
STATES = 64  # automaton states that the rows of a batch are in
MOST_LOGITS = 4_096 * 128_256
MOST_PRODUCTS = 4_096 * 4_096 * 16_384


def _words(n):
    return (n + 31) // 32


def listed():
    return [
        # one sequence, decoded interactively under a grammar: its token's log probability and twenty alternatives for the answer
        {"name": "score_b1", "kind": "score", "N": 1, "V": 128_256, "C": 8_000, "n": 1, "top": 20, "temperature": 1.0, "dtype": "bf16", "pad": 0},
        # a small batch without a grammar, odd vocabulary, rows of a wider buffer: candidates of a draft
        {"name": "score_b12_odd", "kind": "score", "N": 12, "V": 50_003, "C": 0, "n": 1, "top": 8, "temperature": 1.0, "dtype": "f16", "pad": 13},
        # eight choices of an answer compared in every row, no alternatives
        {"name": "score_b64_choices", "kind": "score", "N": 64, "V": 32_000, "C": 683, "n": 8, "top": 0, "temperature": 1.0, "dtype": "f32", "pad": 0},
        # the serving batch at its sampling temperature
        {"name": "score_b256", "kind": "score", "N": 256, "V": 128_256, "C": 8_000, "n": 1, "top": 20, "temperature": 0.2, "dtype": "bf16",
         "pad": 0},
        # a small student learns from the 32 best tokens of a teacher
        {"name": "policy_n512_teacher", "kind": "policy", "N": 512, "V": 32_000, "C": 0, "n": 32, "top": 0, "temperature": 1.5, "dtype": "f16",
         "pad": 0},
        # a ragged batch of single-precision logits trained by rewards, with an entropy bonus
        {"name": "policy_n777_odd", "kind": "policy", "N": 777, "V": 50_003, "C": 3_001, "n": 1, "top": 0, "temperature": 1.0, "dtype": "f32",
         "pad": 5},
        # a training batch of a large model's answers under their grammar's masks
        {"name": "policy_n4096", "kind": "policy", "N": 4_096, "V": 128_256, "C": 8_000, "n": 1, "top": 0, "temperature": 1.0, "dtype": "bf16",
         "pad": 0},
        # a drafting head's residual block for one sequence: the weights are read once
        {"name": "layer_n1", "kind": "layer", "N": 1, "M": 4_096, "D": 4_096, "act": "silu", "bias": True, "residual": True, "dtype": "bf16", "pad": 0},
        # a head's transform for a small batch, odd sizes, hidden states that are a slice of a wider tensor
        {"name": "layer_n33_odd", "kind": "layer", "N": 33, "M": 1_999, "D": 1_000, "act": "gelu", "bias": True, "residual": False, "dtype": "f16",
         "pad": 24},
        # the residual block for the serving batch
        {"name": "layer_n256", "kind": "layer", "N": 256, "M": 4_096, "D": 4_096, "act": "silu", "bias": True, "residual": True, "dtype": "bf16",
         "pad": 0},
        # a ragged batch of a small head in half precision
        {"name": "train_n777_odd", "kind": "train", "N": 777, "M": 1_001, "D": 1_000, "act": "gelu", "bias": True, "residual": True, "dtype": "f16",
         "pad": 5},
        # a training batch of a wide layer of a large model
        {"name": "train_n4096", "kind": "train", "N": 4_096, "M": 16_384, "D": 4_096, "act": "gelu_tanh", "bias": True, "residual": False,
         "dtype": "bf16", "pad": 0},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_hidden_size(rng, most):
    """Mostly whole multiples of 64 or 8, as hidden sizes are; now and then any number."""
    D = _log_int(rng, 64, most)
    step = rng.choice((64, 64, 64, 8, 8, 1))
    return max(step, D // step * step)


def draw(rng):
    kind = rng.choice(("score", "score", "policy", "policy", "layer", "layer", "train", "train"))
    if kind in ("score", "policy"):
        V = _log_int(rng, 1_000, 151_936)
        C = _log_int(rng, 24, min(V // 4, 16_000)) if rng.random() < 0.6 else 0
        top = _log_int(rng, 1, 64) if kind == "score" and rng.random() < 0.7 else 0
        return {"kind": kind, "N": _log_int(rng, 1, min(1_024 if kind == "score" else 4_096, MOST_LOGITS // V)), "V": V, "C": C,
                "n": rng.choice((1, 1, _log_int(rng, 1, 64))), "top": top, "temperature": rng.choice((1.0, 0.2, 0.7, 1.5)),
                "dtype": rng.choice(("bf16", "bf16", "f16", "f32")), "pad": rng.choice((0, 0, 8, 64, 5))}
    D, M = _draw_hidden_size(rng, 8_192), _draw_hidden_size(rng, 16_384)
    return {"kind": kind, "N": _log_int(rng, 1, min(4_096, MOST_PRODUCTS // (D * M))), "M": M, "D": D,
            "act": rng.choice(("none", "relu", "gelu", "gelu_tanh", "silu", "silu")), "bias": rng.random() < 0.7,
            "residual": rng.random() < 0.5, "dtype": rng.choice(("bf16", "bf16", "f16")), "pad": rng.choice((0, 0, 8, 64, 5))}


# ---------------------------------------------------------------- inputs


def _randn(gen, *shape):
    return torch.randn(shape, device="cuda", generator=gen)


def _rand(gen, *shape):
    return torch.rand(shape, device="cuda", generator=gen)


def _wider(x, pad, dtype):
    """x in `dtype` as the first columns of a tensor with `pad` more"""
    out = torch.zeros((x.shape[0], x.shape[1] + pad), dtype=dtype, device="cuda")
    out[:, :x.shape[1]] = x
    return out[:, :x.shape[1]]


def _class_map(gen, V, C):
    """A class map with heavy-tailed class sizes, every class used."""
    cls = (torch.pow(C + 1.0, _rand(gen, V)) - 1.0).long().clamp_(0, C - 1)  # density ~ 1 / (1 + class)
    at = torch.randperm(V, device="cuda", generator=gen)[:C]
    cls[at] = torch.arange(C, device="cuda")
    return cls.to(torch.int32)


def _pack_bits(bits):
    """bool [R][32 * W] to int32 [R][W]"""
    R, n = bits.shape
    shift = torch.arange(32, device=bits.device)
    word = (bits.view(R, n // 32, 32).long() << shift).sum(-1)
    return torch.where(word >= 2**31, word - 2**32, word).to(torch.int32)


def _state_masks(gen, N, C):
    """Masks of rows that are in one of a grammar's states each: the states leave very different shares of the classes, one of
    them (no live state any more) nothing."""
    share = torch.pow(2.0, -8.0 * _rand(gen, STATES, 1))
    share[0], share[1] = 0.0, 0.5
    masks = _pack_bits(_rand(gen, STATES, 32 * _words(C)) < share)
    state = torch.randint(0, STATES, (N,), device="cuda", generator=gen)
    state[0] = 1
    return masks[state].contiguous()


def _admits(bits, class_of_token):
    """bool [N][V]"""
    c = class_of_token.long()
    return ((bits[:, c // 32] >> (c % 32).to(torch.int32)) & 1).bool()


def _prepare_logits(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    N, V, C, n = case["N"], case["V"], case["C"], case["n"]
    s = {"bits": None, "c": None, "case": case}
    if C:
        s["c"], s["bits"] = _class_map(gen, V, C), _state_masks(gen, N, C)
    # tokens that the rows admit, if one is found in 64 tries; some rows are prompt and have none, a few are mistakes in the data
    tokens = torch.randint(0, V, (N, n), device="cuda", generator=gen)
    if C:
        tries = torch.randint(0, V, (N, 64), device="cuda", generator=gen)
        k = s["c"].long()[tries]
        good = (torch.gather(s["bits"], 1, k // 32) >> (k % 32).to(torch.int32)) & 1
        # (the admitted ones first, taken in turn; a row with few of them is given the same token twice)
        order = torch.argsort(good, dim=1, descending=True, stable=True)
        turn = torch.arange(n, device="cuda") % good.sum(1, keepdim=True).clamp(min=1)
        tokens = torch.gather(tries, 1, torch.gather(order, 1, turn))
    u = _rand(gen, N, n)
    u[0, 0] = 0.5
    tokens = torch.where(u < 0.02, torch.randint(0, V, (N, n), device="cuda", generator=gen), tokens)
    s["tokens"] = torch.where(u > 0.95, torch.full_like(tokens, -1), tokens).to(torch.int32)
    # a model's logits: a spread of 2.5, the given tokens' anything from an accident to a certainty
    logits = torch.empty((N, V + case["pad"]), dtype=TYPES[case["dtype"]], device="cuda")
    step = max(1, 2**27 // V)
    for i in range(0, N, step):
        z = _randn(gen, min(step, N - i), V) * 2.5
        z.scatter_add_(1, s["tokens"][i:i + step].long().clamp(min=0), 18.0 * _rand(gen, *s["tokens"][i:i + step].shape))
        logits[i:i + step, :V] = z.to(logits.dtype)
    logits[:, V:] = 0.0
    s["logits"] = logits[:, :V]
    if case["kind"] == "policy":  # weights of both signs (advantages, a teacher's probabilities), divided by the rows; a bonus on the entropy
        size = (1_024.0 if case["dtype"] == "f16" else 1.0) / N
        s["grad_logprob"] = _randn(gen, N, n) * size
        s["grad_entropy"] = (0.5 + _rand(gen, N)) * (0.05 * size)
    return s


def _prepare_layer(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    N, M, D, T = case["N"], case["M"], case["D"], TYPES[case["dtype"]]
    hidden = _randn(gen, N, D)
    hidden[:, :: max(1, D // 6)] *= 8.0  # a few channels stand out, as they do behind a model's last layer
    s = {"case": case, "hidden": _wider(hidden, case["pad"], T), "bias": None, "residual": None}
    s["weight"] = (_randn(gen, M, D) / math.sqrt(D)).to(T)
    if case["bias"]:
        s["bias"] = (0.5 * _randn(gen, M)).to(T)
    if case["residual"]:
        s["residual"] = _wider(_randn(gen, N, M), case["pad"], T)
    if case["kind"] == "train":
        size = (1_024.0 if case["dtype"] == "f16" else 1.0) / N
        s["grad_out"] = (_randn(gen, N, M) * size * torch.exp(_randn(gen, N, 1))).to(T)
    return s


def prepare(case, seed):
    return (_prepare_logits if case["kind"] in ("score", "policy") else _prepare_layer)(case, seed)


# ---------------------------------------------------------------- the plain forms


def _plain_score(s):
    case = s["case"]
    x, t = s["logits"].float(), s["tokens"].long()
    N, V = x.shape
    if s["bits"] is not None:
        x = x.masked_fill(~_admits(s["bits"], s["c"]), NINF)
    z = x / case["temperature"]
    most = z.amax(1, keepdim=True)
    shift = torch.where(most > NINF, most, torch.zeros_like(most))
    e = torch.exp(z - shift)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    there = (t >= 0) & (t < V)
    at = t.clamp(0, V - 1)
    z_t = torch.gather(z, 1, at)
    counts = there & (z_t > NINF)
    logprob = torch.where(counts, (z_t - shift) - log_total, torch.where(there, NINF, 0.0))
    p = torch.where(total > 0, e / total, torch.zeros_like(e))
    log_p = torch.where(p > 0, (z - shift) - log_total, torch.zeros_like(z))
    entropy = -(p * log_p).sum(1)
    out = {"logprob": logprob, "entropy": entropy, "stats": torch.cat([x.amax(1, keepdim=True), log_total], 1)}
    if case["top"]:
        # one whole number for value and place: larger for larger logits, and of equal ones for the lower token
        b = (x + 0.0).view(torch.int32).long()
        order = torch.where(b >= 0, b, -(b & 0x7FFFFFFF))
        key, _ = torch.topk(order * 2**20 + (2**20 - 1 - torch.arange(V, device=x.device)), min(case["top"], V), dim=1)
        token = 2**20 - 1 - key % 2**20
        value = torch.gather(z, 1, token)
        more = value > NINF
        out["top_tokens"] = torch.where(more, token, -torch.ones_like(token)).to(torch.int32)
        out["top_logprobs"] = torch.where(more, (value - shift) - log_total, NINF)
    return out, p, log_p, at, counts


def _plain_policy(s):
    out, p, log_p, at, counts = _plain_score(s)
    g = torch.where(counts, s["grad_logprob"], torch.zeros_like(s["grad_logprob"]))
    d = -p * (g.sum(1, keepdim=True) + s["grad_entropy"][:, None] * (log_p + out["entropy"][:, None]))
    d.scatter_add_(1, at, g)
    out["grad_logits"] = (d / s["case"]["temperature"]).to(s["logits"].dtype)
    return out


def _plain_activation(act, z, slope):
    """act(z), and act'(z) where it is asked for"""
    if act == "none":
        return z, torch.ones_like(z) if slope else None
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z)), (z > 0).to(z.dtype) if slope else None
    if act == "silu":
        y = 1.0 / (1.0 + torch.exp(-z))
        return z * y, y * (1.0 + z * (1.0 - y)) if slope else None
    if act == "gelu":
        half = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
        return z * half, half + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi) if slope else None
    k = math.sqrt(2.0 / math.pi)
    y = torch.tanh(k * (z + 0.044715 * z * z * z))
    d = 0.5 * (1.0 + y) + 0.5 * z * (1.0 - y * y) * k * (1.0 + 3 * 0.044715 * z * z) if slope else None
    return 0.5 * z * (1.0 + y), d


def _plain_layer(s):
    case, T = s["case"], s["hidden"].dtype
    train = case["kind"] == "train"
    hidden, weight = s["hidden"].float(), s["weight"].float()
    z = hidden @ weight.t()
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y, slope = _plain_activation(case["act"], z, train)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = {"out": y.to(T)}
    if train:
        dz = s["grad_out"].float() * slope
        out["grad_hidden"], out["grad_weight"] = (dz @ weight).to(T), (dz.t() @ hidden).to(T)
        if s["bias"] is not None:
            out["grad_bias"] = dz.sum(0).to(T)
    return out


# ---------------------------------------------------------------- one pass


def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        if kind == "score":
            return _plain_score(s)[0]
        return _plain_policy(s) if kind == "policy" else _plain_layer(s)

    import paper_2605_29986_amd as cfgzip
    if kind in ("score", "policy"):
        how = {"temperature": case["temperature"]}
        if s["bits"] is not None:
            how.update(bits=s["bits"], class_of_token=s["c"], C=case["C"])
        logprob, entropy, stats, top_tokens, top_logprobs = cfgzip.cfgzip_token_logprobs(s["logits"], s["tokens"], top=case["top"], **how)
        out = {"logprob": logprob, "entropy": entropy, "stats": stats}
        if case["top"]:
            out.update(top_tokens=top_tokens, top_logprobs=top_logprobs)
        if kind == "policy":
            out["grad_logits"] = cfgzip.cfgzip_token_logprobs_grad(s["logits"], s["tokens"], logprob, stats, s["grad_logprob"], entropy=entropy,
                                                                   grad_entropy=s["grad_entropy"], **how)
        return out
    act = None if case["act"] == "none" else case["act"]
    train = kind == "train"
    y, slope = cfgzip.cfgzip_head_layer(s["hidden"], s["weight"], s["bias"], activation=act, residual=s["residual"],
                                        want_slope=train and act is not None)
    out = {"out": y}
    if train:
        gh, gw, gb = cfgzip.cfgzip_head_layer_grad(s["hidden"], s["weight"], s["grad_out"], slope=slope, want_bias=case["bias"])
        out["grad_hidden"], out["grad_weight"] = gh, gw
        if case["bias"]:
            out["grad_bias"] = gb
    return out


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    """Bytes: every input read once, every output written once.  Operations: one product forwards, two for the gradients."""
    N = case["N"]
    if case["kind"] in ("score", "policy"):
        V, C, n = case["V"], case["C"], case["n"]
        size = 4 if case["dtype"] == "f32" else 2
        total = size * N * V + (4 * V + 4 * N * _words(C) if C else 0) + N * (8 * n + 8 + 8 * case["top"])
        return {"bytes": total + (size * N * V + 4 * N * (n + 1) if case["kind"] == "policy" else 0), "flops": 0}
    M, D = case["M"], case["D"]
    total = 2 * (N * D + M * D + N * M) + (2 * M if case["bias"] else 0) + (2 * N * M if case["residual"] else 0)
    if case["kind"] == "layer":
        return {"bytes": total, "flops": 2 * N * M * D}
    return {"bytes": total + 2 * (N * M + N * D + M * D) + (2 * M if case["bias"] else 0), "flops": 6 * N * M * D}


# ---------------------------------------------------------------- the definition in 64 bits


def _exact_rows(s, lo, hi):
    """The results of the rows lo..hi."""
    case = s["case"]
    V = case["V"]
    raw = s["logits"][lo:hi].double()
    if s["bits"] is not None:
        octets = s["bits"][lo:hi].contiguous().view(torch.uint8).short()
        k = s["c"].long()
        raw[(octets[:, k // 8].bitwise_right_shift((k % 8).short()) & 1) == 0] = NINF
    z = raw / case["temperature"]
    lse = torch.logsumexp(z, 1)
    t = s["tokens"][lo:hi].long()
    none = (t < 0) | (t >= V)
    z_t = torch.gather(z, 1, torch.where(none, 0, t))
    logprob = torch.where(z_t == NINF, NINF, z_t - lse[:, None])
    logprob[none] = 0.0
    log_p = torch.where(z == NINF, NINF, z - lse[:, None])
    p = torch.exp(log_p)
    entropy = -torch.special.xlogy(p, p).sum(1)
    most = raw.max(1).values
    log_sum = torch.where(most == NINF, NINF, lse - most / case["temperature"])
    out = {"logprob": logprob, "entropy": entropy, "stats": torch.stack([most, log_sum], 1)}
    if case["top"]:
        value, token = torch.sort(raw, dim=1, descending=True, stable=True)
        value, token = value[:, :case["top"]], token[:, :case["top"]]
        out["top_tokens"] = torch.where(value == NINF, -1, token).to(torch.int32)
        out["top_logprobs"] = torch.where(value == NINF, NINF, value / case["temperature"] - lse[:, None])
    if case["kind"] == "policy":
        g = s["grad_logprob"][lo:hi].double().clone()
        g[none | (z_t == NINF)] = 0.0
        # of each given token in turn: one at its place less the probabilities
        d = -g.sum(1, keepdim=True) * p
        rows = torch.arange(hi - lo, device=d.device)
        for j in range(t.shape[1]):
            d[rows, torch.where(none[:, j], 0, t[:, j])] += g[:, j]
        d -= s["grad_entropy"][lo:hi, None].double() * (torch.special.xlogy(p, p) + p * entropy[:, None])
        out["grad_logits"] = d / case["temperature"]
    return out


def _exact_activation(act, z):
    """(act(z), act'(z))"""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0.0), torch.where(z > 0, 1.0, 0.0)
    if act == "silu":
        q = torch.sigmoid(z)
        return z * q, q + z * q * torch.sigmoid(-z)
    if act == "gelu":
        q = 0.5 * torch.erfc(-z / math.sqrt(2.0))
        return z * q, q + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    # (1 + tanh u) / 2 is the logistic function of 2 u
    c = 2.0 * math.sqrt(2.0 / math.pi)
    q = torch.sigmoid(c * (z + 0.044715 * z**3))
    return z * q, q + z * q * (1.0 - q) * c * (1.0 + 0.134145 * z**2)


def exact(case, seed):
    s = prepare(case, seed)
    N = case["N"]
    if case["kind"] in ("score", "policy"):
        step = max(1, 2**26 // case["V"])
        parts = [_exact_rows(s, i, min(N, i + step)) for i in range(0, N, step)]
        return {name: torch.cat([p[name] for p in parts]) for name in parts[0]}
    hidden, weight = s["hidden"].double(), s["weight"].double()
    z = torch.mm(hidden, weight.t().contiguous())
    if s["bias"] is not None:
        z += s["bias"].double()
    y, slope = _exact_activation(case["act"], z)
    out = {"out": y if s["residual"] is None else y + s["residual"].double()}
    if case["kind"] == "train":
        dz = s["grad_out"].double() * slope
        out["grad_hidden"] = torch.mm(dz, weight)
        out["grad_weight"] = torch.mm(dz.t().contiguous(), hidden)
        if s["bias"] is not None:
            out["grad_bias"] = dz.sum(0)
    return out
