"""Plain 64-bit forms of cfgzip_token_logprobs and cfgzip_token_logprobs_grad (numpy, on the CPU) and the bounds that their tests hold the
kernels to.

fp32 steps are off by at most F32 = 2^-24 of their result, the exponential and logarithm instructions by two such steps.  With z the logits
divided by the temperature and d = z - (the largest admitted z):
  an exponential    3 (difference, factor, product) |d| + 4 (its own, its sum with others' errors in what raises it)
  a raise           of what was summed to a larger maximum: the differences add up to |d| again, 6 for each; at most one a unit of eight
                    logits that a thread takes, and two where threads and workgroups are joined
  a sum             8 additions a unit of a thread, 24 where threads and workgroups are joined
  sum of d exp(d)   of d that are larger by up to the 8 that a thread's sums may be apart from its largest logit, which are taken back
all in F32, relative to the sum; terms further than 100 from the largest are nothing in any case."""

import numpy as np

from head_reference import F32, HALF_STEP, SMALLEST_HALF_STEP

THREADS = 512  # of a workgroup


def logprobs(x, tokens, allowed, temperature, top):
    """x float64 [N][V], tokens int [N][n], allowed bool [N][V] by the masks; dict of results and of bounds on their errors"""
    N, V = x.shape
    n = tokens.shape[1]
    with np.errstate(all="ignore"):
        admitted = allowed & (x != -np.inf)
        xm = np.where(admitted, x, -np.inf)
        most = xm.max(1)
        some = most > -np.inf
        d = np.where(admitted, (x - np.where(some, most, 0.0)[:, None]) / temperature, -np.inf)
        e = np.exp(d)
        s = e.sum(1)
        log_s = np.where(some, np.log(np.where(some, s, 1.0)), -np.inf)
        p = np.where(admitted, e / np.where(some, s, 1.0)[:, None], 0.0)
        log_p = np.where(admitted, d - np.where(some, log_s, 0.0)[:, None], -np.inf)
        plogp = np.where(p > 0, p * np.where(p > 0, log_p, 0.0), 0.0)
        entropy = -plogp.sum(1)
    rounds = -(-V // (8 * THREADS))
    spread = np.where(some, np.minimum(np.max(np.where(admitted, -np.where(admitted, d, 0.0), 0.0), axis=1), 100.0), 0.0)
    s_err = F32 * (6 * spread + 6 * (rounds + 2) + 4 + 8 * rounds + 24)
    log_err = s_err + 4 * F32 * (np.where(some, np.abs(log_s), 0.0) + 1)
    weight = np.where(p > 0, p * np.where(p > 0, -d, 0.0), 0.0).sum(1)
    out = {"stats": np.stack([most, log_s], 1), "log_sum_err": log_err, "entropy": entropy,
           "entropy_err": log_err + (weight + 8) * (2 * s_err + 8 * F32) + 2 * F32 * np.abs(entropy),
           "p": p, "log_p": log_p, "d": d, "admitted": admitted, "some": some}
    inside = (tokens >= 0) & (tokens < V)
    at = np.clip(tokens, 0, V - 1)
    rows = np.arange(N)[:, None]
    ok = inside & admitted[rows, at] if n else np.zeros((N, 0), bool)
    lp = np.where(ok, log_p[rows, at], np.where(inside, -np.inf, 0.0)) if n else np.zeros((N, 0))
    out["counts"], out["logprob"] = ok, lp

    def err(values):  # of d / temperature less the logarithm
        size = np.where(np.isfinite(values), np.abs(values), 0.0)
        return 4 * F32 * (size + np.where(some, np.abs(log_s), 0.0)[:, None]) + log_err[:, None]

    out["logprob_err"] = err(lp)
    tt = np.full((N, top), -1, np.int64)
    tl = np.full((N, top), -np.inf)
    for i in range(N):
        here = np.flatnonzero(admitted[i])
        order = here[np.argsort(-x[i, here], kind="stable")][:top]
        tt[i, :len(order)], tl[i, :len(order)] = order, log_p[i, order]
    out["top_tokens"], out["top_logprobs"], out["top_err"] = tt, tl, err(tl)
    return out


def gradient(r, tokens, grad_logprob, grad_entropy, temperature, dtype):
    """(grad_logits, bound on its errors) from the dict of logprobs()"""
    N, V = r["p"].shape
    g = np.where(r["counts"], grad_logprob, 0.0)
    ge = np.zeros(N) if grad_entropy is None else grad_entropy
    live = r["some"] & ((g != 0).any(1) | (ge != 0))
    ge = np.where(live, ge, 0.0)[:, None]
    G = np.where(live, g.sum(1), 0.0)[:, None]
    H = r["entropy"][:, None]
    lp = np.where(r["p"] > 0, np.where(r["p"] > 0, r["log_p"], 0.0), 0.0)
    d = -r["p"] * (G + ge * (lp + H))
    given = np.zeros((N, V))
    size = np.zeros((N, V))
    for i in np.flatnonzero(live):
        for j in np.flatnonzero(r["counts"][i]):
            given[i, tokens[i, j]] += g[i, j]
            size[i, tokens[i, j]] += abs(g[i, j])
    out = np.where(r["admitted"], (d + given) / temperature, 0.0)
    # p: an exponential times 2^-(log S / ln 2), whose argument is off by the logarithm's error and two steps of it; the bracket: sums of parts
    log_s = np.where(r["some"], np.abs(r["stats"][:, 1]), 0.0)[:, None]
    far = np.where(r["p"] > 0, np.abs(np.where(r["p"] > 0, r["d"], 0.0)), 0.0)
    p_rel = F32 * (6 * far + 16 + 4 * log_s) + r["log_sum_err"][:, None]
    g_size = np.abs(g).sum(1)[:, None]
    parts = g_size + np.abs(ge) * (H + log_s + far)
    bracket = F32 * parts * (12 + tokens.shape[1]) + np.abs(ge) * (r["entropy_err"] + r["log_sum_err"])[:, None]
    err = (r["p"] * (parts * p_rel + bracket) + F32 * (4 + tokens.shape[1]) * size + 4 * F32 * np.abs(d + given)) / temperature
    err = err * 1.01 + HALF_STEP[dtype] * np.abs(out) * 1.01 + SMALLEST_HALF_STEP[dtype]
    # (fp32 results below the smallest normal number may be 0, and so may exponentials)
    err = err + (parts + size) / temperature * 2.0 ** -126
    return out, np.where(r["admitted"] & live[:, None], err, 0.0)
