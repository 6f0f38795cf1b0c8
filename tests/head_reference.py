"""Plain 64-bit forms of the vocabulary projection's calls (numpy, on the CPU) and the bounds that their tests hold the kernels to.

A rounding to a type is off by at most half a step, HALF_STEP relative to the value; fp32 sums of n terms by at most n times
2^-24 times the sum of the terms' sizes."""

import numpy as np

from synthetic_inputs.configs import words_for

F32 = 2.0 ** -24
HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": F32}
SMALLEST_HALF_STEP = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25, "f32": 2.0 ** -150}  # of subnormal values


def unpack(bits, n):
    """bool [R][n] of int32 [R][W(n)]"""
    octets = np.ascontiguousarray(bits).view(np.uint8)
    return np.unpackbits(octets, axis=1, bitorder="little")[:, :n].astype(bool)


def pack(rows):
    """int32 [R][W(n)] of bool [R][n], pad bits 1 (they are ignored)"""
    R, n = rows.shape
    full = np.ones((R, words_for(n) * 32), dtype=bool)
    full[:, :n] = rows
    return np.packbits(full, axis=1, bitorder="little").view(np.int32).copy()


def loss_and_gradients(h, w, target, allowed, grad_loss, dtype):
    """h [N][D], w [V][D] as float64 values of `dtype`; allowed bool [N][V]; dict of results and of bounds on their errors.
    Rows without a gradient may hold anything in h."""
    N, D = h.shape
    V = w.shape[0]
    with np.errstate(all="ignore"):
        z = h @ w.T
        size = np.abs(h) @ np.abs(w).T
        zm = np.where(allowed, z, -np.inf)
        most = np.max(zm, axis=1)
        shift = np.where(np.isfinite(most), most, 0.0)
        e = np.where(allowed, np.exp(zm - shift[:, None]), 0.0)
        lse = np.where(np.isnan(e.sum(1)), np.nan, shift + np.log(e.sum(1)))
        has = (target >= 0) & (target < V)
        at = np.clip(target, 0, V - 1)
        rows = np.arange(N)
        ok = has & allowed[rows, at]
        loss = np.where(ok, lse - z[rows, at], np.where(has, np.inf, 0.0))
        # a logit: D products summed; the sum of exponentials: chains of at most 32 + 2 + V / 1024 + 32 additions, each term with
        # the errors of its logit, of exp (argument rounded, times log2 e rounded, exp2: 4 steps of the argument and 4 of the result)
        z_err = np.max(np.where(allowed, size, 0.0), axis=1) * (D + 4) * F32
        spread = np.max(np.where(allowed & np.isfinite(zm), shift[:, None] - zm, 0.0), axis=1)
        sum_err = (66 + V / 1024 + 4 * np.minimum(spread, 100.0) + 8) * F32
        lse_err = z_err + sum_err + 4 * F32 * (np.abs(lse) + np.abs(shift))
        # (the losses of rows without a target, or with one that is not admitted, are exact)
        loss_err = np.where(ok, lse_err + size[rows, at] * (D + 4) * F32 + 2 * F32 * np.abs(loss), 0.0)
        out = {"lse": lse, "lse_err": lse_err, "loss": loss, "loss_err": loss_err}
        if grad_loss is None:
            return out
        live = ok & (grad_loss != 0)
        g = np.where(live, grad_loss, 0.0)
        h0 = np.where(live[:, None], h, 0.0)
        p = np.where(live[:, None] & allowed, np.exp(zm - np.where(live, lse, 0.0)[:, None]), 0.0)
    dz = p.copy()
    dz[rows[live], at[live]] -= 1.0
    dz *= g[:, None]
    u = HALF_STEP[dtype]
    p_err = z_err + lse_err + (4 * (spread + np.abs(np.where(live, lse - shift, 0.0))) + 8) * F32
    p_err = np.where(live, p_err, 0.0)
    biggest = np.max(np.abs(g)) if N else 0.0
    # dz is rounded to the type; in fp16 the largest row gradient lies between 2^13 and 2^14 then
    dz_err = u * np.abs(dz) + np.abs(g)[:, None] * (p * p_err[:, None] + 2 * F32) + (biggest * 2.0 ** -38 if dtype == "f16" else 0.0)
    dz_err = np.where(live[:, None] & allowed, dz_err, 0.0)
    gh, gw = dz @ w, dz.T @ h0
    out["grad_hidden"], out["grad_weight"] = gh, gw
    floor = SMALLEST_HALF_STEP[dtype]
    out["grad_hidden_err"] = (dz_err @ np.abs(w)) * 1.01 + (np.abs(dz) @ np.abs(w)) * (V + 64) * F32 + u * np.abs(gh) * 1.01 + floor
    out["grad_weight_err"] = (dz_err.T @ np.abs(h0)) * 1.01 + (np.abs(dz).T @ np.abs(h0)) * (N + 64) * F32 + u * np.abs(gw) * 1.01 + floor
    return out


VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize(x):
    """(codes uint8 [R][16 nb], scales uint8 [R][nb]) of float64 x [R][K], by the definition: the nearest value, ties to the even code"""
    R, K = x.shape
    nb = (K + 31) // 32
    full = np.zeros((R, nb * 32))
    full[:, :K] = x
    b = full.reshape(R, nb, 32)
    most = np.max(np.abs(b), axis=2)
    bad = ~np.isfinite(most)
    safe = np.where(bad | (most == 0), 1.0, most)
    e = np.where(most == 0, -127, np.maximum(np.frexp(safe)[1] - 1 - 2, -127))
    y = np.abs(np.where(bad[..., None], 0.0, b)) / np.ldexp(1.0, e)[..., None]
    far = np.abs(y[..., None] - VALUES)
    # the nearest; of two as near the even code: a little more weight for odd ones, exactly on ties only
    nearest = far.min(-1, keepdims=True)
    tied = far == nearest
    even = tied & (np.arange(8) % 2 == 0)
    index = np.where(even.any(-1), even.argmax(-1), tied.argmax(-1))
    code = (index + 8 * np.signbit(b)).astype(np.uint8)
    code[bad] = 0
    codes = (code[..., 0::2] | code[..., 1::2] << 4).reshape(R, nb * 16)
    return codes, np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes, scales, K):
    R, nb = scales.shape
    c = codes.reshape(R, nb, 16)
    code = np.stack([c & 15, c >> 4], -1).reshape(R, nb, 32)
    v = np.where(code > 7, -1.0, 1.0) * VALUES[code & 7] * np.ldexp(1.0, scales.astype(np.int64) - 127)[..., None]
    v = np.where(scales[..., None] == 255, np.nan, v)
    return v.reshape(R, nb * 32)[:, :K]
