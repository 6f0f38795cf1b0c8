"""The gradients of cfgzip_head_loss_grad in 64 bits from the lse that the call was given, and bounds on their errors that know in which
form dz and the product's other operand are kept, so that a form with fewer bits does not pass.

A rounding to a type is off by at most half a step: 2^-8 of the value in bf16, 2^-11 in fp16 (2^-25 where it is subnormal), 2^-24 in fp32."""

import numpy as np

from head_reference import F32, HALF_STEP, SMALLEST_HALF_STEP


def few_rows(N, D, dtype):
    """Whether dz is kept as two numbers"""
    return N <= (128 if dtype == "bf16" and D % 8 else 256)


def gradients(h, w, target, allowed, g, lse, dtype, few):
    """h [N][D], w [V][D] as float64 values of `dtype`, allowed bool [N][V], g and lse the call's own [N] in float64; dict of the
    gradients and bounds on their errors.  Rows without a gradient may hold anything in h."""
    N, D = h.shape
    V = w.shape[0]
    rows = np.arange(N)
    at = np.clip(target, 0, V - 1)
    live = (target >= 0) & (target < V) & allowed[rows, at] & (g != 0)
    here = live[:, None] & allowed
    g = np.where(live, g, 0.0)
    size_g = np.abs(g)[:, None]
    h = np.where(live[:, None], h, 0.0)
    z = h @ w.T
    lse = np.where(live, lse, 0.0)[:, None]
    p = np.where(here, np.exp(np.where(here, z - lse, 0.0)), 0.0)
    # a logit: D products summed in fp32; exp: its argument rounded, times log2 e rounded, exp2 (four steps of argument and result)
    z_err = (np.abs(h) @ np.abs(w).T) * (D + 4) * F32
    p_rel = z_err + (4 * np.abs(z - lse) + 8) * F32
    if few:  # from the row's own maximum and sum, brought to the lse of the call: their errors, and those of the difference
        top = np.max(np.where(here, z, -np.inf), axis=1, keepdims=True, initial=-1e30)
        top = np.where(live[:, None], top, 0.0)
        spread = np.max(np.where(here, top - z, 0.0), axis=1, keepdims=True)
        most_z = np.max(np.where(here, z_err, 0.0), axis=1, keepdims=True)
        p_rel = z_err + most_z + (66 + V / 1024 + 4 * np.minimum(spread, 100.0) + 8 + 4 * np.abs(z - top) + 8
                                  + 8 * (np.abs(lse) + np.abs(top))) * F32
    dz = p * g[:, None]
    dz[rows[live], at[live]] -= g[live]
    if few and dtype == "bf16":
        form = 2.0 ** -16 * np.abs(dz)
    elif few:  # a row's factor makes its gradient 2^14 to 2^15
        form = 2.0 ** -22 * np.abs(dz) + 2.0 ** -39 * size_g
    else:  # 2^13 to 2^15
        form = 2.0 ** -11 * np.abs(dz) + 2.0 ** -38 * size_g
        if dtype == "f16":  # of the target's element nothing is lost
            form[rows[live], at[live]] = 2 * F32 * np.abs(dz)[rows[live], at[live]]
    dz_err = np.where(here, form * 1.01 + size_g * (p * p_rel + 2 * F32), 0.0)
    w_err = np.zeros_like(w)
    if dtype == "bf16" and not few:
        most = np.max(np.abs(w))
        w_err = np.where((w != 0) & (np.abs(w) < 2.0 ** -31 * most), 2.0 ** -39 * most, 0.0)
    h_err = np.zeros_like(h)  # of g h, divided by g: the largest becomes 2^14 at the least
    if dtype == "f16" or not few:
        share = np.max(np.abs(h) * size_g, initial=0.0) * 2.0 ** -39
        h_err = np.where(live[:, None], share / np.where(live, np.abs(g), 1.0)[:, None], 0.0)
    u, floor = HALF_STEP[dtype], SMALLEST_HALF_STEP[dtype]
    gh, gw = dz @ w, dz.T @ h
    return {
        "grad_hidden": gh, "grad_weight": gw,
        "grad_hidden_err": dz_err @ (np.abs(w) + w_err) + np.abs(dz) @ w_err + (np.abs(dz) @ np.abs(w)) * (V + 64) * F32
        + u * np.abs(gh) * 1.01 + floor,
        "grad_weight_err": dz_err.T @ (np.abs(h) + h_err) + np.abs(dz).T @ h_err + (np.abs(dz).T @ np.abs(h)) * (N + 64) * F32
        + u * np.abs(gw) * 1.01 + floor,
    }
