"""Plain 64-bit forms of cfgzip_head_layer and cfgzip_head_layer_grad (torch, on whatever device the inputs are) and the bounds that their tests
hold the kernels to.

fp32 steps are off by at most F32 = 2^-24 of their result; a sum of n products by at most n of those of the sum of their sizes; exponential and
reciprocal instructions by two, erfc by sixteen.  A rounding to a type is off by at most half a step, HALF_STEP of the value."""

import math

import torch

from head_reference import F32, HALF_STEP, SMALLEST_HALF_STEP

ACTIVATIONS = [None, "relu", "gelu", "gelu_tanh", "silu"]
FLOOR = 2.0 ** -126  # fp32 results below the smallest normal number may be 0


def activation(name, z):
    """(act(z), act'(z))"""
    if name is None:
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0.0), (z > 0).to(z.dtype)
    if name == "gelu":
        q = 0.5 * torch.erfc(-z / math.sqrt(2.0))
        return z * q, q + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    a, b = (1.0, 0.0) if name == "silu" else (2.0 * math.sqrt(2.0 / math.pi), 2.0 * math.sqrt(2.0 / math.pi) * 0.044715)
    q = torch.sigmoid(z * (a + b * z * z))
    return z * q, q + z * q * (1.0 - q) * (a + 3.0 * b * z * z)


def activation_errors(name, z):
    """What the steps of act and act' in fp32 are off by, of an exact z"""
    if name in (None, "relu"):
        return torch.zeros_like(z), torch.zeros_like(z)
    if name == "gelu":
        q = 0.5 * torch.erfc(-z / math.sqrt(2.0))
        q_err = q * F32 * (3.0 * z * z + 40.0)  # the argument's two steps, times 2 x of erfc(x); erfc's own
        phi = z.abs() * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
        return z.abs() * q_err + F32 * (z * q).abs() + FLOOR, q_err + phi * F32 * (2.0 * z * z + 10.0) + 2 * F32 * (q + phi) + FLOOR
    a, b = (1.0, 0.0) if name == "silu" else (2.0 * math.sqrt(2.0 / math.pi), 2.0 * math.sqrt(2.0 / math.pi) * 0.044715)
    u, t = (z * (a + b * z * z)).abs(), a + 3.0 * b * z * z
    q = torch.sigmoid(z * (a + b * z * z))
    # u: four steps, its factor and product two more; the exponential, the sum and the reciprocal
    q_err = q * (1.0 - q) * F32 * (6.0 * u + 3.0) + q * F32 * 4.0 + FLOOR
    y_err = z.abs() * q_err + F32 * (z * q).abs() + FLOOR
    s_err = q_err * (1.0 + z.abs() * t * (1.0 - 2.0 * q).abs()) + z.abs() * t * q * F32 + z.abs() * t * q * (1.0 - q) * 8.0 * F32 + 2.0 * F32 * q + FLOOR
    return y_err, s_err


def slopes(codes):
    """What int16 slopes stand for"""
    q = codes.double()
    return q * q.abs() * 2.0 ** -28


def forward(x, w, bias, name, residual, dtype):
    """Everything in float64 (bias and residual may be None); dtype: of the result.  (out, its errors' bound, slope, its errors' bound)"""
    D = x.shape[1]
    z = torch.mm(x, w.t().contiguous())
    size = torch.mm(x.abs(), w.abs().t().contiguous())
    z_err = size * (D + 64) * F32
    if bias is not None:
        z = z + bias
        z_err = z_err + F32 * z.abs() + F32 * z_err
    y, s = activation(name, z)
    y_err, s_err = activation_errors(name, z)
    # (slopes reach 1.13, and act'' 0.85)
    y_err, s_err = y_err + 1.13 * z_err, s_err + (0.85 * z_err if name not in (None, "relu") else 0.0)
    if name == "relu":  # on either side of 0
        s_err = torch.where(z.abs() <= z_err, torch.ones_like(z), torch.zeros_like(z))
    s_err = s_err + (s.abs() + s_err).sqrt() * 2.0 ** -14 * 1.01 + 2.0 ** -30  # (half a step of 2^-14 of the root)
    if residual is not None:
        y = y + residual
        y_err = y_err + F32 * y.abs()
    return y, y_err * 1.01 + HALF_STEP[dtype] * y.abs() * 1.01 + SMALLEST_HALF_STEP[dtype], s, s_err


def gradients(x, w, grad_out, slope, dtype, exact):
    """slope: the call's own, or None.  exact: dz is grad_out as it is.  dict of (value, bound on its errors)"""
    N, D = x.shape
    M = w.shape[0]
    dz = grad_out if slope is None else grad_out * slope
    u, floor = HALF_STEP[dtype], SMALLEST_HALF_STEP[dtype]
    dz_err = torch.zeros_like(dz)
    if not exact:
        dz_err = (u * 1.01 + F32) * dz.abs() + (float(grad_out.abs().max()) * 2.0 ** -38 if dtype == "f16" else 2.0 ** -134)
    if slope is None and dtype == "bf16" and bool((grad_out.bfloat16().double() == grad_out).all()):
        dz_err = torch.zeros_like(dz)
    a = dz.abs()
    gh, gw, gb = torch.mm(dz, w), torch.mm(dz.t().contiguous(), x), dz.sum(0)
    gh_err = torch.mm(dz_err, w.abs()) + torch.mm(a, w.abs()) * (M + 64) * F32
    gw_err = torch.mm(dz_err.t().contiguous(), x.abs()) + torch.mm(a.t().contiguous(), x.abs()) * (N + 64) * F32
    gb_err = a.sum(0) * (N + 64) * F32
    return {name: (v, e * 1.01 + u * v.abs() * 1.01 + floor) for name, v, e in (("grad_hidden", gh, gh_err), ("grad_weight", gw, gw_err),
                                                                               ("grad_bias", gb, gb_err))}
