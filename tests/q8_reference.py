"""The 8-bit operators from their definitions, in 64 bits on the CPU."""
import numpy as np
import torch

STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half a step, relative


def quantised(p: torch.Tensor):
    """``p`` float64 [tokens, h] -> (q int8, a float64): q = nearest integer to 127 p / a, ties to even; rows of zeros and rows
    that are not finite give zeros."""
    a = p.abs().amax(-1)
    good = torch.isfinite(p).all(-1) & (a > 0)
    q = torch.round(127.0 * torch.where(good[:, None], p, 0.0) / torch.where(good, a, 1.0)[:, None])
    return q.to(torch.int8), a


def rmsnorm(x, weight, eps, residual=None):
    s = x.double()
    if residual is not None:
        # the sum in 32 bits is exact or rounded once, then rounded to the type, as the definition has it
        s = (x.float() + residual.float()).to(x.dtype)
        held = s
        s = s.double()
    p = s * weight.double()
    q, a = quantised(torch.where(torch.isfinite(s), p, torch.nan))
    scale = a / torch.sqrt((s * s).mean(-1) + eps) / 127.0
    return (q, scale) if residual is None else (q, scale, held)


def silu_mul(gate, up):
    g = gate.double()
    q, a = quantised(g / (1.0 + torch.exp(-g)) * up.double())
    return q, a / 127.0


def rows(x):
    q, a = quantised(x.double())
    return q, a / 127.0


def dense_of(values, indices, k, tile_t):
    """int8 [c_out, kk], uint16 [n_tiles, kk] -> float64 [c_out, k]"""
    values, indices = np.asarray(values), np.asarray(indices).astype(np.int64)
    out = np.zeros((values.shape[0], k))
    for o in range(values.shape[0]):
        out[o, indices[o // tile_t]] = values[o]
    return out


def linear_limits(x, x_scale, dense, w_scale, bias, dtype):
    """(y, limit): the product in 64 bits and how far a result in `dtype` may be: the sum's conversion and the product with
    the token's scale are rounded to 32 bits each, the channel's scale and the bias go in with one more rounding, then the type's."""
    prod = (x.astype(np.float64) @ dense.T) * x_scale.astype(np.float64)[:, None] * w_scale.astype(np.float64)
    y = prod + (bias.astype(np.float64) if bias is not None else 0.0)
    u = 2.0 ** -24
    half = STEP[dtype] if dtype != torch.float32 else 0.0
    least = 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -126   # half of the least number, with room
    limit = np.abs(prod) * 2.0 * u * (1 + 4 * u) + np.abs(y) * u
    return y, limit + (np.abs(y) + limit) * half + least
