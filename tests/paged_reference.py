"""The operators on the paged cache, stated plainly in 64 bits (test infrastructure; torch tensors on any device).

Shares nothing with the kernels: codes are taken apart bit by bit, angles are evaluated as complex exponentials, the
attention is a softmax over a row's gathered positions.
"""
from __future__ import annotations

import math

import torch

# Half a step of each type, relative to the value.
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def round16(n):
    return -(-n // 16) * 16


def code_values(codes):
    """uint8 codes (1 sign, 4 exponent, 3 mantissa bits, bias 7) -> doubles."""
    c = codes.long()
    field, frac = (c >> 3) & 15, (c & 7).double()
    mag = torch.where(field == 0, frac * 2.0 ** -9, (8 + frac) * torch.ldexp(torch.ones_like(frac), field - 10))
    mag = torch.where((c & 127) == 127, torch.full_like(mag, math.nan), mag)
    return torch.where(c >= 128, -mag, mag)


def pool_values(pool, H, B, D):
    """A pool's blocks as doubles [n_blocks, H, B, D] (uint8: the 8-bit layout)."""
    if pool.dtype != torch.uint8:
        return pool.double()
    n = pool.shape[0]
    v = code_values(pool[:, : H * B * D].reshape(n, H, B, D))
    e = pool[:, H * B * D: H * B * D + H * B].reshape(n, H, B, 1).long() - 127
    return torch.ldexp(v, e)


def row_values(values, table, r, n):
    """Positions 0 .. n of row r from pool_values' blocks: [H, n, D]."""
    B = values.shape[2]
    nb = -(-n // B)
    return values[table[r, :nb].long()].permute(1, 0, 2, 3).flatten(1, 2)[:, :n]


def attend(q, k_rows, v_rows, scale):
    """q [Hq, D], k_rows / v_rows [H, n, D] doubles -> out [Hq, D], lse [Hq], and the sums the error bounds need."""
    H, n, D = k_rows.shape
    Hq = q.shape[0]
    qq = q.double().view(H, Hq // H, D)
    if n == 0:
        z = torch.zeros(Hq, D, dtype=torch.float64, device=q.device)
        return z, torch.full((Hq,), -math.inf, dtype=torch.float64, device=q.device), z, torch.zeros_like(z[:, 0])
    s = torch.einsum("hgd,hnd->hgn", qq, k_rows) * scale
    p = torch.softmax(s, -1)
    out = torch.einsum("hgn,hnd->hgd", p, v_rows).reshape(Hq, D)
    absv = torch.einsum("hgn,hnd->hgd", p, v_rows.abs()).reshape(Hq, D)
    reach = torch.einsum("hgd,hnd->hgn", qq.abs(), k_rows.abs()).amax(-1).reshape(Hq) * abs(scale)
    return out, torch.logsumexp(s, -1).reshape(Hq), absv, reach


def attend_bound(out, absv, reach, n, D, dtype, weight_step):
    """How far an attention in 32-bit sums may be off, elementwise.

    A score is a sum of D products, each rounded at most once on the way into it and once when it is added: (D + 2) u
    reach, with u = 2^-24; its scaling, and the exponent formed from it, add at most 8 u (1 + reach) more (values up to
    2 reach log2 e, rounded twice), the exponential itself 4 u.  So a weight is off by eps_w = (D + 10) u reach + 12 u of
    itself, plus weight_step where it is rounded for the matrix unit.  Numerator and denominator are sums of n terms,
    joined in a tree over at most 64 partial results: (n + 64) u each.  The quotient is rounded into dtype.
    """
    u = 2.0 ** -24
    eps = 2 * ((D + 10) * u * reach + 12 * u + (n + 64) * u) + weight_step
    return 1.01 * (eps[:, None] * (absv + out.abs()) + HALF_STEP[dtype] * out.abs()) + 1e-30


def rotate(x, pos, freqs, layout, mscale=1.0):
    """x [n, heads, D] -> doubles with rotary positions."""
    rot = 2 * len(freqs)
    angle = pos.double()[:, None, None] * freqs.double()[None, None, :]
    unit = torch.polar(torch.full_like(angle, mscale), angle)
    y = x.double().clone()
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    w = torch.complex(y[..., a].contiguous(), y[..., b].contiguous()) * unit
    y[..., a], y[..., b] = w.real, w.imag
    return y


def quantise(x):
    """[.., D] doubles -> (scale exponents [..], nearest 8-bit values times the scale [.., D])."""
    fin = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x))
    top = fin.amax(-1)
    e = torch.full(top.shape, -60, dtype=torch.long, device=x.device)
    for cand in range(-60, 60):  # smallest exponent that is enough, by trying all
        e = torch.where(top > 448.0 * 2.0 ** cand, torch.full_like(e, cand + 1), e)
    s = torch.ldexp(torch.ones_like(top), e)[..., None]
    y = x / s
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    q = (torch.round(y / step) * step).clamp(-448, 448)
    return e, torch.where(torch.isfinite(x), q, torch.full_like(q, math.nan)) * s
