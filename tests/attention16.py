"""64-bit references of the paged and prompt attention operators, and the tolerances of their outputs."""
import math

import torch

D = 128
# unit roundoff: the most, relative, that rounding to the type moves a value (8 and 11 significant bits)
ROUNDOFF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def attend(q, k, v, seen, scale):
    """q [rows][hq][128], k, v [keys][hkv][128], seen [rows] = keys that each row sees (the first ones).
    Returns out, lse and what bounds the error: the average |v| and the largest sum of |q k| of a row."""
    q, k, v = q.double(), k.double(), v.double()
    rows, hq, keys, hkv = q.shape[0], q.shape[1], k.shape[0], k.shape[1]
    g = hq // hkv
    qg = q.view(rows, hkv, g, D)
    s = torch.einsum("rhgd,khd->hgrk", qg, k) * scale
    size = torch.einsum("rhgd,khd->hgrk", qg.abs(), k.abs()) * scale
    mask = torch.arange(keys, device=q.device)[None, :] < seen[:, None]
    s = s.masked_fill(~mask, -math.inf)
    top = s.amax(-1, keepdim=True) if keys else torch.full((hkv, g, rows, 1), -math.inf, dtype=s.dtype, device=s.device)
    p = torch.where(mask, torch.exp(s - torch.where(top == -math.inf, 0.0, top)), 0.0)
    total = p.sum(-1, keepdim=True)
    w = p / torch.where(total == 0, 1.0, total)
    out = torch.einsum("hgrk,khd->rhgd", w, v).reshape(rows, hq, D)
    mean = torch.einsum("hgrk,khd->rhgd", w, v.abs()).reshape(rows, hq, D)
    lse = (top + torch.log(total)).squeeze(-1).permute(2, 0, 1).reshape(rows, hq)
    big = torch.where(mask, size, 0.0).amax(-1) if keys else torch.zeros((hkv, g, rows), device=q.device).double()
    return out, lse, mean, big.permute(2, 0, 1).reshape(rows, hq)


def check(got, lse, ref, dtype, keys, vmax):
    """out: its own rounding, the probabilities' rounding to the type, and the scores' error in binary32 (a dot
    product of 128 terms, at most 2^-17 of the sum of its terms' sizes; so does exp's argument move, up and down);
    FP16 probabilities below 2^-14 lose up to 2^-25 of the largest each.  lse: the scores' error and binary32's."""
    out, rlse, mean, big = ref
    u = ROUNDOFF[dtype]
    delta = 2.0 ** -17 * big + 2.0 ** -20
    tol = u * out.abs() + (u + 2.0 * delta[..., None]) * mean * 1.01 + 2.0 ** -25
    if dtype == torch.float16:
        tol = tol + 2.0 ** -25 * keys * vmax
    err = (got.double() - out).abs()
    bad = ~(err <= tol)
    assert not bad.any(), "out: %d of %d off, worst %g of its tolerance" % (bad.sum(), bad.numel(), (err / tol).nan_to_num(9e9).max())
    if lse is not None:
        empty = rlse == -math.inf
        assert torch.equal(lse.double() == -math.inf, empty)
        err = (lse.double() - rlse).abs()[~empty]
        tol = (delta + 2.0 ** -22 * rlse.abs() + 2.0 ** -20)[~empty]
        assert bool((err <= tol).all()), "lse: worst %g of its tolerance" % (err / tol).max()


def turned(x, table, pos, rot_dim, interleaved, sections):
    """x [tokens][heads][128] rotated in 64 bits; pos [tokens] or [3][tokens] int32."""
    half = rot_dim // 2
    y = x.double().clone()
    t = table.double()
    pos = pos.long().clamp(0, table.shape[0] - 1)
    for i in range(half):
        p = pos if sections is None else pos[0 if i < sections[0] else 1 if i < sections[0] + sections[1] else 2]
        c, s = t[p, i][:, None], t[p, half + i][:, None]
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        xa, xb = x[..., a].double(), x[..., b].double()
        y[..., a], y[..., b] = xa * c - xb * s, xa * s + xb * c
    return y


def check_turned(got, x, want, dtype):
    """One rounding to the type of a binary32 result whose two products are each up to the pair's size."""
    tol = ROUNDOFF[dtype] * want.abs() + 2.0 ** -22 * 2 * x.double().abs().amax() + 2.0 ** -25
    assert bool(((got.double() - want).abs() <= tol).all())


def table(length, rot_dim, device):
    half = rot_dim // 2
    a = torch.arange(length, dtype=torch.float64, device=device)[:, None] * 1e4 ** (-torch.arange(half, dtype=torch.float64, device=device) / half)
    return torch.cat([a.cos(), a.sin()], 1).float()
