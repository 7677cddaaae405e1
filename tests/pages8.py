"""References of the 8-bit paged cache: what its pages hold, block by block, and the tolerance of attention over them."""
import math

import torch

from attention16 import D, ROUNDOFF

BLOCK = 16
F8 = torch.float8_e4m3fn
NAN_CODE = 0x7f


def power(amax):
    """The least power of two s >= 2^-126 with amax <= 448 s."""
    if amax == 0:
        return 2.0 ** -126
    part, e = math.frexp(amax)  # amax = part 2^e; 448 = 0.875 2^9
    return 2.0 ** max(e - 9 + (part > 0.875), -126)


def encode(x, s):
    """e4m3 codes (bytes) of x / s in 32 bits, nearest even; NaN and infinities are NaN."""
    y = torch.where(x.isfinite(), x.float() / s, torch.full_like(x, math.nan, dtype=torch.float32))
    return one_nan(y.to(F8).view(torch.uint8))


def one_nan(codes):
    """NaN has two codes: one for both."""
    return torch.where((codes & 0x7f) == NAN_CODE, torch.full_like(codes, NAN_CODE), codes)


def decode(codes):
    return codes.view(F8).double()


def append(codes, scales, table, length, rows):
    """One request's last rows [n][heads][D] (32 bits, CPU) into codes [pages][heads][page][D] and scales, in place."""
    size, end, first = codes.shape[2], length, length - rows.shape[0]
    for block in range(first // BLOCK, -(-end // BLOCK)):
        lo, hi = max(first, block * BLOCK), min(end, (block + 1) * BLOCK)
        at = block * BLOCK
        if at < 0 or at // size >= len(table):
            continue
        page = int(table[at // size])
        if page < 0 or page >= codes.shape[0]:
            continue
        at %= size
        for h in range(codes.shape[1]):
            x = rows[lo - first:hi - first, h]
            finite = x[x.isfinite()].abs()
            s = power(float(finite.max()) if finite.numel() else 0.0)
            if lo > block * BLOCK:
                old = float(scales[page, h, at // BLOCK])
                part, e = math.frexp(old)
                s = max(s, min(max(2.0 ** (e - (part == 0.5)) if old else 0.0, 2.0 ** -126), 2.0 ** 126))
                if s != old:
                    kept = codes[page, h, at:at + lo % BLOCK]
                    codes[page, h, at:at + lo % BLOCK] = encode(decode(kept).float() * (old / s), 1.0)
            scales[page, h, at // BLOCK] = s
            codes[page, h, lo % size:lo % size + hi - lo] = encode(x, s)


def values(codes, scales):
    """code * scale in 64 bits, [pages][heads][page][D]."""
    n, h, size, _ = codes.shape
    x = decode(codes.contiguous().view(torch.uint8)).view(n, h, size // BLOCK, BLOCK, D)
    return (x * scales.double()[..., None, None]).view(n, h, size, D)


def check(got, lse, ref, dtype, keys, top_scale):
    """out: its own rounding, the probabilities' rounding to FP16, the scores' error in binary32 (a dot product of 128
    exact products, at most 2^-17 of the sum of their sizes, and exp's argument moves up and down), and terms that FP16
    loses: a probability times its block's scale, over the largest scale (to a power of two: up to twice), is off by 2^-25
    at most where it is subnormal, of 2^7 for the largest, times a code of up to 448.  lse: the scores' error and
    binary32's."""
    out, rlse, mean, big = ref
    delta = 2.0 ** -17 * big + 2.0 ** -20
    tol = ROUNDOFF[dtype] * out.abs() + (2.0 ** -11 + 2.0 * delta[..., None]) * mean * 1.01 + 2.0 ** -25
    tol = tol + 2.0 ** -31 * 448 * top_scale * keys
    err = (got.double() - out).abs()
    bad = ~(err <= tol)
    assert not bad.any(), "out: %d of %d off, worst %g of its tolerance" % (bad.sum(), bad.numel(), (err / tol).nan_to_num(9e9).max())
    if lse is not None:
        empty = rlse == -math.inf
        assert torch.equal(lse.double() == -math.inf, empty)
        err = (lse.double() - rlse).abs()[~empty]
        tol = (delta + 2.0 ** -22 * rlse.abs() + 2.0 ** -20)[~empty]
        assert bool((err <= tol).all()), "lse: worst %g of its tolerance" % (err / tol).max()
