"""The 8-bit paged cache at the ends of its types' ranges: values as large as BF16 holds, queries and keys whose factors are
beyond binary32, blocks of great and of small values together, scales of other writers next to a 16-bit type's midpoints."""
import math
from fractions import Fraction

import pytest
import torch

import paper_2609_35800_gb300 as hg
from attention16 import ROUNDOFF, attend
from pages8 import BLOCK, F8
from test_gpu_pages8 import BF16, D, F16, TYPES, Pool, _begins, _check_decode, _gen, _ints, _randn, _random_pool, _run_decode
from test_gpu_pages8 import _tables, _workspace

pytestmark = pytest.mark.gpu
MOST = {BF16: float(torch.finfo(BF16).max), F16: 65504.0}


@pytest.mark.parametrize("group", [4, 12])
@pytest.mark.parametrize("tokens", [1, 40, 1000, 20011])
@pytest.mark.parametrize("scale,codes", [(2.0 ** 103, (0, 0x7f)), (2.0 ** 112, (0, 0x7f)), (2.0 ** 119, (0, 0x7f)), (2.0 ** 126, (0x30, 0x3e))])
def test_decode_largest_values(scale, codes, tokens, group):
    """Averages of values up to BF16's end are in its range, whatever the number of tokens and the sums on the way."""
    g = _gen(tokens)
    tab, pages = _tables(g, [tokens], 64)
    pool = _random_pool(g, pages, 2, 64)
    c = torch.randint(*codes, pool.codes[1].shape, generator=g, device="cuda", dtype=torch.uint8)
    c[:, 1] |= torch.randint(0, 2, c[:, 1].shape, generator=g, device="cuda", dtype=torch.uint8) << 7  # both signs in one head
    pool.codes[1].copy_(c)
    pool.scales[1].copy_(torch.where(torch.rand(pool.scales[1].shape, generator=g, device="cuda") < 0.3, scale * 2.0 ** -9, scale))
    q = _randn(g, 1, 2 * group, D, scale=0.2)
    out, lse = _run_decode(pool, q, tab, [tokens])
    assert bool(out.isfinite().all())
    _check_decode(q, pool, tab, [tokens], out, lse)


@pytest.mark.parametrize("value", [2.0 ** 111, 2.0 ** 121, 1.75 * 2.0 ** 127, -1.75 * 2.0 ** 127])
def test_values_that_e4m3_holds_come_back(value):
    """One value for all tokens, which a code and a power of two hold: the average of any number of them."""
    g = _gen(3)
    lens = [1, 17, 700]
    tab, pages = _tables(g, lens, 16)
    pool = Pool(g, pages, 1, 16)
    k = _randn(g, sum(lens), 1, D)
    v = torch.full_like(k, value)
    hg.hg_pages8_append(pool.hg, None, k, v, None, None, _begins(lens), tab, _ints(lens))
    q = torch.zeros((3, 4, D), dtype=BF16, device="cuda")  # even probabilities
    out, lse = _run_decode(pool, q, tab, lens)
    assert torch.equal(out, torch.full_like(out, value))
    # a step's new token: a query far along its key, so that it is the sum
    lens = [n + 1 for n in lens]
    k1 = torch.full((3, 1, D), 16.0, dtype=BF16, device="cuda")
    out = torch.empty_like(out)
    tab2, pages2 = _tables(g, lens, 16)
    pool = Pool(g, pages2, 1, 16)
    pool.fill(g, tab2, [n - 1 for n in lens])
    hg.hg_pages8_decode_step(pool.hg, torch.ones_like(q), k1, torch.full_like(k1, value), None, None, tab2, _ints(lens), out, None,
                             0.0, _workspace(pool, 3, 4))
    assert torch.equal(out, torch.full_like(out, value))


@pytest.mark.parametrize("group", [4, 12])
@pytest.mark.parametrize("q_at,k_at", [(2.0 ** 100, 2.0 ** 60), (2.0 ** 70, 2.0 ** 90), (2.0 ** 120, 2.0 ** 119)])
def test_decode_far_factors_of_zeros(q_at, k_at, group):
    """Queries and keys that share no channel: every score is 0, however large both are."""
    g = _gen(5)
    lens = [1, 33, 500]
    tab, pages = _tables(g, lens, 16)
    pool = Pool(g, pages, 2, 16)
    k, v = (_randn(g, sum(lens), 2, D) for _ in "kv")
    k = k.clamp(-4, 4) * k_at
    k[..., ::3] = 0.0
    hg.hg_pages8_append(pool.hg, None, k, v, None, None, _begins(lens), tab, _ints(lens))
    q = torch.zeros((3, 2 * group, D), dtype=BF16, device="cuda")
    q[..., ::3] = q_at
    out, lse = _run_decode(pool, q, tab, lens)
    _check_decode(q, pool, tab, lens, out, lse)


@TYPES
@pytest.mark.parametrize("apart", [0, 8, 16, 20])
def test_decode_small_values_beside_great_ones_of_small_probability(dtype, apart):
    """Every fourth block's values are 2^apart larger, at probabilities of e^-30: the others' average is what is left.  Each
    term of the second product, a probability times its block's scale over the largest scale, 2^7 for a token of the largest
    score, is rounded to FP16: off by 2^-11 of it, or by 2^-25 where it is subnormal, times its code."""
    g = _gen(40 + apart)
    n = 2048
    tab, pages = _tables(g, [n], 32)
    pool = Pool(g, pages, 1, 32, dtype, fill=0)
    q = torch.zeros((1, 6, D), dtype=dtype, device="cuda")
    q[..., 0] = 1.0
    pool.codes[1].copy_(torch.randint(0x28, 0x48, pool.codes[1].shape, generator=g, device="cuda", dtype=torch.uint8))  # 0.25 to 3.75
    for s in pool.scales:
        s.fill_(1.0)
    great = tab[0, :n // 32:2].long()  # their first blocks
    pool.codes[0][great, 0, :BLOCK, 0] = 0xfe  # -448
    pool.scales[0][great, 0, 0] = 30 / 448
    pool.scales[1][great, 0, 0] = 2.0 ** apart
    out, lse = _run_decode(pool, q, tab, [n], scale=1.0)
    k, v = pool.rows(0, tab, 0, n), pool.rows(1, tab, 0, n)
    want, rlse, mean, _ = attend(q, k, v, torch.tensor([n], device="cuda"), 1.0)
    size = torch.where(torch.arange(n, device="cuda") // BLOCK % 4 == 0, 2.0 ** apart, 1.0)
    codes, total = (v / size[:, None, None]).sum(0)[0], n * 3 // 4
    # (a score of 0 is exact; exponentials and sums of positive terms in binary32: 2^-19)
    tol = ROUNDOFF[dtype] * want.abs() + 1.01 * (2.0 ** -11 + 2.0 ** -19) * mean + 2.0 ** (apart - 32) * codes / total
    assert bool(((out.double() - want).abs() <= tol).all())
    assert bool(((lse.double() - rlse).abs() <= 2.0 ** -18).all())


def _nearest(x, dtype):
    """x (a Fraction) rounded once to the type, ties to even, within its range."""
    bits, least, most = (8 if dtype == BF16 else 11), (-133 if dtype == BF16 else -24), MOST[dtype]
    if x == 0:
        return 0.0
    exponent = math.floor(math.log2(abs(x.numerator))) - math.floor(math.log2(x.denominator))
    while abs(x) >= Fraction(2) ** (exponent + 1):
        exponent += 1
    while abs(x) < Fraction(2) ** exponent:
        exponent -= 1
    step = Fraction(2) ** max(exponent - bits + 1, least)
    return max(-most, min(most, float(round(x / step) * step)))


@TYPES
def test_dequantize_rounds_once(dtype):
    """Every code under scales of 24 bits that bring one of them next to a midpoint of the type: exact products, rounded once."""
    g = _gen(9)
    bits = 8 if dtype == BF16 else 11
    scales = []
    for odd in (9, 11, 13, 15):  # a code's significand in eighths
        for j in range(6):
            # odd * m / 2^26 next to the midpoint (2 i + 1) / 2^bits in [1, 2)
            target = Fraction(2 * (2 ** (bits - 1) + 17 * j + 3) + 1, 2 ** bits)
            m = round(target * 2 ** 26 / odd)
            scales += [(m + d) * 2.0 ** -23 for d in (-1, 0, 1)]
    scales += [0.37, 1.37, 2.0 ** -126 * 1.1, 2.0 ** -130 * 1.3, 2.0 ** -8 * 1.0625, 1000.0, 2.0 ** 126 * 0.9, 1.0, 2.0 ** -140]
    scales += [s * 2.0 ** e for s in scales[:40] for e in (-20, -115, 90)]
    scales = [float(torch.tensor(s, dtype=torch.float32)) for s in scales]
    pages = len(scales)
    pool = Pool(g, pages, 1, 16, dtype, fill=0)
    codes = torch.arange(256, dtype=torch.uint8, device="cuda")
    for i in range(2):
        pool.codes[i][:, 0, :2] = codes.view(2, D)
        pool.scales[i].copy_(torch.tensor(scales, device="cuda").view(pages, 1, 1))
    tab = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, pages)
    out, v_out = (torch.empty((16 * pages, 1, D), dtype=dtype, device="cuda") for _ in "kv")
    hg.hg_pages8_dequantize(pool.hg, _ints([0, 16 * pages]), tab, out, v_out)
    assert torch.equal(out.view(torch.int16), v_out.view(torch.int16))
    got = out.view(pages, 16, D)[:, :2].reshape(pages, 256).double().tolist()
    exact = codes.cpu().view(F8).double().tolist()
    off = [(s, c, a) for s, row in zip(scales, got) for c, a in zip(exact, row)
           if c == c and a != _nearest(Fraction(c) * Fraction(s), dtype)]
    assert not off, "%d off, the first: scale %r, code %r, got %r" % ((len(off),) + off[0])
    assert bool(out.view(pages, 16, D)[:, :2].reshape(pages, 256)[:, [0x7f, 0xff]].isnan().all())
