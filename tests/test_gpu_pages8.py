"""The 8-bit paged cache on the GPU: what append stores bit for bit, dense rows exactly, decode against 64-bit references."""
import math

import pytest
import torch

import pages8 as ref8
import paper_2609_35800_gb300 as hg
from attention16 import ROUNDOFF, attend, check_turned, table, turned
from pages8 import BLOCK, F8

pytestmark = pytest.mark.gpu
D = 128
BF16, F16 = torch.bfloat16, torch.float16
TYPES = pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
NAN = float("nan")


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape, dtype=BF16, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _begins(lens):
    return _ints([0] + list(torch.tensor(lens).cumsum(0)) if lens else [0])


class Pool:
    """A pool whose bytes are random (NaN codes among them) and whose scales are NaN until something is stored."""

    def __init__(self, g, pages, heads, size, dtype=BF16, token_major=False, fill=None):
        shape = (pages, size, heads, D) if token_major else (pages, heads, size, D)
        self.codes, self.scales, self.size = [], [], size
        for _ in range(2):
            x = torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8)
            if fill is not None:
                x.fill_(fill)
            self.codes.append(x.transpose(1, 2) if token_major else x)
            self.scales.append(torch.full((pages, heads, size // BLOCK), NAN, device="cuda"))
        self.hg = hg.hg_pages8_create(*self.codes, *self.scales, dtype)

    def fill(self, g, tab, lens, scale=1.0):
        """The requests' first tokens, quantized; everything else stays as it is."""
        for i in range(2):
            codes, scales = self.codes[i].cpu(), self.scales[i].cpu()
            for b, n in enumerate(lens):
                rows = _randn(g, n, codes.shape[1], D, scale=scale).float().cpu()
                ref8.append(codes, scales, tab[b].cpu(), n, rows)
            self.codes[i].copy_(codes)
            self.scales[i].copy_(scales)

    def snapshot(self):
        return [x.cpu() for x in self.codes], [x.cpu() for x in self.scales]

    def rows(self, i, tab, b, n):
        """Request b's first n tokens [n][heads][128] in 64 bits; pages outside the pool are zeros."""
        heads = self.codes[i].shape[1]
        ids = tab[b, :-(-n // self.size)].long()
        ok = (ids >= 0) & (ids < self.codes[i].shape[0])
        at = torch.where(ok, ids, 0)
        x = ref8.values(self.codes[i][at], self.scales[i][at])
        x = torch.where(ok[:, None, None, None], x, 0.0)
        return x.transpose(1, 2).reshape(-1, heads, D)[:n]

    def top_scale(self, tab, b, n):
        ids = tab[b, :-(-n // self.size)].long()
        ids = ids[(ids >= 0) & (ids < self.codes[1].shape[0])]
        s = self.scales[1][ids]
        return float(s[s.isfinite()].max()) if n and ids.numel() and s.isfinite().any() else 0.0


def _tables(g, lens, size, spare=5):
    per = [-(-max(n, 0) // size) for n in lens]
    pages = sum(per) + spare
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    tab = torch.randint(-2 ** 31, 2 ** 31 - 1, (len(lens), max(max(per), 1)), generator=g, device="cuda").to(torch.int32)
    at = 0
    for b, n in enumerate(per):
        tab[b, :n] = order[at:at + n]
        at += n
    return tab, pages


def _same(got, want):
    """Pools alike: codes bit for bit (NaN is NaN), scales bit for bit."""
    for a, b in zip(got[0], want[0]):
        assert torch.equal(ref8.one_nan(a), ref8.one_nan(b))
    for a, b in zip(got[1], want[1]):
        assert torch.equal(a.view(torch.int32), b.view(torch.int32))


def _expect(pool, before, tab, begin, lens, k, v):
    """What the pool has to hold after rows k, v (exact in 32 bits) came."""
    codes, scales = [x.clone() for x in before[0]], [x.clone() for x in before[1]]
    for i, x in enumerate((k.float().cpu(), v.float().cpu())):
        for b, n in enumerate(lens):
            ref8.append(codes[i], scales[i], tab[b].cpu(), n, x[begin[b]:begin[b + 1]])
    return codes, scales


# -- append ------------------------------------------------------------------------------------------------------------

CACHED = [0, 0, 5, 15, 16, 31, 100, 7, 0, 33]
NEW = [1, 40, 30, 1, 16, 17, 0, 9, 0, 95]


@TYPES
@pytest.mark.parametrize("heads,group,size,token_major", [(4, 7, 16, False), (2, 3, 32, True), (8, 1, 256, False),
                                                         (1, 16, 64, True), (5, 12, 128, False), (3, 1, 32, True),
                                                         (1, 1, 16, False)])
def test_append(dtype, heads, group, size, token_major):
    """Without a rotation the stored values are the inputs' own: every byte and scale of the pool as defined."""
    g = _gen(heads * 10 + group)
    lens = [a + b for a, b in zip(CACHED, NEW)]
    tab, pages = _tables(g, lens, size)
    pool = Pool(g, pages, heads, size, dtype, token_major)
    pool.fill(g, tab, CACHED)
    begin, total, hq = _begins(NEW), sum(NEW), heads * group
    qkv = _randn(g, total, hq + 2 * heads, D, dtype=dtype, scale=1.0)
    # rows of very different sizes: some scales rise and some do not; a block of zeros
    qkv *= torch.exp2(torch.randint(-6, 7, (total, 1, 1), generator=g, device="cuda").to(dtype))
    qkv[1:17] = 0
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + heads], qkv[:, hq + heads:]
    before = pool.snapshot()
    q_out = torch.full((total, hq, D), NAN, dtype=dtype, device="cuda")
    k_out, v_out = (torch.full((heads, total, D), NAN, dtype=dtype, device="cuda").transpose(0, 1) for _ in "kv")
    hg.hg_pages8_append(pool.hg, q, k, v, None, None, begin, tab, _ints(lens), q_out, k_out, v_out)
    assert torch.equal(q_out, q) and torch.equal(k_out, k) and torch.equal(v_out, v)
    want = _expect(pool, before, tab, begin.tolist(), lens, k, v)
    _same(pool.snapshot(), want)
    # the same rows again: nothing moves
    hg.hg_pages8_append(pool.hg, None, k, v, None, None, begin, tab, _ints(lens))
    _same(pool.snapshot(), want)


ROTATIONS = {"half": (128, False, None), "pairs": (128, True, None), "part": (64, False, None),
             "part_pairs": (48, True, None), "small": (16, False, None), "three": (128, False, (16, 24, 24)),
             "three_part": (96, False, (8, 0, 40))}


@TYPES
@pytest.mark.parametrize("rotation", list(ROTATIONS))
def test_append_rotated(dtype, rotation):
    g = _gen(7)
    heads, group, size = 3, 2, 32
    cached, new = [0, 21, 3], [50, 1, 40]
    lens = [a + b for a, b in zip(cached, new)]
    tab, pages = _tables(g, lens, size)
    pool = Pool(g, pages, heads, size, dtype)
    pool.fill(g, tab, cached, scale=0.01)
    total, hq = sum(new), heads * group
    q, k, v = (_randn(g, total, n, D, dtype=dtype, scale=3.0) for n in (hq, heads, heads))
    dim, interleaved, sections = ROTATIONS[rotation]
    tab_cs = table(64, dim, "cuda")
    rot = hg.Rotation(tab_cs, interleaved=interleaved, sections=sections)
    pos = torch.randint(-3, 70, (3, total), generator=g, device="cuda", dtype=torch.int32)
    pos = pos if sections else pos[0].contiguous()
    before = pool.snapshot()
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    hg.hg_pages8_append(pool.hg, q, k, v, rot, pos, _begins(new), tab, _ints(lens), q_out, k_out)
    # the same turned rows as the 16-bit cache's
    kp = torch.zeros((-(-total // 16), heads, 16, D), dtype=dtype, device="cuda")
    pool16 = hg.hg_pages_create(kp, torch.zeros_like(kp))
    q16, k16 = torch.empty_like(q), torch.empty_like(k)
    hg.hg_pages_append(pool16, q, k, v, rot, pos, torch.arange(total, dtype=torch.int32, device="cuda"), q16, k16)
    assert torch.equal(q16, q_out) and torch.equal(k16, k_out)
    check_turned(k_out, k, turned(k, tab_cs, pos, dim, interleaved, sections), dtype)
    # values exactly; keys to within binary32's rounding of the rotation (2^-21 of the row's largest) and the code's own
    want = _expect(pool, before, tab, _begins(new).tolist(), lens, k, v)
    got = pool.snapshot()
    _same((got[0][1:], got[1][1:]), (want[0][1:], want[1][1:]))
    exact = turned(k, tab_cs, pos, dim, interleaved, sections)
    at = 0
    for b, n in enumerate(lens):
        first = n - new[b]
        rows = exact[at:at + new[b]]
        at += new[b]
        held = pool.rows(0, tab, b, n)
        for block in range(first // BLOCK, -(-n // BLOCK)):
            lo, hi = max(first, block * BLOCK), min(n, (block + 1) * BLOCK)
            page, place = int(tab[b, block * BLOCK // size]), block * BLOCK % size // BLOCK
            for h in range(heads):
                x = rows[lo - first:hi - first, h]
                s = float(pool.scales[0][page, h, place])
                amax = float(x.abs().max())
                assert math.frexp(s)[0] == 0.5 and amax <= 448 * s * (1 + 2.0 ** -20)
                if lo == block * BLOCK:
                    assert amax > 224 * s * (1 - 2.0 ** -20)
                tol = 2.0 ** -4 * x.abs() + 2.0 ** -10 * s + 2.0 ** -20 * amax
                assert bool(((held[lo:hi, h] - x).abs() <= tol).all())


def test_append_scale_borders():
    """Blocks whose largest entry is at, and next to, 448 times a power of two, at the ends of BF16's range, and zero."""
    g = _gen(5)
    tops = [448.0, 450.0, 446.0, 224.0, 1.75, 1.7578125, 2.0 ** -126, 2.0 ** -133, 0.0, 3.3895313892515355e38, 2.0 ** -118 * 1.75]
    n = len(tops)
    tab, pages = _tables(g, [16 * n], 16)
    pool = Pool(g, pages, 2, 16)
    k = (torch.rand((16 * n, 2, D), generator=g, device="cuda") * 2 - 1)
    for i, t in enumerate(tops):
        k[16 * i:16 * i + 16] = (k[16 * i:16 * i + 16].double() * t * 0.99).float()
        k[16 * i + 3, 1, 77] = -t
        k[16 * i + 9, 0, 0] = t
    k = k.to(BF16)
    before = pool.snapshot()
    hg.hg_pages8_append(pool.hg, None, k, -k, None, None, _begins([16 * n]), tab, _ints([16 * n]))
    want = _expect(pool, before, tab, [0, 16 * n], [16 * n], k, -k)
    _same(pool.snapshot(), want)
    assert [float(x) for x in pool.scales[0][tab[0].long(), 0, 0]] == [ref8.power(abs(float(torch.tensor(t).to(BF16)))) for t in tops]


@TYPES
def test_append_ties_to_even(dtype):
    """Every midpoint between two codes, its neighbour in 16 bits and the codes themselves, under a scale of 1."""
    g = _gen(6)
    codes = torch.arange(0, 0x7f, dtype=torch.uint8).view(F8).float()
    mid = (codes[1:] + codes[:-1]) / 2
    above = (mid.to(dtype).view(torch.int16) + 1).view(dtype).float()
    x = torch.cat([mid, above, codes])
    x = torch.cat([x, -x])
    rows = torch.zeros(-(-x.numel() // 127), 128)
    padded = torch.zeros(rows.shape[0] * 127)
    padded[:x.numel()] = x
    rows[:, :127] = padded.view(-1, 127)
    rows[:, 127] = 448.0  # every row's block has scale 1
    k = rows[:, None].to(dtype).cuda()
    n = k.shape[0]
    tab, pages = _tables(g, [n], 32)
    pool = Pool(g, pages, 1, 32, dtype)
    before = pool.snapshot()
    hg.hg_pages8_append(pool.hg, None, k, k, None, None, _begins([n]), tab, _ints([n]))
    _same(pool.snapshot(), _expect(pool, before, tab, [0, n], [n], k, k))


def test_append_nan_and_infinities():
    """They are stored as NaN, and the other entries of their block as if they were not there."""
    g = _gen(8)
    tab, pages = _tables(g, [37], 16)
    pool = Pool(g, pages, 1, 16)
    k = _randn(g, 37, 1, D)
    k[3, 0, 5], k[4, 0, 6], k[5, 0, 7] = NAN, math.inf, -math.inf
    k[16:32] = math.inf
    before = pool.snapshot()
    hg.hg_pages8_append(pool.hg, None, k, k, None, None, _begins([37]), tab, _ints([37]))
    want = _expect(pool, before, tab, [0, 37], [37], k, k)
    _same(pool.snapshot(), want)
    assert float(pool.scales[0][int(tab[0, 1]), 0, 0]) == 2.0 ** -126
    # a later token in a block with NaN: they stay NaN as the block is stored again
    more = _randn(g, 1, 1, D, scale=100.0)
    hg.hg_pages8_append(pool.hg, None, more, more, None, None, _begins([1]), tab, _ints([38]))
    codes, scales = [x.clone() for x in want[0]], [x.clone() for x in want[1]]
    for i in range(2):
        ref8.append(codes[i], scales[i], tab[0].cpu(), 38, more.float().cpu())
    _same(pool.snapshot(), (codes, scales))


def test_append_token_by_token():
    """As decoding does it, sizes up and down, and with blocks of another writer's scales, which are no powers of two."""
    g = _gen(9)
    size, heads, lens = 32, 2, [0, 13, 30]
    tab, pages = _tables(g, [n + 40 for n in lens], size)
    pool = Pool(g, pages, heads, size)
    pool.fill(g, tab, lens)
    for s in pool.scales:
        s *= 1.37
    want = pool.snapshot()
    for step in range(40):
        lens = [n + 1 for n in lens]
        k, v = (_randn(g, 3, heads, D, scale=2.0 ** ((step * 5) % 17 - 8)) for _ in "kv")
        hg.hg_pages8_append(pool.hg, None, k, v, None, None, _ints([0, 1, 2, 3]), tab, _ints(lens))
        want = _expect(pool, want, tab, [0, 1, 2, 3], lens, k, v)
        _same(pool.snapshot(), want)


def test_append_places():
    """Pages outside the pool, tokens outside the table, rows outside the requests, requests in no need of a page."""
    g = _gen(10)
    size, heads, hq = 16, 2, 4
    new, lens = [20, 40, 3, 0, 18], [20, 45, 2, 9, 18]  # the third has fewer tokens than rows
    tab, pages = _tables(g, [20, 32, 16, 16, 18], size)  # the second is longer than its row of the table
    pool = Pool(g, pages, heads, size)
    tab[0, 0], tab[4, 1] = -1, pages
    pool.fill(g, tab, [0, 5, 0, 9, 0])
    total = sum(new) + 12
    begin = _begins(new) + 5  # five rows ahead of the first request, seven behind the last
    qkv = _randn(g, total, hq + 2 * heads, D)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + heads], qkv[:, hq + heads:]
    before = pool.snapshot()
    q_out, k_out, v_out = (torch.full((total, n, D), NAN, dtype=BF16, device="cuda") for n in (hq, heads, heads))
    hg.hg_pages8_append(pool.hg, q, k, v, None, None, begin, tab, _ints(lens), q_out, k_out, v_out)
    for out, x in ((q_out, q), (k_out, k), (v_out, v)):
        assert torch.equal(out[5:-7], x[5:-7])
        assert bool(out[:5].isnan().all()) and bool(out[-7:].isnan().all())
    codes, scales = before
    for i, x in enumerate((k.float().cpu(), v.float().cpu())):
        at = 5
        for b, n in enumerate(new):
            rows = x[at:at + n]
            at += n
            skip = max(0, n - lens[b])  # (a token before the request's first)
            ref8.append(codes[i], scales[i], tab[b].cpu(), lens[b], rows[skip:])
    _same(pool.snapshot(), (codes, scales))


def test_append_in_place():
    g = _gen(11)
    tab, pages = _tables(g, [30], 16)
    pool = Pool(g, pages, 2, 16)
    q, k, v = _randn(g, 30, 4, D), _randn(g, 30, 2, D), _randn(g, 30, 2, D)
    cs = table(40, D, "cuda")
    rot, pos = hg.Rotation(cs), torch.arange(30, dtype=torch.int32, device="cuda")
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    hg.hg_pages8_append(pool.hg, q, k, v, rot, pos, _begins([30]), tab, _ints([30]), q_out, k_out)
    want = pool.snapshot()
    hg.hg_pages8_append(pool.hg, q, k, v, rot, pos, _begins([30]), tab, _ints([30]), q, k, v)
    assert torch.equal(q, q_out) and torch.equal(k, k_out)
    _same(pool.snapshot(), want)


def test_append_many_requests():
    """More requests than one round of a warp's search, and many without a token."""
    g = _gen(12)
    new = [int(x) for x in torch.randint(0, 4, (1500,), generator=g, device="cuda").cpu()]
    cached = [int(x) for x in torch.randint(0, 40, (1500,), generator=g, device="cuda").cpu()]
    lens = [a + b for a, b in zip(cached, new)]
    tab, pages = _tables(g, lens, 16)
    pool = Pool(g, pages, 1, 16, fill=0)
    for s in pool.scales:
        s.fill_(0.25)
    total = sum(new)
    k, v = _randn(g, total, 1, D), _randn(g, total, 1, D)
    before = pool.snapshot()
    hg.hg_pages8_append(pool.hg, None, k, v, None, None, _begins(new), tab, _ints(lens))
    _same(pool.snapshot(), _expect(pool, before, tab, _begins(new).tolist(), lens, k, v))


# -- dense rows --------------------------------------------------------------------------------------------------------

@TYPES
@pytest.mark.parametrize("heads,size,token_major,lens", [(4, 16, False, [0, 1, 15, 16, 17, 33, 100]), (1, 64, True, [257]),
                                                        (5, 32, True, [31, 0, 0, 64, 5]), (64, 256, False, [3, 300])])
def test_dequantize(dtype, heads, size, token_major, lens):
    g = _gen(heads)
    tab, pages = _tables(g, lens, size)
    pool = Pool(g, pages, heads, size, dtype, token_major)
    pool.fill(g, tab, lens)
    total = sum(lens)
    begin = _begins(lens) + 3
    k = torch.full((total + 8, heads, D), NAN, dtype=dtype, device="cuda")
    v = torch.full((heads, total + 8, D), NAN, dtype=dtype, device="cuda").transpose(0, 1)
    hg.hg_pages8_dequantize(pool.hg, begin, tab, k, v)
    for i, x in enumerate((k, v)):
        want = torch.cat([pool.rows(i, tab, b, n) for b, n in enumerate(lens)])
        assert torch.equal(x[3:3 + total], want.to(dtype))
        assert bool(x[:3].isnan().all()) and bool(x[3 + total:].isnan().all())
    # rows that are 16-byte aligned, no more
    narrow = torch.full((total + 8, heads, D + 8), NAN, dtype=dtype, device="cuda")
    hg.hg_pages8_dequantize(pool.hg, begin, tab, narrow[:, :, 8:], v)
    assert torch.equal(narrow[3:3 + total, :, 8:], k[3:3 + total]) and bool(narrow[:, :, :8].isnan().all())
    # one of the two alone
    k2, v2 = torch.full_like(k, NAN), torch.full_like(v, NAN)
    hg.hg_pages8_dequantize(pool.hg, begin, tab, k2)
    hg.hg_pages8_dequantize(pool.hg, begin, tab, None, v2)
    assert torch.equal(k2[3:3 + total], k[3:3 + total]) and torch.equal(v2[3:3 + total], v[3:3 + total])


def test_dequantize_many_requests():
    """Most of them without a row, others with one, a few with many."""
    g = _gen(23)
    lens = [int(x) for x in torch.randint(0, 3, (3000,), generator=g, device="cuda").cpu()]
    lens = [0 if i % 7 else n for i, n in enumerate(lens)]
    lens[100], lens[2999], lens[0] = 300, 50, 0
    tab, pages = _tables(g, lens, 16)
    pool = _random_pool(g, pages, 2, 16)
    total = sum(lens)
    k, v = (torch.full((total, 2, D), NAN, dtype=BF16, device="cuda") for _ in "kv")
    hg.hg_pages8_dequantize(pool.hg, _begins(lens), tab, k, v)
    for i, x in enumerate((k, v)):
        want = torch.cat([pool.rows(i, tab, b, n) for b, n in enumerate(lens) if n])
        assert torch.equal(x, want.to(BF16))


def test_dequantize_every_code_and_range():
    g = _gen(2)
    pool = Pool(g, 3, 1, 16, F16, fill=0)
    codes = torch.arange(256, dtype=torch.uint8, device="cuda")
    tab = _ints([[2, 0, 7]])
    for i in range(2):
        pool.codes[i][2, 0, :2] = codes.view(2, D)
        pool.codes[i][0, 0, :2] = codes.view(2, D)
        pool.scales[i][2], pool.scales[i][0] = 0.37, 1000.0
    out = torch.empty((50, 1, D), dtype=F16, device="cuda")
    hg.hg_pages8_dequantize(pool.hg, _ints([0, 50]), tab, out)
    exact = codes.view(F8).float()
    assert torch.equal(out[:2].view(-1).nan_to_num(7.0), (exact * 0.37).to(F16).nan_to_num(7.0))
    big = (exact * 1000.0).clamp(-65504, 65504)
    assert torch.equal(out[16:18].view(-1).nan_to_num(7.0), big.to(F16).nan_to_num(7.0))
    assert bool((out[32:] == 0).all())  # a page outside the pool, a place outside the table


# -- decode ------------------------------------------------------------------------------------------------------------

def _workspace(pool, n, hq):
    ws = torch.full((hg.hg_pages8_decode_workspace_size(pool.hg, n, hq),), 255, dtype=torch.uint8, device="cuda")
    hg.hg_workspace_clear(ws)
    return ws


def _check_decode(q, pool, tab, lens, out, lse, scale=None):
    for b, n in enumerate(lens):
        n = min(max(n, 0), tab.shape[1] * pool.size)
        k, v = pool.rows(0, tab, b, n), pool.rows(1, tab, b, n)
        ref = attend(q[b:b + 1], k, v, torch.tensor([n], device="cuda"), scale or D ** -0.5)
        ref8.check(out[b:b + 1], None if lse is None else lse[b:b + 1], ref, q.dtype, n, pool.top_scale(tab, b, n))


def _run_decode(pool, q, tab, lens, scale=0.0, ws=None):
    n, hq = q.shape[:2]
    ws = _workspace(pool, n, hq) if ws is None else ws
    out = torch.full((n, hq, D), NAN, dtype=q.dtype, device="cuda")
    lse = torch.full((n, hq), NAN, device="cuda")
    hg.hg_pages8_decode_attention(pool.hg, q, tab, _ints(lens), out, lse, scale, ws)
    assert hg.hg_workspace_status(ws) == 0
    return out, lse


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 63, 64, 65, 127, 128, 129, 255, 256, 257, 500, 1023]


@TYPES
@pytest.mark.parametrize("heads,group,size,token_major", [(4, 7, 16, False), (2, 8, 64, True), (3, 1, 32, False),
                                                         (1, 16, 128, False), (5, 12, 32, True), (2, 2, 256, False),
                                                         (8, 4, 16, True), (1, 9, 64, False), (16, 1, 16, False)])
def test_decode_edges(dtype, heads, group, size, token_major):
    """Random bytes (NaN among them) and NaN scales around every request."""
    g = _gen(heads * 100 + group)
    tab, pages = _tables(g, EDGES, size)
    pool = Pool(g, pages, heads, size, dtype, token_major)
    pool.fill(g, tab, EDGES)
    n, hq = len(EDGES), heads * group
    q = _randn(g, n, hq, D, dtype=dtype)
    out, lse = _run_decode(pool, q, tab, EDGES)
    _check_decode(q, pool, tab, EDGES, out, lse)
    # the same again, without lse, into a strided output from a strided query: bit for bit
    wide = torch.full((n, hq + 3, D), NAN, dtype=dtype, device="cuda")
    wide_q = torch.cat([q[:, :1], q], 1)
    hg.hg_pages8_decode_attention(pool.hg, wide_q[:, 1:], tab, _ints(EDGES), wide[:, 2:2 + hq], None, 0.0,
                                  _workspace(pool, n, hq))
    assert torch.equal(wide[:, 2:2 + hq], out)
    assert bool(wide[:, :2].isnan().all()) and bool(wide[:, 2 + hq:].isnan().all())


def _random_pool(g, pages, heads, size, dtype=BF16):
    """Every code but NaN anywhere, scales of no particular form."""
    pool = Pool(g, pages, heads, size, dtype)
    for c, s in zip(pool.codes, pool.scales):
        c.copy_(torch.where((c & 0x7f) == 0x7f, torch.full_like(c, 1), c))
        s.copy_(torch.rand(s.shape, generator=g, device="cuda") * 0.02 + 0.003)
    return pool


@pytest.mark.parametrize("batch,length,heads,group,size", [(1, 1, 4, 7, 16), (1, 70001, 2, 4, 64), (1, 20011, 1, 1, 16),
                                                          (3, 9001, 4, 7, 128), (130, 333, 2, 8, 32), (700, 40, 1, 3, 16),
                                                          (2, 30000, 1, 16, 256), (40, 2000, 8, 8, 64), (200, 9000, 2, 4, 32),
                                                          (170, 6300, 2, 12, 64)])
def test_decode_long_and_wide(batch, length, heads, group, size):
    g = _gen(length)
    lens = [max(1, length - 37 * b) for b in range(batch)]
    tab, pages = _tables(g, lens, size)
    pool = _random_pool(g, pages, heads, size)
    q = _randn(g, batch, heads * group, D, scale=0.2)
    ws = _workspace(pool, batch, heads * group)
    out, lse = _run_decode(pool, q, tab, lens, ws=ws)
    for b in sorted({0, 1, batch // 2, batch - 1} & set(range(batch))):
        _check_decode(q[b:b + 1], pool, tab[b:b + 1], lens[b:b + 1], out[b:b + 1], lse[b:b + 1])
    for _ in range(3):  # whoever comes last
        again, lse2 = _run_decode(pool, q, tab, lens, ws=ws)
        assert torch.equal(again, out) and torch.equal(lse2, lse)


@TYPES
def test_decode_scales(dtype):
    """Values whose blocks' scales are 2^40 apart in any order, zero scales, keys of very different blocks."""
    g = _gen(3)
    lens = [700, 64, 333]
    tab, pages = _tables(g, lens, 32)
    pool = _random_pool(g, pages, 2, 32, dtype)
    pool.scales[1] *= torch.exp2(torch.randint(-20, 5, pool.scales[1].shape, generator=g, device="cuda").float())
    pool.scales[0] *= torch.exp2(torch.randint(-10, 3, pool.scales[0].shape, generator=g, device="cuda").float())
    pool.scales[1][::3, :, 1], pool.scales[0][::2, :, 0] = 0.0, 0.0
    q = _randn(g, 3, 10, D, dtype=dtype)
    out, lse = _run_decode(pool, q, tab, lens)
    _check_decode(q, pool, tab, lens, out, lse)
    pool.scales[1].fill_(0.0)
    out, _ = _run_decode(pool, q, tab, lens)
    assert bool((out == 0).all())


@pytest.mark.parametrize("at", [2.0 ** -100, 2.0 ** -30, 2.0 ** 30, 2.0 ** 100])
def test_decode_far_ranges(at):
    """Queries, keys and values far from 1 (BF16), entries of a query 2^30 apart."""
    g = _gen(4)
    lens = [300]
    tab, pages = _tables(g, lens, 16)
    pool = _random_pool(g, pages, 1, 16)
    q = _randn(g, 1, 4, D, scale=0.2)
    q[:, :, ::5] *= 2.0 ** -30
    want, lse = _run_decode(pool, q, tab, lens)
    _check_decode(q, pool, tab, lens, want, lse)
    pool.scales[0] /= at
    pool.scales[1] *= at
    moved, lse2 = _run_decode(pool, q * at, tab, lens)
    assert torch.equal(moved.double() / at, want.double())  # powers of two throughout
    assert torch.equal(lse2, lse)


def test_decode_large_and_rising_scores():
    g = _gen(13)
    lens = [1000, 77]
    tab, pages = _tables(g, lens, 16)
    pool = _random_pool(g, pages, 2, 16)
    q = _randn(g, 2, 6, D, scale=3000.0)
    out, lse = _run_decode(pool, q, tab, lens)
    _check_decode(q, pool, tab, lens, out, lse)
    # keys that grow along the request: the maximum moves in every tile
    for b, n in enumerate(lens):
        for t in range(0, n, 16):
            pool.codes[0][tab[b, t // 16], :] = 0x30 + 0x80  # -0.5
            pool.scales[0][tab[b, t // 16], :] = 0.01 * (n - t)
    q = torch.ones((2, 6, D), dtype=BF16, device="cuda")
    out, lse = _run_decode(pool, q, tab, lens)
    _check_decode(q, pool, tab, lens, out, lse)


def test_decode_nan_shows():
    """A NaN code of a request's own token, or in its query, makes those rows NaN and no others."""
    g = _gen(14)
    lens = [50, 50, 50, 50]
    tab, pages = _tables(g, lens, 16)
    pool = _random_pool(g, pages, 2, 16)
    q = _randn(g, 4, 4, D)
    clean, _ = _run_decode(pool, q, tab, lens)
    pool.codes[0][tab[0, 1], 1, 3, 9] = 0x7f
    pool.codes[1][tab[1, 2], 0, 2, 9] = 0xff  # token 34: one channel of the values
    q[2, 3, 5] = NAN
    out, lse = _run_decode(pool, q, tab, lens)
    assert bool(out[0, 2:].isnan().all()) and torch.equal(out[0, :2], clean[0, :2])
    assert bool(out[1, :2, 9].isnan().all()) and int(out[1].isnan().sum()) == 2
    assert bool(out[2, 3].isnan().all()) and torch.equal(out[2, :3], clean[2, :3])
    assert torch.equal(out[3], clean[3])


def test_decode_odd_places():
    """Lengths below 0 and beyond the table, pages outside the pool (zeros), a table without a column."""
    g = _gen(15)
    tab, pages = _tables(g, [64, 64, 64, 64], 16)
    pool = _random_pool(g, pages, 2, 16)
    tab[1, 1], tab[2, 0] = -5, 2 ** 31 - 1
    lens = [-7, 60, 50, 2 ** 31 - 1]
    q = _randn(g, 4, 8, D)
    out, lse = _run_decode(pool, q, tab, lens)
    _check_decode(q, pool, tab, lens, out, lse)
    assert bool((out[0] == 0).all())
    out, lse = _run_decode(pool, q, tab[:, :0], lens)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


@TYPES
def test_decode_most_heads(dtype):
    """64 KV heads of 16 queries each."""
    g = _gen(24)
    lens = [1, 70, 300, 1000]
    tab, pages = _tables(g, lens, 64)
    pool = _random_pool(g, pages, 64, 64, dtype)
    q = _randn(g, 4, 1024, D, dtype=dtype, scale=0.2)
    out, lse = _run_decode(pool, q, tab, lens)
    _check_decode(q, pool, tab, lens, out, lse)


def test_keys_and_values_in_one_tensor():
    """Pages that lie [pages][2][heads][tokens][128], heads and tokens with room between them: append, decode, dense rows."""
    g = _gen(25)
    lens, heads, size = [100, 7, 65], 3, 32
    tab, pages = _tables(g, lens, size)
    both = torch.randint(0, 256, (pages, 2, heads + 1, size + 2, D + 16), generator=g, device="cuda", dtype=torch.uint8)
    kept = both.clone()
    view = both[:, :, :heads, :size, :D]
    pool, twin = Pool(_gen(1), pages, heads, size), Pool(_gen(1), pages, heads, size)
    pool.codes = [view[:, 0], view[:, 1]]
    pool.hg = hg.hg_pages8_create(*pool.codes, *pool.scales, BF16)
    k, v = (_randn(g, sum(lens), heads, D) for _ in "kv")
    for x in (pool, twin):
        hg.hg_pages8_append(x.hg, None, k, v, None, None, _begins(lens), tab, _ints(lens))
    for i in range(2):
        for b, n in enumerate(lens):
            assert torch.equal(pool.rows(i, tab, b, n), twin.rows(i, tab, b, n))
    q = _randn(g, 3, 2 * heads, D)
    out, lse = _run_decode(pool, q, tab, lens)
    want, lse2 = _run_decode(twin, q, tab, lens)
    assert torch.equal(out, want) and torch.equal(lse, lse2)
    rows = [torch.empty_like(k) for _ in range(4)]
    hg.hg_pages8_dequantize(pool.hg, _begins(lens), tab, *rows[:2])
    hg.hg_pages8_dequantize(twin.hg, _begins(lens), tab, *rows[2:])
    assert torch.equal(rows[0], rows[2]) and torch.equal(rows[1], rows[3])
    inside = torch.zeros_like(both, dtype=torch.bool)
    inside[:, :, :heads, :size, :D] = True
    assert torch.equal(both[~inside], kept[~inside])  # nothing between the rows is touched


@pytest.mark.parametrize("scale", [0.5, 1e-3])
def test_decode_softmax_scale(scale):
    g = _gen(16)
    tab, pages = _tables(g, [200], 64)
    pool = _random_pool(g, pages, 1, 64, F16)
    q = _randn(g, 1, 5, D, dtype=F16)
    out, lse = _run_decode(pool, q, tab, [200], scale)
    _check_decode(q, pool, tab, [200], out, lse, scale)


def test_decode_far_pages():
    """Codes beyond 2^32 bytes from the pool's start."""
    g = _gen(17)
    size, heads = 256, 1
    pages = 2 ** 32 // (size * D) + 40
    codes = [torch.empty((pages, heads, size, D), dtype=torch.uint8, device="cuda") for _ in "kv"]
    scales = [torch.empty((pages, heads, size // BLOCK), device="cuda") for _ in "kv"]
    tab = _ints([[pages - 1, 3, pages - 17]])
    small = _random_pool(g, 3, heads, size)
    for i in range(2):
        codes[i][tab[0].long()] = small.codes[i]
        scales[i][tab[0].long()] = small.scales[i]
    pool = hg.hg_pages8_create(*codes, *scales, BF16)
    q = _randn(g, 1, 8, D)
    near = _ints([[0, 1, 2]])
    want, _ = _run_decode(small, q, near, [700])
    out = torch.empty_like(want)
    hg.hg_pages8_decode_attention(pool, q, tab, _ints([700]), out, None, 0.0, _workspace(small, 1, 8))
    assert torch.equal(out, want)
    k, v = _randn(g, 30, heads, D), _randn(g, 30, heads, D)
    hg.hg_pages8_append(pool, None, k, v, None, None, _begins([30]), tab, _ints([730]))
    hg.hg_pages8_append(small.hg, None, k, v, None, None, _begins([30]), near, _ints([730]))
    rows = [torch.empty((730, heads, D), dtype=BF16, device="cuda") for _ in range(4)]
    hg.hg_pages8_dequantize(pool, _begins([730]), tab, *rows[:2])
    hg.hg_pages8_dequantize(small.hg, _begins([730]), near, *rows[2:])
    assert torch.equal(rows[0], rows[2]) and torch.equal(rows[1], rows[3])


# -- step --------------------------------------------------------------------------------------------------------------

@TYPES
@pytest.mark.parametrize("heads,group,size,rotation", [(4, 7, 16, "three"), (2, 8, 64, "half"), (5, 12, 32, "part_pairs"),
                                                      (1, 16, 128, None), (3, 1, 256, "pairs")])
def test_step(dtype, heads, group, size, rotation):
    """Stores what append stores, bit for bit, and attends to it."""
    g = _gen(heads + size)
    lens = [1, 2, 16, 17, 18, 31, 32, 33, 48, 64, 65, 100, 257, 640]
    n, hq = len(lens), heads * group
    tab, pages = _tables(g, lens, size)
    pool, twin = (Pool(_gen(1), pages, heads, size, dtype) for _ in range(2))
    for x in (pool, twin):
        x.fill(_gen(2), tab, [t - 1 for t in lens])
    rot, pos = None, None
    if rotation:
        dim, interleaved, sections = ROTATIONS[rotation]
        rot = hg.Rotation(table(700, dim, "cuda"), interleaved=interleaved, sections=sections)
        pos = torch.randint(0, 700, (3, n), generator=g, device="cuda", dtype=torch.int32)
        pos = pos if sections else pos[0].contiguous()
    for scale in (0.01, 1.0, 30.0):  # below the block's scale, about it, above it
        q, k, v = (_randn(g, n, h, D, dtype=dtype, scale=s) for h, s in ((hq, 1.0), (heads, scale), (heads, scale)))
        kept = [x.clone() for x in (q, k, v)]
        out, lse = torch.full((n, hq, D), NAN, dtype=dtype, device="cuda"), torch.full((n, hq), NAN, device="cuda")
        ws = _workspace(pool, n, hq)
        hg.hg_pages8_decode_step(pool.hg, q, k, v, rot, pos, tab, _ints(lens), out, lse, 0.0, ws)
        assert hg.hg_workspace_status(ws) == 0
        assert all(torch.equal(a, b) for a, b in zip(kept, (q, k, v)))
        q_rot = torch.empty_like(q)
        hg.hg_pages8_append(twin.hg, q, k, v, rot, pos, _ints(list(range(n + 1))), tab, _ints(lens), q_rot)
        _same(pool.snapshot(), twin.snapshot())
        _check_decode(q_rot, pool, tab, lens, out, lse)
        again, _ = _run_decode(pool, q_rot, tab, lens)
        assert torch.equal(again, out)


def test_step_odd_places():
    """Length 0, a request that has grown past its table, a last page outside the pool: as the header says."""
    g = _gen(18)
    heads, hq, size = 2, 4, 16
    tab, pages = _tables(g, [64] * 5, size)
    lens = [0, 65, 64, 50, 33]
    pool = _random_pool(g, pages, heads, size)
    tab[3, 3], tab[4, 2] = -1, pages
    before = pool.snapshot()
    q, k, v = _randn(g, 5, hq, D), _randn(g, 5, heads, D), _randn(g, 5, heads, D)
    out, lse = torch.full((5, hq, D), NAN, dtype=BF16, device="cuda"), torch.full((5, hq), NAN, device="cuda")
    ws = _workspace(pool, 5, hq)
    hg.hg_pages8_decode_step(pool.hg, q, k, v, None, None, tab, _ints(lens), out, lse, 0.0, ws)
    codes, scales = before
    for i, x in enumerate((k.float().cpu(), v.float().cpu())):
        ref8.append(codes[i], scales[i], tab[2].cpu(), 64, x[2:3])
    _same(pool.snapshot(), (codes, scales))
    assert bool((out[0] == 0).all()) and bool((lse[0] == -math.inf).all())
    _check_decode(q[:3], pool, tab[:3], lens[:3], out[:3], lse[:3])
    for b in (3, 4):  # zeros where the page is missing, the new token with a scale of its own
        n = lens[b]
        rows = []
        for i, x in enumerate((k, v)):
            r = pool.rows(i, tab, b, n)
            for h in range(heads):
                s = ref8.power(float(x[b, h].abs().max()))
                r[n - 1, h] = ref8.decode(ref8.encode(x[b, h].float().cpu(), s)).cuda() * s
            rows.append(r)
        top = max(pool.top_scale(tab, b, n), ref8.power(float(v[b].abs().max())))
        ref8.check(out[b:b + 1], lse[b:b + 1], attend(q[b:b + 1], *rows, torch.tensor([n], device="cuda"), D ** -0.5), BF16, n, top)


# -- together ----------------------------------------------------------------------------------------------------------

def test_stream_and_graph():
    """Plan, append, step and dense rows captured once, replayed as the requests grow."""
    g = _gen(19)
    heads, hq, size, n = 2, 6, 16, 3
    pool = Pool(g, 40, heads, size)
    tab = torch.zeros((n, 12), dtype=torch.int32, device="cuda")
    lens, free = _ints([5, 0, 31]), torch.arange(40, dtype=torch.int32, device="cuda")
    counts, new, begin = _ints([40, 0, 0, 0]), _ints([5, 0, 31]), _ints([0] * (n + 1))
    slots, pos = _ints([0] * 36), _ints([0] * 36)
    zero = _ints([0, 0, 0])
    hg.hg_pages_plan(tab, zero, new, free, counts[:1], size, lens, begin, slots, pos, counts)
    k, v = _randn(g, 36, heads, D), _randn(g, 36, heads, D)
    hg.hg_pages8_append(pool.hg, None, k, v, None, None, begin, tab, lens)
    keys, vals = ([list(x[:5]), [], list(x[5:])] for x in (k, v))
    one, slots1, pos1, begin1 = _ints([1] * n), _ints([0] * n), _ints([0] * n), _ints([0] * (n + 1))
    q1, k1, v1 = (torch.empty((n, h, D), dtype=BF16, device="cuda") for h in (hq, heads, heads))
    out, lse = torch.empty((n, hq, D), dtype=BF16, device="cuda"), torch.empty((n, hq), device="cuda")
    ws = _workspace(pool, n, hq)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        hg.hg_pages_plan(tab, lens, one, free, counts[:1], size, lens, begin1, slots1, pos1, counts)
        hg.hg_pages8_decode_step(pool.hg, q1, k1, v1, None, None, tab, lens, out, lse, 0.0, ws)
    for step in range(40):
        for x in (q1, k1, v1):
            x.copy_(_randn(g, *x.shape))
        for b in range(n):
            keys[b].append(k1[b].clone())
            vals[b].append(v1[b].clone())
        graph.replay()
        have = [len(x) for x in keys]
        assert lens.tolist() == have and counts.tolist()[1:] == [0, n, max(have)]
        assert slots1.tolist() == [int(tab[b, (t - 1) // size]) * size + (t - 1) % size for b, t in enumerate(have)]
        _check_decode(q1, pool, tab, have, out, lse)
    assert int(counts[0]) == 40 - sum(-(-t // size) for t in have)
    assert hg.hg_workspace_status(ws) == 0
    # what the pages hold is the rows that came, to e4m3's precision (blocks were stored again as they grew: twice at most
    # half a step of 2^-3 below the block's range)
    for i, rows in enumerate((keys, vals)):
        for b in range(n):
            x = torch.stack(rows[b]).double()
            held = pool.rows(i, tab, b, len(rows[b]))
            s = torch.stack([pool.scales[i][tab[b, t // size].long(), :, t % size // BLOCK] for t in range(len(rows[b]))])
            assert bool(((held - x).abs() <= 2.0 ** -3 * x.abs() + 2.0 ** -9 * s[..., None].double()).all())


def test_other_stream():
    g = _gen(20)
    lens = [333, 90]
    tab, pages = _tables(g, lens, 32)
    pool = _random_pool(g, pages, 2, 32)
    q = _randn(g, 2, 8, D)
    want, _ = _run_decode(pool, q, tab, lens)
    out = torch.full_like(want, NAN)
    ws, lengths = _workspace(pool, 2, 8), _ints(lens)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    hg.hg_pages8_decode_attention(pool.hg, q, tab, lengths, out, None, 0.0, ws, stream=side)
    side.synchronize()
    assert torch.equal(out, want)


def test_a_workspace_serves_both_kinds_of_pool():
    g = _gen(21)
    lens = [333, 2000, 90]
    tab, pages = _tables(g, lens, 32)
    pool = _random_pool(g, pages, 2, 32)
    kp, vp = (_randn(g, pages, 2, 32, D) for _ in "kv")
    pool16 = hg.hg_pages_create(kp, vp)
    q = _randn(g, 3, 8, D)
    ws = _workspace(pool, 3, 8)
    assert ws.numel() == hg.hg_pages_decode_workspace_size(pool16, 3, 8)
    out16 = [torch.empty_like(q) for _ in range(2)]
    first, _ = _run_decode(pool, q, tab, lens, ws=ws)
    hg.hg_pages_decode_attention(pool16, q, tab, _ints(lens), out16[0], None, 0.0, ws)
    second, _ = _run_decode(pool, q, tab, lens, ws=ws)
    hg.hg_pages_decode_attention(pool16, q, tab, _ints(lens), out16[1], None, 0.0, ws)
    assert torch.equal(first, second) and torch.equal(out16[0], out16[1])


def test_prompt_after_cached_tokens():
    """A prompt's second piece: stored, read back as dense rows with the first, attended to by the prompt kernel."""
    g = _gen(22)
    heads, hq, size = 2, 6, 32
    cached, new = [50, 0, 129], [20, 33, 64]
    lens = [a + b for a, b in zip(cached, new)]
    tab, pages = _tables(g, lens, size)
    pool = Pool(g, pages, heads, size)
    pool.fill(g, tab, cached)
    q, k, v = (_randn(g, sum(new), h, D) for h in (hq, heads, heads))
    hg.hg_pages8_append(pool.hg, None, k, v, None, None, _begins(new), tab, _ints(lens))
    dk, dv = (torch.empty((heads, sum(lens), D), dtype=BF16, device="cuda").transpose(0, 1) for _ in "kv")
    hg.hg_pages8_dequantize(pool.hg, _begins(lens), tab, dk, dv)
    out = torch.empty_like(q)
    ws = torch.empty(hg.hg_prompt_workspace_size(), dtype=torch.uint8, device="cuda")
    hg.hg_workspace_clear(ws)
    hg.hg_prompt_attention(q, dk, dv, _begins(new).cpu(), _begins(lens).cpu(), out, None, True, 0.0, ws)
    at = 0
    for b, n in enumerate(lens):
        kk, vv = pool.rows(0, tab, b, n).to(BF16), pool.rows(1, tab, b, n).to(BF16)
        seen = torch.arange(new[b], device="cuda") + cached[b] + 1
        want = attend(q[at:at + new[b]], kk, vv, seen, D ** -0.5)
        # (probabilities in BF16: the 16-bit kernels' tolerance)
        tol = ROUNDOFF[BF16] * want[0].abs() + (ROUNDOFF[BF16] + 2.0 ** -16 * want[3][..., None]) * want[2] * 1.02 + 2.0 ** -20
        assert bool(((out[at:at + new[b]].double() - want[0]).abs() <= tol).all())
        at += new[b]
