"""Paged append, paged decode attention and prompt attention on the GPU against 64-bit references."""
import math

import pytest
import torch

import paper_2609_35800_gb300 as hg
from attention16 import ROUNDOFF, attend, check, check_turned, table, turned

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


def _pool(g, pages, heads, size, dtype, token_major, fill=None):
    shape = (pages, size, heads, D) if token_major else (pages, heads, size, D)
    out = []
    for _ in range(2):
        x = _randn(g, *shape, dtype=dtype) if fill is None else torch.full(shape, fill, dtype=dtype, device="cuda")
        out.append(x.transpose(1, 2) if token_major else x)
    return out


def _bits(x):
    return x.contiguous().view(torch.int16)


def _workspace(n):
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    hg.hg_workspace_clear(ws)
    return ws


# -- append ------------------------------------------------------------------------------------------------------------

ROTATIONS = {"none": None, "half": (128, False, None), "pairs": (128, True, None), "part": (64, False, None),
             "part_pairs": (48, True, None), "small": (16, False, None), "three": (128, False, (16, 24, 24)),
             "three_part": (96, False, (8, 0, 40))}


@TYPES
@pytest.mark.parametrize("rotation", list(ROTATIONS))
@pytest.mark.parametrize("tokens,heads,group,size,token_major", [(1, 4, 7, 16, False), (37, 2, 3, 32, True),
                                                                (300, 8, 1, 256, False), (2, 1, 16, 64, True)])
def test_append(dtype, rotation, tokens, heads, group, size, token_major):
    g = _gen(tokens + heads)
    hq = heads * group
    pages = -(-tokens // size) + 3
    kp, vp = _pool(g, pages, heads, size, dtype, token_major)
    k0, v0 = _bits(kp).clone(), _bits(vp).clone()
    pool = hg.hg_pages_create(kp, vp)
    qkv = _randn(g, tokens, hq + 2 * heads, D, dtype=dtype, scale=3.0)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + heads], qkv[:, hq + heads:]
    slots = torch.randperm(pages * size, generator=g, device="cuda")[:tokens].to(torch.int32)
    if tokens > 4:  # not stored: negative, just past the pool, far past it
        slots[0], slots[1], slots[2] = -1, pages * size, 2 ** 31 - 1
    rot, spec = None, ROTATIONS[rotation]
    pos = torch.randint(-3, 70, (3, tokens), generator=g, device="cuda", dtype=torch.int32)
    if spec:
        tab = table(64, spec[0], "cuda")
        rot = hg.Rotation(tab, interleaved=spec[1], sections=spec[2])
        if spec[2] is None:
            pos = pos[0].contiguous()
        want_q, want_k = (turned(x, tab, pos, spec[0], spec[1], spec[2]) for x in (q, k))
    else:
        want_q, want_k = q.double(), k.double()
    q_out = torch.full((tokens, hq, D), NAN, dtype=dtype, device="cuda")
    k_out = torch.full((heads, tokens, D), NAN, dtype=dtype, device="cuda").transpose(0, 1)
    v_out = torch.full((heads, tokens, D), NAN, dtype=dtype, device="cuda").transpose(0, 1)
    hg.hg_pages_append(pool, q, k, v, rot, pos, slots, q_out, k_out, v_out)
    check_turned(q_out, q, want_q, dtype)
    check_turned(k_out, k, want_k, dtype)
    assert torch.equal(_bits(v_out), _bits(v))
    keep = (slots >= 0) & (slots < pages * size)
    at = slots[keep].long()
    k0[at // size, :, at % size] = _bits(k_out)[keep]
    v0[at // size, :, at % size] = _bits(v)[keep]
    assert torch.equal(_bits(kp), k0) and torch.equal(_bits(vp), v0)


def test_append_in_place_and_without_queries():
    g = _gen(3)
    kp, vp = _pool(g, 4, 2, 16, BF16, False)
    pool = hg.hg_pages_create(kp, vp)
    q, k, v = _randn(g, 5, 6, D), _randn(g, 5, 2, D), _randn(g, 5, 2, D)
    tab = table(50, 128, "cuda")
    rot, pos = hg.Rotation(tab), torch.arange(5, dtype=torch.int32, device="cuda") * 7
    slots = torch.arange(9, 14, dtype=torch.int32, device="cuda")
    want_q, want_k = turned(q, tab, pos, 128, False, None), turned(k, tab, pos, 128, False, None)
    q0, k0 = q.clone(), k.clone()
    hg.hg_pages_append(pool, None, k, v, rot, pos, slots)
    assert torch.equal(k, k0)
    stored = kp[0, :, 9:14].clone()
    hg.hg_pages_append(pool, q, k, v, rot, pos, slots, q, k)
    check_turned(q, q0, want_q, BF16)
    check_turned(k, k0, want_k, BF16)
    assert torch.equal(kp[0, :, 9:14], stored) and torch.equal(k.transpose(0, 1), stored)
    hg.hg_pages_append(pool, q[:0], k[:0], v[:0], rot, pos[:0], slots[:0], q[:0])  # nothing to do


# -- decode ------------------------------------------------------------------------------------------------------------

def _tables(g, lens, size, spare=5):
    """A page table that gives every request its own pages in no order, and the pool's size."""
    per = [-(-max(n, 0) // size) for n in lens]
    pages = sum(per) + spare
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    tab = torch.randint(-2 ** 31, 2 ** 31 - 1, (len(lens), max(max(per), 1)), generator=g, device="cuda").to(torch.int32)
    at = 0
    for b, n in enumerate(per):
        tab[b, :n] = order[at:at + n]
        at += n
    return tab, pages


def _gather(pool, tab, b, n, size):
    """Request b's first n rows [n][heads][128]."""
    if n <= 0:
        return torch.zeros((0, pool.shape[1], D), dtype=pool.dtype, device="cuda")
    ids = tab[b, :-(-n // size)].long()
    ok = (ids >= 0) & (ids < pool.shape[0])
    x = pool[torch.where(ok, ids, 0)] * ok[:, None, None, None].to(pool.dtype)
    return x.transpose(1, 2).reshape(-1, pool.shape[1], D)[:n]


def _poison(pool, tab, lens, size):
    """NaN everywhere but at the requests' own tokens."""
    for x in pool:
        clean = x.clone()
        x.fill_(NAN)
        for b, n in enumerate(lens):
            for p in range(-(-n // size)):
                m = min(size, n - p * size)
                x[tab[b, p], :, :m] = clean[tab[b, p], :, :m]


def _check_decode(q, kp, vp, tab, lens, size, out, lse, scale=None):
    dtype = q.dtype
    for b, n in enumerate(lens):
        k, v = _gather(kp, tab, b, n, size), _gather(vp, tab, b, n, size)
        n = k.shape[0]
        ref = attend(q[b:b + 1], k, v, torch.tensor([n], device="cuda"), scale or D ** -0.5)
        vmax = float(v.double().abs().max()) if n else 0.0
        check(out[b:b + 1], None if lse is None else lse[b:b + 1], ref, dtype, n, vmax)


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 500, 1023]


@TYPES
@pytest.mark.parametrize("heads,group,size,token_major", [(4, 7, 16, False), (2, 8, 64, True), (3, 1, 32, False),
                                                         (1, 16, 128, False), (5, 12, 32, True), (2, 2, 256, False),
                                                         (8, 4, 16, True), (1, 9, 64, False), (64, 1, 16, False)])
def test_decode_edges(dtype, heads, group, size, token_major):
    g = _gen(heads * 100 + group)
    tab, pages = _tables(g, EDGES, size)
    kp, vp = _pool(g, pages, heads, size, dtype, token_major)
    _poison((kp, vp), tab, EDGES, size)
    pool = hg.hg_pages_create(kp, vp)
    n, hq = len(EDGES), heads * group
    q = _randn(g, n, hq, D, dtype=dtype)
    lens = torch.tensor(EDGES, dtype=torch.int32, device="cuda")
    ws = _workspace(hg.hg_pages_decode_workspace_size(pool, n, hq))
    out, lse = torch.full((n, hq, D), NAN, dtype=dtype, device="cuda"), torch.full((n, hq), NAN, device="cuda")
    hg.hg_pages_decode_attention(pool, q, tab, lens, out, lse, 0.0, ws)
    assert hg.hg_workspace_status(ws) == 0
    _check_decode(q, kp, vp, tab, EDGES, size, out, lse)
    # the same again, without lse, into a strided output from a strided query: bit for bit
    wide = torch.full((n, hq + 3, D), NAN, dtype=dtype, device="cuda")
    wide_q = torch.cat([q[:, :1], q], 1)
    hg.hg_pages_decode_attention(pool, wide_q[:, 1:], tab, lens, wide[:, 2:2 + hq], None, 0.0, ws)
    assert torch.equal(_bits(wide[:, 2:2 + hq]), _bits(out))
    assert bool(wide[:, :2].isnan().all()) and bool(wide[:, 2 + hq:].isnan().all())


@pytest.mark.parametrize("batch,length,heads,group,size", [(1, 1, 4, 7, 16), (1, 70001, 2, 4, 64), (1, 20011, 1, 1, 16),
                                                          (3, 9001, 4, 7, 128), (130, 333, 2, 8, 32), (700, 40, 1, 3, 16),
                                                          (2, 30000, 1, 16, 256)])
def test_decode_long_and_wide(batch, length, heads, group, size):
    g = _gen(length)
    lens = [max(1, length - 37 * b) for b in range(batch)]
    tab, pages = _tables(g, lens, size)
    kp, vp = _pool(g, pages, heads, size, BF16, False)
    pool = hg.hg_pages_create(kp, vp)
    hq = heads * group
    q = _randn(g, batch, hq, D, scale=2.0)
    ws = _workspace(hg.hg_pages_decode_workspace_size(pool, batch, hq))
    out, lse = torch.empty((batch, hq, D), dtype=BF16, device="cuda"), torch.empty((batch, hq), device="cuda")
    dl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    hg.hg_pages_decode_attention(pool, q, tab, dl, out, lse, 0.2, ws)
    first = out.clone(), lse.clone()
    some = sorted({0, 1, batch // 2, batch - 1} & set(range(batch)))
    _check_decode(q[some], kp, vp, tab[some], [lens[b] for b in some], size, out[some], lse[some], scale=0.2)
    for _ in range(3):  # the join does not depend on which part comes last
        hg.hg_pages_decode_attention(pool, q, tab, dl, out, lse, 0.2, ws)
        assert torch.equal(_bits(out), _bits(first[0])) and torch.equal(lse, first[1])
    assert hg.hg_workspace_status(ws) == 0


def test_decode_pages_outside_the_pool_and_lengths_outside_the_table():
    g = _gen(5)
    kp, vp = _pool(g, 6, 2, 16, BF16, False)
    pool = hg.hg_pages_create(kp, vp)
    q = _randn(g, 4, 6, D)
    tab = torch.tensor([[0, -1, 2], [6, 2 ** 31 - 1, 3], [1, 4, 5], [5, 4, 3]], dtype=torch.int32, device="cuda")
    given = torch.tensor([40, 48, 1000, -7], dtype=torch.int32, device="cuda")
    ws = _workspace(hg.hg_pages_decode_workspace_size(pool, 4, 6))
    out, lse = torch.empty_like(q), torch.empty((4, 6), device="cuda")
    hg.hg_pages_decode_attention(pool, q, tab, given, out, lse, 0.0, ws)
    _check_decode(q, kp, vp, tab, [40, 48, 48, 0], 16, out, lse)


@TYPES
def test_decode_extreme_scores(dtype):
    """Scores far beyond exp's range, of one sign and of both, and keys whose size is the type's largest."""
    g = _gen(6)
    lens = [300, 300, 300, 300]
    tab, pages = _tables(g, lens, 16)
    kp, vp = _pool(g, pages, 2, 16, dtype, False)
    for b, scale in enumerate((200.0, 2000.0, 1.0, 1e-4)):
        kp[tab[b].long()] = (kp[tab[b].long()].float() * scale).to(dtype)
    q = _randn(g, 4, 8, D, dtype=dtype)
    top = torch.finfo(dtype).max
    kp[tab[2, 3].long(), :, 5] = 0.0
    kp[tab[2, 3].long(), :, 5, 0] = top
    q[2, :, 0] = 2.0 ** -14
    pool = hg.hg_pages_create(kp, vp)
    ws = _workspace(hg.hg_pages_decode_workspace_size(pool, 4, 8))
    out, lse = torch.empty_like(q), torch.empty((4, 8), device="cuda")
    hg.hg_pages_decode_attention(pool, q, tab, torch.tensor(lens, dtype=torch.int32, device="cuda"), out, lse, 0.0, ws)
    _check_decode(q, kp, vp, tab, lens, 16, out, lse)


def test_decode_infinite_and_nan_entries_reach_only_their_request():
    g = _gen(7)
    lens = [100, 100, 100]
    tab, pages = _tables(g, lens, 16)
    kp, vp = _pool(g, pages, 1, 16, BF16, False)
    kp[tab[1, 2].long(), 0, 3, 7] = NAN
    vp[tab[2, 1].long(), 0, 3, 9] = math.inf
    pool = hg.hg_pages_create(kp, vp)
    q = _randn(g, 3, 4, D)
    ws = _workspace(hg.hg_pages_decode_workspace_size(pool, 3, 4))
    out, lse = torch.empty_like(q), torch.empty((3, 4), device="cuda")
    hg.hg_pages_decode_attention(pool, q, tab, torch.tensor(lens, dtype=torch.int32, device="cuda"), out, lse, 0.0, ws)
    _check_decode(q[:1], kp, vp, tab[:1], lens[:1], 16, out[:1], lse[:1])
    assert bool(out[1].isnan().all()) and bool(lse[1].isnan().all())
    assert bool((out[2, :, 9] == math.inf).all()) and bool(out[2, :, :9].isfinite().all())


def test_decode_page_offsets_beyond_32_bits():
    """Pages 2^26 elements apart: the last ones start beyond 2^32 elements and 2^33 bytes."""
    g = _gen(8)
    apart, count, heads, size = 1 << 26, 70, 2, 64
    flat = [torch.empty(apart * (count - 1) + heads * size * D, dtype=BF16, device="cuda") for _ in range(2)]
    kp, vp = (f.as_strided((count, heads, size, D), (apart, size * D, D, 1)) for f in flat)
    for x in (kp, vp):
        x.copy_(_randn(g, count, heads, size, D))
    pool = hg.hg_pages_create(kp, vp)
    lens = [64 * 60 + 5, 130]
    tab = torch.stack([torch.randperm(count, generator=g, device="cuda")[:61] for _ in lens]).to(torch.int32)
    tab[1, 0] = count - 1
    q = _randn(g, 2, 8, D)
    ws = _workspace(hg.hg_pages_decode_workspace_size(pool, 2, 8))
    out, lse = torch.empty_like(q), torch.empty((2, 8), device="cuda")
    hg.hg_pages_decode_attention(pool, q, tab, torch.tensor(lens, dtype=torch.int32, device="cuda"), out, lse, 0.0, ws)
    _check_decode(q, kp, vp, tab, lens, size, out, lse)
    k, v = _randn(g, 1, heads, D), _randn(g, 1, heads, D)
    hg.hg_pages_append(pool, None, k, v, None, None, torch.tensor([count * size - 3], dtype=torch.int32, device="cuda"))
    assert torch.equal(kp[count - 1, :, size - 3], k[0]) and torch.equal(vp[count - 1, :, size - 3], v[0])


def test_decode_on_other_streams_and_in_a_graph():
    g = _gen(9)
    size, cap = 16, 400
    lens = [200, 17, 399]
    tab, pages = _tables(g, [cap] * 3, size)
    kp, vp = _pool(g, pages, 2, size, BF16, True)
    pool = hg.hg_pages_create(kp, vp)
    q = _randn(g, 3, 8, D)
    ws = _workspace(hg.hg_pages_decode_workspace_size(pool, 3, 8))
    dl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((3, 8), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    hg.hg_pages_decode_attention(pool, q, tab, dl, out, lse, 0.0, ws, stream=side)
    side.synchronize()
    _check_decode(q, kp, vp, tab, lens, size, out, lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hg.hg_pages_decode_attention(pool, q, tab, dl, out, lse, 0.0, ws)
    for lens in ([1, 400, 33], [0, 64, 128]):
        dl.copy_(torch.tensor(lens, dtype=torch.int32))
        q.copy_(_randn(g, 3, 8, D))
        graph.replay()
        torch.cuda.synchronize()
        _check_decode(q, kp, vp, tab, lens, size, out, lse)


def test_decode_one_workspace_for_many_shapes():
    """A workspace of the largest batch serves others, of other pools, in turn."""
    g = _gen(10)
    made = []
    for heads, group, size, lens in [(4, 7, 16, [900, 3, 77]), (1, 16, 64, [5000]), (8, 1, 32, [64] * 40), (2, 8, 16, [0, 1300])]:
        tab, pages = _tables(g, lens, size)
        kp, vp = _pool(g, pages, heads, size, F16, False)
        made.append((hg.hg_pages_create(kp, vp), kp, vp, tab, lens, size, _randn(g, len(lens), heads * group, D, dtype=F16)))
    ws = _workspace(max(hg.hg_pages_decode_workspace_size(m[0], 40, m[6].shape[1]) for m in made))
    for _ in range(2):
        for pool, kp, vp, tab, lens, size, q in made:
            out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
            hg.hg_pages_decode_attention(pool, q, tab, torch.tensor(lens, dtype=torch.int32, device="cuda"), out, lse, 0.0, ws)
            _check_decode(q, kp, vp, tab, lens, size, out, lse)


# -- decode step -------------------------------------------------------------------------------------------------------

@TYPES
@pytest.mark.parametrize("rotation", ["none", "half", "pairs", "part", "three"])
@pytest.mark.parametrize("heads,group,size,token_major", [(4, 7, 16, False), (2, 12, 64, True), (3, 1, 256, False)])
def test_step(dtype, rotation, heads, group, size, token_major):
    g = _gen(heads + group)
    n, hq = len(EDGES), heads * group
    tab, pages = _tables(g, EDGES, size)
    kp, vp = _pool(g, pages, heads, size, dtype, token_major)
    _poison((kp, vp), tab, [max(0, x - 1) for x in EDGES], size)  # the new token's place holds NaN before
    pool = hg.hg_pages_create(kp, vp)
    qkv = _randn(g, n, hq + 2 * heads, D, dtype=dtype)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + heads], qkv[:, hq + heads:]
    before = qkv.clone()
    spec = ROTATIONS[rotation]
    rot, tab_r, pos = None, None, None
    if spec:
        tab_r = table(1100, spec[0], "cuda")
        rot = hg.Rotation(tab_r, interleaved=spec[1], sections=spec[2])
        pos = torch.randint(0, 1100, (3, n), generator=g, device="cuda", dtype=torch.int32)
        pos = pos if spec[2] else pos[0].contiguous()
    # what the append stores is what the step stores
    kq, vq = kp.clone(), vp.clone()
    slots = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    for b, t in enumerate(EDGES):
        if t:
            slots[b] = tab[b, (t - 1) // size] * size + (t - 1) % size
    q_rot = torch.empty((n, hq, D), dtype=dtype, device="cuda")
    hg.hg_pages_append(hg.hg_pages_create(kq, vq), q, k, v, rot, pos, slots, q_rot)
    ws = _workspace(hg.hg_pages_decode_workspace_size(pool, n, hq))
    out, lse = torch.full((n, hq, D), NAN, dtype=dtype, device="cuda"), torch.full((n, hq), NAN, device="cuda")
    lens = torch.tensor(EDGES, dtype=torch.int32, device="cuda")
    hg.hg_pages_decode_step(pool, q, k, v, rot, pos, tab, lens, out, lse, 0.0, ws)
    assert hg.hg_workspace_status(ws) == 0
    assert torch.equal(_bits(qkv), _bits(before))
    assert torch.equal(_bits(kp), _bits(kq)) and torch.equal(_bits(vp), _bits(vq))
    if spec:
        check_turned(q_rot, q, turned(q, tab_r, pos, *spec), dtype)
    _check_decode(q_rot, kp, vp, tab, EDGES, size, out, lse)


def test_step_without_a_page_for_the_new_token():
    """The last page is outside the pool: nothing is stored, the new token counts all the same."""
    g = _gen(12)
    kp, vp = _pool(g, 4, 2, 16, BF16, False)
    pool = hg.hg_pages_create(kp, vp)
    tab = torch.tensor([[0, 1], [2, -1], [99, 0]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([20, 17, 1], dtype=torch.int32, device="cuda")
    q, k, v = _randn(g, 3, 4, D), _randn(g, 3, 2, D), _randn(g, 3, 2, D)
    k0, v0 = kp.clone(), vp.clone()
    ws = _workspace(hg.hg_pages_decode_workspace_size(pool, 3, 4))
    out, lse = torch.empty_like(q), torch.empty((3, 4), device="cuda")
    hg.hg_pages_decode_step(pool, q, k, v, None, None, tab, lens, out, lse, 0.0, ws)
    k0[1, :, 3], v0[1, :, 3] = k[0], v[0]
    assert torch.equal(kp, k0) and torch.equal(vp, v0)
    _check_decode(q[:1], kp, vp, tab[:1], [20], 16, out[:1], lse[:1])
    for b, old in ((1, 16), (2, 0)):
        kk = torch.cat([_gather(kp, tab, b, old, 16), k[b:b + 1]])
        vv = torch.cat([_gather(vp, tab, b, old, 16), v[b:b + 1]])
        ref = attend(q[b:b + 1], kk, vv, torch.tensor([old + 1], device="cuda"), D ** -0.5)
        check(out[b:b + 1], lse[b:b + 1], ref, BF16, old + 1, 5.0)


# -- prompts -----------------------------------------------------------------------------------------------------------

def _prompt(g, q_lens, k_lens, heads, group, dtype, layout, gap=0, scale=1.0):
    """Packed inputs with `gap` NaN rows before and after; layout: token-major, head-major or one fused tensor."""
    hq, nq, nk = heads * group, sum(q_lens) + 2 * gap, sum(k_lens) + 2 * gap
    if layout == "fused":
        assert nq == nk
        x = _randn(g, nq, hq + 2 * heads, D, dtype=dtype, scale=scale)
        q, k, v = x[:, :hq], x[:, hq:hq + heads], x[:, hq + heads:]
    elif layout == "heads":
        q, k, v = (_randn(g, h, n, D, dtype=dtype, scale=scale).transpose(0, 1) for h, n in ((hq, nq), (heads, nk), (heads, nk)))
    else:
        q, k, v = (_randn(g, n, h, D, dtype=dtype, scale=scale) for h, n in ((hq, nq), (heads, nk), (heads, nk)))
    if gap:
        for x in (q, k, v):
            x[:gap] = NAN
            x[-gap:] = NAN
    begin = [torch.tensor([gap] + list(n), dtype=torch.int32).cumsum(0, dtype=torch.int32) for n in (q_lens, k_lens)]
    return q, k, v, begin[0], begin[1]


def _run_prompt(q, k, v, qb, kb, causal, scale=0.0, ws=None, lse=True):
    out = torch.full(q.shape, NAN, dtype=q.dtype, device="cuda")
    got = torch.full(q.shape[:2], NAN, device="cuda") if lse else None
    if ws is None:
        ws = _workspace(hg.hg_prompt_workspace_size())
    hg.hg_prompt_attention(q, k, v, qb, kb, out, got, causal, scale, ws)
    assert hg.hg_workspace_status(ws) == 0
    return out, got


def _check_prompt(q, k, v, qb, kb, causal, out, lse, scale=None, some=None):
    qb, kb = qb.tolist(), kb.tolist()
    for i in some if some is not None else range(len(qb) - 1):
        a, b, c, d = qb[i], qb[i + 1], kb[i], kb[i + 1]
        if b == a:
            continue
        nq, nk = b - a, d - c
        for r in range(0, nq, 512):  # bounds the reference's memory
            rows = torch.arange(r, min(r + 512, nq), device="cuda")
            seen = (rows + 1 + nk - nq).clamp(min=0) if causal else torch.full_like(rows, nk)
            ref = attend(q[a + r:a + r + len(rows)], k[c:d], v[c:d], seen, scale or D ** -0.5)
            vmax = float(v[c:d].double().abs().max()) if nk else 0.0
            check(out[a + r:a + r + len(rows)], None if lse is None else lse[a + r:a + r + len(rows)], ref, q.dtype, nk, vmax)
    assert bool(out[:qb[0]].isnan().all()) and bool(out[qb[-1]:].isnan().all())


RAGGED = [1, 2, 17, 0, 18, 19, 35, 36, 37, 63, 64, 65, 127, 128, 129, 130, 255, 256, 257, 300, 513]


@TYPES
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,group,layout", [(4, 7, "tokens"), (2, 1, "heads"), (1, 16, "fused"), (3, 5, "heads"),
                                                (2, 8, "tokens"), (5, 12, "fused"), (1, 2, "tokens"), (8, 4, "heads")])
def test_prompt_ragged(dtype, causal, heads, group, layout):
    g = _gen(heads * 31 + group)
    q, k, v, qb, kb = _prompt(g, RAGGED, RAGGED, heads, group, dtype, layout, gap=3)
    out, lse = _run_prompt(q, k, v, qb, kb, causal)
    _check_prompt(q, k, v, qb, kb, causal, out, lse)
    again, none = _run_prompt(q, k, v, qb, kb, causal, lse=False)
    assert torch.equal(_bits(again), _bits(out))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,group", [(4, 7), (2, 1), (1, 16)])
def test_prompt_more_or_fewer_keys_than_queries(causal, heads, group):
    """Cached tokens before the prompt's own; more queries than keys (rows that see nothing); no keys at all."""
    g = _gen(heads)
    q_lens = [1, 64, 5, 200, 40, 300, 7, 130, 260]
    k_lens = [1000, 777, 5, 130, 0, 1, 500, 258, 129]
    q, k, v, qb, kb = _prompt(g, q_lens, k_lens, heads, group, BF16, "tokens", gap=2)
    out, lse = _run_prompt(q, k, v, qb, kb, causal)
    _check_prompt(q, k, v, qb, kb, causal, out, lse)
    if causal:  # row 0 of 200 queries over 130 keys sees nothing
        at = int(qb[3])
        assert bool((out[at] == 0).all()) and bool((lse[at] == -math.inf).all())


@pytest.mark.parametrize("nq,nk,heads,group,causal", [(64, 9000, 4, 7, True), (1, 20000, 2, 8, True), (3, 5000, 1, 1, False),
                                                      (700, 4100, 1, 4, True), (129, 129 + 4096, 2, 16, True)])
def test_prompt_few_rows_over_long_keys(nq, nk, heads, group, causal):
    g = _gen(nk)
    q, k, v, qb, kb = _prompt(g, [nq], [nk], heads, group, BF16, "tokens", gap=1)
    ws = _workspace(hg.hg_prompt_workspace_size())
    out, lse = _run_prompt(q, k, v, qb, kb, causal, scale=0.15, ws=ws)
    _check_prompt(q, k, v, qb, kb, causal, out, lse, scale=0.15)
    for _ in range(3):
        again, lse2 = _run_prompt(q, k, v, qb, kb, causal, scale=0.15, ws=ws)
        assert torch.equal(_bits(again), _bits(out)) and torch.equal(lse[1:-1], lse2[1:-1])


@pytest.mark.parametrize("dtype,lens,heads,group,layout", [(BF16, [2600], 2, 8, "heads"), (F16, [1460], 4, 7, "fused"),
                                                           (BF16, [1500, 900, 40, 2100], 8, 4, "tokens"),
                                                           (F16, [2200] * 6, 16, 2, "heads")])
def test_prompt_long(dtype, lens, heads, group, layout):
    g = _gen(sum(lens))
    q, k, v, qb, kb = _prompt(g, lens, lens, heads, group, dtype, layout)
    out, lse = _run_prompt(q, k, v, qb, kb, True)
    _check_prompt(q, k, v, qb, kb, True, out, lse, some=range(min(len(lens), 3)))


def test_prompts_without_any_key_and_an_empty_batch():
    g = _gen(25)
    q = _randn(g, 70, 6, D)
    none = torch.empty(0, 2, D, dtype=BF16, device="cuda")
    qb, kb = torch.tensor([0, 40, 70], dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for causal in (True, False):
        out, lse = _run_prompt(q, none, none, qb, kb, causal)
        assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    out, lse = _run_prompt(q, none, none, qb[:1], kb[:1], True)  # no prompt
    assert bool(out.isnan().all())


@TYPES
@pytest.mark.parametrize("heads,group", [(2, 8), (3, 5), (1, 16), (4, 1)])
def test_prompt_output_strides(dtype, heads, group):
    """Outputs heads first, and every second head of a wider tensor: whole tiles and those that end a prompt."""
    g = _gen(heads * 7 + group)
    lens = [300, 31, 16, 1, 256, 129]
    q, k, v, qb, kb = _prompt(g, lens, lens, heads, group, dtype, "tokens")
    n, hq = q.shape[0], q.shape[1]
    dense, lse = _run_prompt(q, k, v, qb, kb, True)
    _check_prompt(q, k, v, qb, kb, True, dense, lse)
    ws = _workspace(hg.hg_prompt_workspace_size())
    first = torch.full((hq, n, D), NAN, dtype=dtype, device="cuda").transpose(0, 1)
    hg.hg_prompt_attention(q, k, v, qb, kb, first, None, True, 0.0, ws)
    assert torch.equal(_bits(first), _bits(dense))
    wide = torch.full((n, 2 * hq, D), NAN, dtype=dtype, device="cuda")
    hg.hg_prompt_attention(q, k, v, qb, kb, wide[:, ::2], None, True, 0.0, ws)
    assert torch.equal(_bits(wide[:, ::2]), _bits(dense)) and bool(wide[:, 1::2].isnan().all())


def test_prompt_many_prompts():
    """More prompts than one launch takes."""
    g = _gen(20)
    lens = [(7 * i) % 23 for i in range(600)]
    q, k, v, qb, kb = _prompt(g, lens, lens, 2, 3, BF16, "tokens")
    out, lse = _run_prompt(q, k, v, qb, kb, True)
    _check_prompt(q, k, v, qb, kb, True, out, lse, some=[1, 2, 250, 255, 256, 257, 300, 511, 512, 513, 599])
    whole = [torch.cat([x[a:b] for a, b in zip(qb.tolist(), qb.tolist()[1:])]) for x in (out, lse)]
    assert bool(whole[0].isfinite().all()) and bool(whole[1].isfinite().all())


@TYPES
def test_prompt_extreme_scores(dtype):
    g = _gen(21)
    lens = [400, 400, 300]
    q, k, v, qb, kb = _prompt(g, lens, lens, 2, 4, dtype, "tokens")
    k[:400] *= 200.0
    k[400:800] *= 2000.0
    k[900] = 0.0
    k[900, :, 0] = torch.finfo(dtype).max
    q[800:, :, 0] = 2.0 ** -14
    out, lse = _run_prompt(q, k, v, qb, kb, True)
    _check_prompt(q, k, v, qb, kb, True, out, lse)


def test_prompt_rising_scores():
    """Every key's score is above the one before: the running maximum moves at every tile."""
    g = _gen(22)
    n = 1000
    q, k, v, qb, kb = _prompt(g, [n], [n], 1, 4, BF16, "tokens")
    q[:, :, 0], k[:, :, 0] = 8.0, torch.arange(n, device="cuda", dtype=torch.float32).to(BF16)[:, None] / 2
    out, lse = _run_prompt(q, k, v, qb, kb, True)
    _check_prompt(q, k, v, qb, kb, True, out, lse)


def test_prompt_nan_and_infinity_stay_in_their_prompt():
    g = _gen(23)
    lens = [100, 130, 77, 200]
    q, k, v, qb, kb = _prompt(g, lens, lens, 2, 3, BF16, "tokens")
    k[100:230] = NAN
    v[100:230] = math.inf
    v[307 + 199:] = NAN  # the last prompt's last row
    out, lse = _run_prompt(q, k, v, qb, kb, False)
    _check_prompt(q, k, v, qb, kb, False, out, lse, some=[0, 2])
    assert bool(out[100:230].isnan().all())
    assert bool(out[307:].isnan().all())


def test_prompt_on_another_stream():
    g = _gen(24)
    q, k, v, qb, kb = _prompt(g, [150, 20], [150, 20], 2, 2, F16, "tokens")
    ws = _workspace(hg.hg_prompt_workspace_size())
    side = torch.cuda.Stream()
    out = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    hg.hg_prompt_attention(q, k, v, qb, kb, out, None, True, 0.0, ws, stream=side)
    side.synchronize()
    _check_prompt(q, k, v, qb, kb, True, out, None)


def _apart(shape, dtype, fill=NAN):
    """A dense tensor that starts 16 bytes past a 32-byte boundary."""
    n = math.prod(shape)
    return torch.full((n + 24,), fill, dtype=dtype, device="cuda")[8:8 + n].view(shape)


@TYPES
def test_rows_aligned_to_16_bytes_only(dtype):
    g = _gen(40)
    heads, group, lens = 2, 4, [150, 33]
    hq, n = heads * group, sum(lens)
    q, k, v, qb, kb = _prompt(g, lens, lens, heads, group, dtype, "tokens")
    shifted = [_apart(x.shape, dtype) for x in (q, k, v, q)]
    assert all(x.data_ptr() % 32 == 16 for x in shifted)
    for to, x in zip(shifted, (q, k, v)):
        to.copy_(x)
    ws = _workspace(hg.hg_prompt_workspace_size())
    hg.hg_prompt_attention(*shifted[:3], qb, kb, shifted[3], None, True, 0.0, ws)
    _check_prompt(q, k, v, qb, kb, True, shifted[3], None)
    kp, vp = _apart((20, heads, 16, D), dtype), _apart((20, heads, 16, D), dtype)
    pool = hg.hg_pages_create(kp, vp)
    slots = torch.arange(n, dtype=torch.int32, device="cuda") + 16
    hg.hg_pages_append(pool, *shifted[:3], None, None, slots, shifted[3])
    assert torch.equal(_bits(shifted[3]), _bits(q))
    tab = torch.arange(1, 13, dtype=torch.int32, device="cuda")[None].contiguous()
    out, dws = _apart((1, hq, D), dtype), _workspace(hg.hg_pages_decode_workspace_size(pool, 1, hq))
    hg.hg_pages_decode_attention(pool, shifted[0][:1], tab, torch.tensor([n], dtype=torch.int32, device="cuda"), out, None,
                                 0.0, dws)
    _check_decode(q[:1], kp, vp, tab, [n], 16, out, None)


# -- together ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("heads,group,lens", [(4, 7, [70, 5, 200, 33]), (1, 2, [2500, 40])])  # (whole items; pieces)
def test_serving_run(heads, group, lens):
    """Prompts admitted together, three tokens each, against one attention over everything in 64 bits."""
    from paper_2609_35800_gb300.paged import PagedRunner
    g = _gen(30)
    hq = heads * group
    tab = table(max(lens) + 8, 128, "cuda")
    run = PagedRunner(sum(lens) // 16 + 40, 16, hq, heads, hg.Rotation(tab), max_batch=8, max_tokens=2600)
    for _ in range(2):  # the second time in pages that the first gave back
        n = sum(lens)
        qkv = _randn(g, n, hq + 2 * heads, D)
        pos = torch.cat([torch.arange(x) for x in lens]).to(torch.int32).cuda()
        k_dense = torch.empty(n, heads, D, dtype=BF16, device="cuda")
        out = run.admit(qkv[:, :hq], qkv[:, hq:hq + heads], qkv[:, hq + heads:], lens, pos, k_out=k_dense)
        rot = [turned(x, tab, pos, 128, False, None).to(BF16) for x in (qkv[:, :hq], qkv[:, hq:hq + heads])]
        begin = [sum(lens[:i]) for i in range(len(lens) + 1)]
        keys = [rot[1][a:b] for a, b in zip(begin, begin[1:])]
        vals = [qkv[a:b, hq + heads:] for a, b in zip(begin, begin[1:])]
        for i, (a, b) in enumerate(zip(begin, begin[1:])):
            ref = attend(rot[0][a:b], keys[i], vals[i], torch.arange(1, b - a + 1, device="cuda"), D ** -0.5)
            # a rotated entry may round to either neighbour: one unit more in every score
            ref = ref[:3] + (ref[3] + 2.0 ** 17 * 2.0 ** -8 * ref[3],)
            check(out[a:b], None, ref, BF16, b - a, 5.0)
        for step in range(3):
            qkv = _randn(g, len(lens), hq + 2 * heads, D)
            pos = torch.tensor([x + step for x in lens], dtype=torch.int32, device="cuda")
            got = run.step(qkv[:, :hq], qkv[:, hq:hq + heads], qkv[:, hq + heads:], pos)
            rot = [turned(x, tab, pos, 128, False, None).to(BF16) for x in (qkv[:, :hq], qkv[:, hq:hq + heads])]
            for i in range(len(lens)):
                keys[i] = torch.cat([keys[i], rot[1][i:i + 1]])
                vals[i] = torch.cat([vals[i], qkv[i:i + 1, hq + heads:]])
                ref = attend(rot[0][i:i + 1], keys[i], vals[i], torch.tensor([len(keys[i])], device="cuda"), D ** -0.5)
                ref = ref[:3] + (ref[3] + 2.0 ** 17 * 2.0 ** -8 * ref[3],)
                check(got[i:i + 1], None, ref, BF16, len(keys[i]), 5.0)
        run.release()


def test_a_prompt_goes_on_in_the_packed_cache():
    """Rotated keys and values written heads first are what hg_quantize_kv takes, as they are."""
    from paper_2609_35800_gb300 import workloads as wl
    from paper_2609_35800_gb300.runner import config_of, shape_of
    g = _gen(41)
    w = wl.custom("prompt", 1, 1, 8, 2, 24, 64, 40, wl.BASE_MINMAX, 4, 0, decode_steps=2, protected=[(0, 1)])
    n, heads, hq = w.seq_len, 2, 8
    kp, vp = _pool(g, 12, heads, 16, BF16, False)
    pool = hg.hg_pages_create(kp, vp)
    qkv, tab = _randn(g, n, hq + 2 * heads, D), table(n, 128, "cuda")
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    k, v = torch.empty(1, heads, n, D, dtype=BF16, device="cuda"), torch.empty(1, heads, n, D, dtype=BF16, device="cuda")
    q = torch.empty(n, hq, D, dtype=BF16, device="cuda")
    hg.hg_pages_append(pool, qkv[:, :hq], qkv[:, hq:hq + heads], qkv[:, hq + heads:], hg.Rotation(tab), pos, pos, q,
                       k[0].transpose(0, 1), v[0].transpose(0, 1))
    begin = torch.tensor([0, n], dtype=torch.int32)
    out, lse = _run_prompt(q, k[0].transpose(0, 1), v[0].transpose(0, 1), begin, begin, True)
    _check_prompt(q, k[0].transpose(0, 1), v[0].transpose(0, 1), begin, begin, True, out, lse)
    shape, config, mask = shape_of(w), config_of(w), wl.protection_mask(w).numpy()
    arena = torch.empty(hg.hg_cache_layout(shape, config, mask), dtype=torch.uint8, device="cuda")
    cache = hg.hg_cache_create(shape, config, mask, arena)
    hg.hg_quantize_kv(cache, 0, [k], [v])
    kd, vd = torch.empty_like(k), torch.empty_like(v)
    hg.hg_dequantize_kv(cache, 0, 1, kd, vd, False)
    for got, want in ((kd, k), (vd, v)):
        assert torch.equal(got[:, 1], want[:, 1])  # the protected head, and all text
        assert torch.equal(got[:, :, :24], want[:, :, :24]) and torch.equal(got[:, :, 88:], want[:, :, 88:])
        span = want[:, 0, 24:88].float()  # 4-bit codes: at most half a step off, and the rounding to BF16
        step = (span.amax(-1, keepdim=True) - span.amin(-1, keepdim=True)) / 15
        assert bool(((got[:, 0, 24:88].float() - span).abs() <= step * 0.501 + span.abs() * 2.0 ** -8).all())


@TYPES
@pytest.mark.parametrize("heads,group,size,rotated", [(2, 4, 16, True), (1, 12, 64, False), (3, 1, 32, True)])
def test_step_of_requests_longer_than_their_table(dtype, heads, group, size, rotated):
    """No place for the new token: nothing is stored, and the table's last token stays what it was."""
    g = _gen(50 + heads)
    hq, per = heads * group, 5
    cap = per * size
    given = [cap, cap + 1, cap + 2, 2 ** 31 - 1, cap - 1, 0, -5]
    n, kept = len(given), [cap, cap, cap, cap, cap - 1, 0, 0]
    tab, pages = _tables(g, [cap] * n, size)
    kp, vp = _pool(g, pages, heads, size, dtype, False)
    pool = hg.hg_pages_create(kp, vp)
    q, k, v = (_randn(g, n, h, D, dtype=dtype) for h in (hq, heads, heads))
    rot = hg.Rotation(table(64, D, "cuda")) if rotated else None
    pos = torch.randint(0, 64, (n,), generator=g, device="cuda", dtype=torch.int32)
    kq, vq, q_rot = kp.clone(), vp.clone(), torch.empty_like(q)
    slots = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    for b in (0, 4):  # the two that have a place
        slots[b] = tab[b, (given[b] - 1) // size] * size + (given[b] - 1) % size
    hg.hg_pages_append(hg.hg_pages_create(kq, vq), q, k, v, rot, pos, slots, q_rot)
    ws = _workspace(hg.hg_pages_decode_workspace_size(pool, n, hq))
    out, lse = torch.full((n, hq, D), NAN, dtype=dtype, device="cuda"), torch.full((n, hq), NAN, device="cuda")
    lens = torch.tensor(given, dtype=torch.int32, device="cuda")
    hg.hg_pages_decode_step(pool, q, k, v, rot, pos, tab, lens, out, lse, 0.0, ws)
    assert hg.hg_workspace_status(ws) == 0
    assert torch.equal(_bits(kp), _bits(kq)) and torch.equal(_bits(vp), _bits(vq))
    _check_decode(q_rot, kp, vp, tab, kept, size, out, lse)


@TYPES
@pytest.mark.parametrize("causal", [True, False])
def test_prompt_keys_that_are_nan_over_whole_pieces(dtype, causal):
    """Few rows over long keys are joined from pieces: one whose scores are all NaN makes its rows NaN like any other."""
    g = _gen(60)
    nq, nk, heads, group = 40, 9000, 4, 7
    q, k, v, qb, kb = _prompt(g, [nq, 30], [nk, 30], heads, group, dtype, "tokens")
    k[1000:3100, 1] = NAN
    q[7, 3] = NAN
    out, lse = _run_prompt(q, k, v, qb, kb, causal)
    sick = torch.zeros(nq + 30, heads * group, dtype=torch.bool, device="cuda")
    sick[:nq, group:2 * group] = True
    sick[7, 3] = True
    assert bool(out[sick].isnan().all()) and bool(lse[sick].isnan().all())
    assert bool(out[~sick].isfinite().all()) and bool(lse[~sick].isfinite().all())
    whole = [h for h in range(heads * group) if h // group != 1 and h != 3]
    for h in whole[::5]:
        kv = h // group
        _check_prompt(q[:, h:h + 1], k[:, kv:kv + 1], v[:, kv:kv + 1], qb, kb, causal, out[:, h:h + 1], lse[:, h:h + 1])


def _small_terms(keys, heads, at, dtype):
    """Keys at `at` whose probability is 1, all the others' about 2^-25.4 each; the others' values alone are not 0."""
    g = _gen(keys)
    k, v = (torch.zeros(keys, heads, D, dtype=dtype, device="cuda") for _ in range(2))
    k[:, :, 0] = (torch.rand((keys, heads), generator=g, device="cuda") * 0.6 - 0.3).to(dtype)
    v[:] = (1000.0 + 10.0 * torch.randn((keys, heads, D), generator=g, device="cuda")).to(dtype)
    k[at, :, 0], v[at] = 17.59375, 0.0
    return k, v


def _check_small_terms(out, lse, q, k, v, seen, scale):
    """As `check`, with what FP16 cannot hold of a probability 2^7 times larger: half of 2^-24, times 2^-7."""
    ref, rlse, mean, big = attend(q, k, v, seen, scale)
    u, delta = ROUNDOFF[q.dtype], 2.0 ** -17 * big + 2.0 ** -20
    tol = u * ref.abs() + (u + 2.0 * delta[..., None]) * mean * 1.01 + 2.0 ** -25
    if q.dtype == F16:
        tol = tol + 2.0 ** -32 * k.shape[0] * float(v.double().abs().max())
    assert float(ref.min()) > 8.0 * float(tol.max())  # the terms show: 2^6.6 over the largest keys' number (3 to 8)
    assert bool(((out.double() - ref).abs() <= tol).all())
    assert bool(((lse.double() - rlse).abs() <= delta + 2.0 ** -22 * rlse.abs() + 2.0 ** -20).all())


@TYPES
@pytest.mark.parametrize("heads,group", [(8, 4), (8, 12)])
def test_decode_many_small_terms(dtype, heads, group):
    """Requests that are not cut: the first tiles of every warp hold the largest score, thousands of keys follow."""
    size, n, length = 64, 48, 8000
    tab, pages = _tables(_gen(70), [length] * n, size)
    kp, vp = (torch.zeros((pages, heads, size, D), dtype=dtype, device="cuda") for _ in range(2))
    k, v = _small_terms(length, heads, torch.tensor([0, 32, 64]), dtype)
    for pool, x in ((kp, k), (vp, v)):
        pool[tab.long()] = x.view(length // size, size, heads, D).transpose(1, 2)
    q = torch.zeros(n, heads * group, D, dtype=dtype, device="cuda")
    q[:, :, 0] = 1.0
    pool = hg.hg_pages_create(kp, vp)
    ws = _workspace(hg.hg_pages_decode_workspace_size(pool, n, heads * group))
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    lens = torch.full((n,), length, dtype=torch.int32, device="cuda")
    hg.hg_pages_decode_attention(pool, q, tab, lens, out, lse, 1.0, ws)
    for b in (0, 17, n - 1):
        _check_small_terms(out[b:b + 1], lse[b:b + 1], q[b:b + 1], k, v, lens[b:b + 1].long(), 1.0)


@TYPES
@pytest.mark.parametrize("nq,nk,copies", [(300, 60000, 1), (16, 9000, 40)])  # (cut in pieces; and not)
def test_prompt_many_small_terms(dtype, nq, nk, copies):
    heads, group = 4, 8
    k, v = _small_terms(nk, heads, torch.arange(0, nk, 8192), dtype)
    q = torch.zeros(nq * copies, heads * group, D, dtype=dtype, device="cuda")
    q[:, :, 0] = 1.0
    qb, kb = (torch.arange(copies + 1, dtype=torch.int32) * n for n in (nq, nk))
    out, lse = _run_prompt(q, k.repeat(copies, 1, 1), v.repeat(copies, 1, 1), qb, kb, False, scale=1.0)
    for i in {0, copies // 2, copies - 1}:
        rows = slice(i * nq, i * nq + 8)
        _check_small_terms(out[rows], lse[rows], q[rows], k, v, torch.full((8,), nk, device="cuda"), 1.0)


def test_decode_workspace_of_another_pool():
    """A workspace made for a pool of one KV head serves a pool of many, at the same batch and below."""
    g = _gen(80)
    small = hg.hg_pages_create(*_pool(g, 2, 1, 16, BF16, False))
    ws = _workspace(hg.hg_pages_decode_workspace_size(small, 37, 1))
    for heads, group, lens in [(64, 1, [5, 900] * 18 + [3]), (1, 16, [4000] * 37), (32, 2, [20000])]:
        tab, pages = _tables(g, lens, 32)
        kp, vp = _pool(g, pages, heads, 32, BF16, False)
        pool = hg.hg_pages_create(kp, vp)
        q = _randn(g, len(lens), heads * group, D)
        for _ in range(2):
            out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
            hg.hg_pages_decode_attention(pool, q, tab, torch.tensor(lens, dtype=torch.int32, device="cuda"), out, lse, 0.0, ws)
            _check_decode(q[:3], kp, vp, tab[:3], lens[:3], 32, out[:3], lse[:3])
    assert hg.hg_workspace_status(ws) == 0


@TYPES
@pytest.mark.parametrize("top", [22, 24, 26, 28, 30])
def test_prompt_scores_whose_maxima_round_alike(dtype, top):
    """Scores 2^k apart around 2^`top` in units of the exponent, where binary32 holds their scaled maxima half as finely as
    the scores themselves: keys far above the maximum so far are found all the same, whatever the maxima round to."""
    # score = 2^15 * 65024 + 128 j exactly (binary32 holds it); times scale log2(e) just above 2^top
    heads, group, n = 2, 4, 4
    base, step = 32768.0 * 65024.0, 128.0
    keys = 128 * (n + 1)
    g = _gen(top)
    for i in range(12):
        scale = float(torch.tensor(2.0 ** top * (1.001 + 0.0007 * i) / base * math.log(2.0), dtype=torch.float32))
        j = torch.zeros(keys, dtype=torch.float64, device="cuda")
        for b in range(1, n + 1):  # each block's first key a few steps above the block before
            j[128 * b:] += (i + b) % 4
        q, k = torch.zeros(32, heads * group, D, dtype=dtype, device="cuda"), torch.zeros(keys, heads, D, dtype=dtype, device="cuda")
        q[:, :, 0], q[:, :, 1], k[:, :, 0], k[:, :, 1] = 32768.0, step, 65024.0, j.to(dtype)[:, None]
        v = _randn(g, keys, heads, D, dtype=dtype)
        begin = [torch.tensor([0, x], dtype=torch.int32) for x in (32, keys)]
        out, lse = _run_prompt(q, k, v, *begin, False, scale=scale)
        s = (base + step * j) * scale
        w = torch.softmax(s, 0)
        ref = torch.einsum("k,khd->hd", w, v.double()).repeat_interleave(group, 0)
        mean = torch.einsum("k,khd->hd", w, v.double().abs()).repeat_interleave(group, 0)
        u = ROUNDOFF[dtype]
        # (a term's exponent is a difference of at most 64 units, 2^-23 of which its factors' roundings move)
        tol = u * ref.abs() + (u + 2.0 ** -16) * mean * 1.01 + 2.0 ** -25 + 2.0 ** -32 * keys * float(v.abs().max())
        assert bool(((out.double() - ref).abs() <= tol).all())
        assert bool(((lse.double() - torch.logsumexp(s, 0)).abs() <= 2.0 ** -21 * float(s.max())).all())
