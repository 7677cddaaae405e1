"""Performance cases of the operators for paged caches held in 8 bits, and of page tables built on the GPU: what is
timed, on which inputs, the same results in plain torch and in 64 bits.

A case is one pass through one operator as a serving program calls it:

  plan     page tables, slot map and positions from request lengths, pages taken from and given back to a free list
           (hg_pages_plan)
  append   a batch's new tokens: queries and keys rotated by their positions, keys and values rounded to e4m3 with a
           scale for each 16 tokens and head, stored in pages (hg_pages8_append)
  decode   attention of one new token per request over the 8-bit pages (hg_pages8_decode_attention)
  step     the same with the new token's rotation and its store in the cache (hg_pages8_decode_step)
  dense    the tokens of the 8-bit pages as dense 16-bit rows (hg_pages8_dequantize)

Inputs: K ~ N(0, 1) with four outlier channels 8z + 3 per KV head, Q and V ~ N(0, 1).
"""
import math

import torch

own = False  # set by the tools that measure: False computes the plain form, True calls the package

D = 128
BLOCK = 16  # tokens that share a scale (with their head)
BF16, F16 = "bf16", "f16"
_TYPES = {BF16: torch.bfloat16, F16: torch.float16}
F8 = torch.float8_e4m3fn
F8_MAX = 448.0


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------

def _case(name, op, dtype, kv_heads, group, batch, longest, spread=False, context=0, page=16, token_major=False,
          rot_dim=128, interleaved=False, mrope=False, keep_k=True, ending=0):
    """`longest`: tokens of the longest request (new ones for plan and append, cached ones otherwise); `spread`: the
    requests' tokens run from 1 to it evenly in their logarithm, else all have it; `context`: about as many tokens are
    cached before the new ones (plan, append); `token_major`: pages lie [tokens][heads], else heads first; `keep_k`:
    the rotated keys are wanted as a dense 16-bit tensor too; `ending`: every so many-th request ends (plan)."""
    return {"name": name, "op": op, "dtype": dtype, "kv_heads": kv_heads, "group": group, "batch": batch,
            "longest": longest, "spread": spread, "context": context, "page": page, "token_major": token_major,
            "rot_dim": rot_dim, "interleaved": interleaved, "mrope": mrope, "keep_k": keep_k, "ending": ending}


def listed():
    return [
        # Every token of a running batch: one more token for each request, a few of which have ended.
        _case("plan_step", "plan", BF16, 1, 1, 64, 1, context=1475, ending=9),
        # A wave of prompts admitted at once beside requests that end.
        _case("plan_prompts", "plan", BF16, 1, 1, 1000, 4001, spread=True, context=700, page=32, ending=7),
        # The smallest append: a running batch's new tokens, each in a block that has tokens already.
        _case("append8_token", "append", BF16, 4, 7, 16, 1, context=1474, mrope=True, keep_k=False),
        # A Qwen2.5-VL-7B-shaped prompt, image and text, with three-part positions.
        _case("append8_prompt", "append", BF16, 4, 7, 1, 1460, mrope=True),
        # Pieces of prompts of many lengths after cached tokens: 12 queries per KV head, half of the channels rotated
        # as neighbours.
        _case("append8_packed", "append", F16, 5, 12, 48, 4001, spread=True, context=333, page=64, token_major=True,
              rot_dim=64, interleaved=True),
        # One request with a short context: the latency of a token.
        _case("decode8_short", "decode", BF16, 4, 7, 1, 321),
        # Requests of all ages side by side, 12 queries per KV head.
        _case("decode8_mixed", "decode", F16, 5, 12, 37, 9001, spread=True, page=32, token_major=True),
        # A Qwen2.5-VL-7B-shaped batch generates a token: rotation, store and attention.
        _case("step8_7b", "step", BF16, 4, 7, 16, 1475, mrope=True),
        # A Qwen2.5-VL-72B-shaped batch with long contexts.
        _case("decode8_72b", "decode", BF16, 8, 8, 32, 8577, page=64),
        # One request with a very long context: the work lies along the cache.
        _case("decode8_long", "decode", BF16, 8, 4, 1, 131073, page=128),
        # The cached tokens that the next piece of one long prompt attends to.
        _case("dense8_chunk", "dense", BF16, 4, 7, 1, 16064),
        # The same for a Qwen2.5-VL-72B-shaped batch of requests of all ages.
        _case("dense8_72b", "dense", F16, 8, 8, 24, 8577, spread=True, page=64, token_major=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# A drawn case costs at most about this: bytes moved; tokens that a plan places.
_DRAW_BYTES, _DRAW_TOKENS = 3e8, 300000


def draw(rng):
    op = rng.choice(["plan", "append", "append", "decode", "decode", "decode", "step", "dense"])
    kv, group = rng.choice([(4, 7), (8, 8), (8, 4), (32, 1), (2, 16), (5, 12), (1, 8), (16, 2), (3, 5)])
    c = _case("", op, rng.choice([BF16, F16]), kv, group, _log(rng, 1, 64), 1, rng.random() < 0.5,
              page=rng.choice([16, 32, 64, 128, 256]), token_major=rng.random() < 0.5,
              rot_dim=rng.choice([128, 128, 64, 32]), interleaved=rng.random() < 0.3, keep_k=rng.random() < 0.7)
    c["mrope"] = c["rot_dim"] == 128 and not c["interleaved"] and rng.random() < 0.5
    c["longest"] = _log(rng, 1, 8192) if op in ("plan", "append") else _log(rng, 1, 16384)
    if op in ("plan", "append") and rng.random() < 0.6:
        c["context"] = _log(rng, 1, 4096)
    if op == "plan":
        c["batch"] = _log(rng, 1, 2048)
        c["ending"] = rng.choice([0, 0, 2, 5, 11])
    while work(c)["bytes"] > _DRAW_BYTES or (op == "plan" and sum(_lengths(c)) > _DRAW_TOKENS):
        widest = max(("batch", "longest"), key=lambda n: math.log(c[n]) / (1 if n == "longest" else 0.5))
        c[widest] = max(1, c[widest] * 3 // 4)
    del c["name"]
    return c


def _lengths(c):
    """Tokens of each request, longest last."""
    n, top = c["batch"], c["longest"]
    if not c["spread"] or n == 1:
        return [top] * n
    return [max(1, int(round(top ** (i / (n - 1))))) for i in range(n)]


def _cached(c):
    """Tokens that each request has before the call, at every place of a block."""
    return [max(0, c["context"] - 7 * i % BLOCK) for i in range(c["batch"])]


def _ends(c):
    return [c["ending"] > 0 and i % c["ending"] == c["ending"] - 1 for i in range(c["batch"])]


def work(c):
    kv, hq, lens = c["kv_heads"], c["kv_heads"] * c["group"], _lengths(c)
    n, ps = len(lens), c["page"]
    row = D * 2
    if c["op"] == "plan":
        # two lengths in, one length and one begin out a request; an id in and out for every page that changes hands;
        # a slot and a position a token
        pages = tokens = 0
        for new, cached, end in zip(lens, _cached(c), _ends(c)):
            have = -(-cached // ps)
            pages += have if end else -(-(cached + new) // ps) - have
            tokens += 0 if end else new
        return {"bytes": 16 * n + 8 * pages + 8 * tokens, "flops": 4 * tokens + 8 * n}
    total = sum(lens)
    if c["op"] == "append":
        # every row read once; queries and, where wanted, dense keys written in 16 bits, keys and values in 8; the
        # scales; a table row, a position and a page id for each token's needs
        blocks = sum(-(-(a + t) // BLOCK) - a // BLOCK for a, t in zip(_cached(c), lens))
        b = total * (row * (2 * hq + 2 * kv + (kv if c["keep_k"] else 0)) + 2 * kv * D)
        b += 8 * kv * blocks + total * (c["rot_dim"] * 4 + 4 * (3 if c["mrope"] else 1)) + 12 * n
        return {"bytes": b, "flops": total * ((hq + kv) * c["rot_dim"] * 3 + 4 * kv * D)}
    pages, blocks = sum(-(-t // ps) for t in lens), sum(-(-t // BLOCK) for t in lens)
    held = 2 * kv * (total * D + 4 * blocks) + 4 * pages + 4 * n  # codes, scales, page ids, lengths
    if c["op"] == "dense":
        return {"bytes": held + 2 * total * kv * row, "flops": 2 * total * kv * D}
    b = held + n * hq * (2 * row + 4)
    if c["op"] == "step":
        b += n * (2 * kv * (row + D + 4) + c["rot_dim"] * 4 + 4 * (3 if c["mrope"] else 1))
    return {"bytes": b, "flops": 4 * D * hq * total}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _ints(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def _begins(lens):
    return torch.tensor([0] + lens).cumsum(0)


def _keys(shape, heads_at, g, dev):
    """N(0, 1) with four outlier channels 8z + 3 per head (axis `heads_at`), float32."""
    heads = shape[heads_at]
    scale = torch.ones(heads, D, device=dev)
    off = torch.zeros(heads, D, device=dev)
    at = torch.rand(heads, D, generator=g, device=dev).argsort(1)[:, :4]
    scale.scatter_(1, at, 8.0)
    off.scatter_(1, at, 3.0)
    view = [1] * len(shape)
    view[heads_at], view[-1] = heads, D
    x = torch.randn(shape, generator=g, device=dev)
    return x.mul_(scale.view(view)).add_(off.view(view))


def _power(amax):
    """The least power of two s with amax <= 448 s, 2^-126 at least (448 = 1.75 * 2^8)."""
    part, e = torch.frexp(amax)  # amax = part 2^e, part in [0.5, 1)
    e = torch.where(amax > 0, e - 9 + (part > 0.875).to(e.dtype), torch.full_like(e, -126)).clamp(min=-126)
    return torch.ldexp(torch.ones_like(amax), e)


def _quantized(x):
    """x [pages][heads][page][D] float32 -> e4m3 codes, scales [pages][heads][page / 16]."""
    shape = x.shape
    x = x.view(shape[0], shape[1], -1, BLOCK * D)
    s = _power(x.abs().amax(-1))
    return (x / s[..., None]).to(F8).view(shape), s


def _table(length, rot_dim, dev):
    """Cosines and sines of every position: [length][rot_dim], the cosines of the rot_dim / 2 pairs first."""
    half = rot_dim // 2
    freq = 1e6 ** (-torch.arange(half, dtype=torch.float64, device=dev) / half)
    angle = torch.arange(length, dtype=torch.float64, device=dev)[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _positions(c, first, g, dev):
    """Positions of the new tokens: one each, or three (time, height, width) as an image's patches have them."""
    if not c["mrope"]:
        return first
    patch = torch.randint(0, 36, (2, first.numel()), generator=g, device=dev, dtype=torch.int32)
    return torch.stack([first, first // 2 + patch[0], first // 3 + patch[1]])


def _sections(c):
    """Pairs that turn by each of the three positions, as Qwen2.5-VL divides its 64."""
    return (16, 24, 24) if c["mrope"] else (c["rot_dim"] // 2, 0, 0)


def _page_table(per, extra, g, dev):
    """Each request's pages, of a pool that holds `extra` more, in no order; and the pool's other pages."""
    n, used = len(per), sum(per)
    order = torch.randperm(used + extra, generator=g, device=dev).to(torch.int32)
    table = torch.zeros(n, max(max(per), 1), dtype=torch.int32, device=dev)
    row = torch.repeat_interleave(torch.arange(n, device=dev), torch.tensor(per, device=dev))
    col = torch.arange(used, device=dev) - _begins(per).to(dev)[row]
    table[row, col] = order[:used]
    return table, order[used:]


def _prepare_plan(c, g, dev):
    lens, cached, ends, ps = _lengths(c), _cached(c), _ends(c), c["page"]
    have, want = ([-(-t // ps) for t in x] for x in (cached, [a + t for a, t in zip(cached, lens)]))
    table, free = _page_table(have, sum(want) - sum(have) + 64, g, dev)
    wide = torch.zeros(len(lens), max(want) + 2, dtype=torch.int32, device=dev)
    wide[:, :table.shape[1]] = table
    room = sum(lens)
    # the list has room for every page of the pool; its first entries are the free ones
    held = torch.full((free.numel() + sum(have),), -1, dtype=torch.int32, device=dev)
    held[:free.numel()] = free
    n = len(lens)
    return {"table": wide, "cached": _ints(cached, dev), "new": _ints([-1 if e else t for t, e in zip(lens, ends)], dev),
            "free": held, "free_count": _ints([free.numel()], dev), "lengths": torch.empty(n, dtype=torch.int32, device=dev),
            "begin": torch.empty(n + 1, dtype=torch.int32, device=dev),
            "slots": torch.empty(room, dtype=torch.int32, device=dev),
            "positions": torch.empty(room, dtype=torch.int32, device=dev),
            "counts": torch.empty(4, dtype=torch.int32, device=dev)}


def prepare(case, seed):
    c, dev = case, _device()
    dtype = _TYPES[c["dtype"]]
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 7919 + 13)
    s = {"case": c}
    if c["op"] == "plan":
        return {**s, **_prepare_plan(c, g, dev)}
    kv, hq, lens, ps = c["kv_heads"], c["kv_heads"] * c["group"], _lengths(c), c["page"]
    n, total = len(lens), sum(lens)
    cached = _cached(c) if c["op"] == "append" else [t - 1 for t in lens]
    after = [a + t for a, t in zip(cached, lens)] if c["op"] == "append" else lens
    per = [-(-t // ps) for t in after]
    s["table"], _ = _page_table(per, max(4, sum(per) // 16), g, dev)
    pool = sum(per) + max(4, sum(per) // 16)
    s["lens"] = _ints(after, dev)
    # what the pages hold before the call: a cache that was filled in the same way
    for x, fill in (("k", lambda shape: _keys(shape, 1, g, dev)),
                    ("v", lambda shape: torch.randn(shape, generator=g, device=dev))):
        codes, s[x + "_scales"] = _quantized(fill((pool, kv, ps, D)))
        # seen as [pages][heads][tokens][channels], whatever the order in memory
        s[x + "_pages"] = codes.view(torch.uint8).transpose(1, 2).contiguous().transpose(1, 2).view(F8) \
            if c["token_major"] else codes
        del codes
    if c["op"] in ("append", "step"):
        # a fused projection's output: queries, keys and values of a token side by side
        rows = total if c["op"] == "append" else n
        qkv = torch.empty((rows, hq + 2 * kv, D), dtype=dtype, device=dev)
        qkv[:, :hq] = torch.randn((rows, hq, D), generator=g, device=dev)
        qkv[:, hq:hq + kv] = _keys((rows, kv, D), 1, g, dev)
        qkv[:, hq + kv:] = torch.randn((rows, kv, D), generator=g, device=dev)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + kv], qkv[:, hq + kv:]
        if c["op"] == "append":
            s["begin"] = _begins(lens).to(torch.int32).to(dev)
            seq = torch.repeat_interleave(torch.arange(n, device=dev), torch.tensor(lens, device=dev))
            at = torch.arange(total, device=dev) - s["begin"].long()[seq] + torch.tensor(cached, device=dev)[seq]
            s["positions"] = _positions(c, at.to(torch.int32), g, dev)
        else:
            s["positions"] = _positions(c, _ints(cached, dev), g, dev)
        s["rotation"] = _table(max(after) + 64, c["rot_dim"], dev)
    elif c["op"] == "decode":
        s["q"] = torch.randn((n, hq, D), generator=g, device=dev).to(dtype)
    if c["op"] == "append":
        s["q_out"] = torch.empty((total, hq, D), dtype=dtype, device=dev)
        s["k_out"] = torch.empty((total, kv, D), dtype=dtype, device=dev) if c["keep_k"] else None
    elif c["op"] == "dense":
        s["begin"] = _begins(lens).to(torch.int32).to(dev)
        s["k_out"], s["v_out"] = (torch.empty((kv, total, D), dtype=dtype, device=dev).transpose(0, 1) for _ in "kv")
    else:
        s["out"] = torch.empty((n, hq, D), dtype=dtype, device=dev)
        s["lse"] = torch.empty((n, hq), device=dev)
    if own:
        import paper_2609_35800_gb300 as hg
        s["pages"] = hg.hg_pages8_create(s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"], dtype)
        if c["op"] in ("append", "step"):
            s["rot"] = hg.Rotation(s["rotation"], interleaved=c["interleaved"],
                                   sections=_sections(c) if c["mrope"] else None)
        if c["op"] in ("decode", "step"):
            s["ws"] = torch.empty(hg.hg_pages8_decode_workspace_size(s["pages"], n, hq), dtype=torch.uint8, device=dev)
            hg.hg_workspace_clear(s["ws"])
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _planned(s):
    return {x: s[x] for x in ("table", "lengths", "begin", "slots", "positions", "counts", "free")}


def _held(s):
    return {x: s[x] for x in ("k_pages", "v_pages", "k_scales", "v_scales")}


def _run_own(s):
    import paper_2609_35800_gb300 as hg
    c = s["case"]
    if c["op"] == "plan":
        hg.hg_pages_plan(s["table"], s["cached"], s["new"], s["free"], s["free_count"], c["page"], s["lengths"],
                         s["begin"], s["slots"], s["positions"], s["counts"])
        return _planned(s)
    if c["op"] == "append":
        hg.hg_pages8_append(s["pages"], s["q"], s["k"], s["v"], s["rot"], s["positions"], s["begin"], s["table"],
                            s["lens"], s["q_out"], s["k_out"])
        return _appended(s, s["q_out"], s["k_out"])
    if c["op"] == "dense":
        hg.hg_pages8_dequantize(s["pages"], s["begin"], s["table"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    if c["op"] == "decode":
        hg.hg_pages8_decode_attention(s["pages"], s["q"], s["table"], s["lens"], s["out"], s["lse"], 0.0, s["ws"])
        return {"out": s["out"], "lse": s["lse"]}
    hg.hg_pages8_decode_step(s["pages"], s["q"], s["k"], s["v"], s["rot"], s["positions"], s["table"], s["lens"],
                             s["out"], s["lse"], 0.0, s["ws"])
    return {"out": s["out"], "lse": s["lse"], **_held(s)}


def _appended(s, q_out, k_out):
    out = {"q": q_out, **_held(s)}
    if k_out is not None:
        out["k"] = k_out
    return out


def _plan_plain(s):
    ps, dev = s["case"]["page"], s["table"].device
    cached, new, table, free = s["cached"].long(), s["new"].long(), s["table"].long(), s["free"].long()
    count, room = s["free_count"].long(), s["slots"].numel()
    ends = new < 0
    have = (cached + ps - 1) // ps
    after = torch.where(ends, torch.zeros_like(cached), cached + new)
    want = torch.where(ends, have, (cached + new + ps - 1) // ps)
    col = torch.arange(table.shape[1], device=dev)
    # pages given back, request by request, behind the free ones; taken from the end
    back = (ends[:, None] & (col < have[:, None])).flatten()
    rank = back.long().cumsum(0) - 1
    freed = back.sum()
    at = torch.where(back, count + rank, torch.full_like(rank, free.numel()))
    pile = torch.cat([free, free[:1]]).scatter(0, at, table.flatten())[:-1]
    take = want - have
    first = take.cumsum(0) - take
    taken = take.sum()
    fresh = (col >= have[:, None]) & (col < want[:, None])
    which = (count + freed - 1 - first[:, None] - (col - have[:, None])).clamp(0, pile.numel() - 1)
    table = torch.where(fresh, pile[which], table)
    tokens = torch.where(ends, torch.zeros_like(new), new)
    begin = torch.cat([torch.zeros_like(count), tokens.cumsum(0)])
    i = torch.arange(room, device=dev)
    r = torch.searchsorted(begin[1:].contiguous(), i, right=True).clamp(max=cached.numel() - 1)
    t = cached[r] + i - begin[r]
    placed = i < begin[-1]
    slots = torch.where(placed, table[r, (t // ps).clamp(0, table.shape[1] - 1)] * ps + t % ps, torch.full_like(t, -1))
    left = count + freed - taken
    # behind the free ones that were there, what is left of the pages given back
    behind = torch.arange(free.numel(), device=dev)
    free = torch.where((behind >= count) & (behind < left), pile, free)
    s["table"].copy_(table)
    s["free"].copy_(free)
    s["lengths"].copy_(after)
    s["begin"].copy_(begin)
    s["slots"].copy_(slots)
    s["positions"].copy_(torch.where(placed, t, torch.zeros_like(t)))
    s["counts"].copy_(torch.cat([left, torch.zeros_like(count), begin[-1:], after.max().view(1)]))
    return _planned(s)


def _angles(s):
    """Cosine and sine of every (token, pair)."""
    c = s["case"]
    half = c["rot_dim"] // 2
    if not c["mrope"]:
        rows = s["rotation"][s["positions"].long()]
        return rows[:, :half], rows[:, half:]
    which = torch.tensor([0] * 16 + [1] * 24 + [2] * 24, device=s["positions"].device)
    pos = s["positions"].long()[which].t()
    pair = torch.arange(half, device=pos.device)
    return s["rotation"][pos, pair], s["rotation"][pos, half + pair]


def _rotated(x, cos, sin, c):
    """x [tokens][heads][128] turned in 32 bits."""
    r, x = c["rot_dim"], x.float()
    cos, sin = cos[:, None], sin[:, None]
    if c["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _store(s, x, rows, seq, at, cached):
    """rows [tokens][heads][D] float32: tokens `at` of the requests `seq`, which had `cached` tokens, into the pages."""
    c, codes, scales = s["case"], s[x + "_pages"].view(torch.uint8), s[x + "_scales"]
    ps, table = c["page"], s["table"].long()
    page, block = table[seq, at // ps], at % ps // BLOCK
    # the new tokens' scale of each block, and the one of the tokens that it has
    flat = page * (ps // BLOCK) + block
    top = torch.zeros(scales.shape[0] * scales.shape[2], scales.shape[1], device=rows.device)
    top = top.scatter_reduce(0, flat[:, None].expand(-1, scales.shape[1]), rows.abs().amax(-1), "amax")
    need = _power(top)[flat]
    had = (at // BLOCK * BLOCK < cached[seq])[:, None]
    new = torch.where(had, torch.maximum(need, scales[page, :, block]), need)
    # the tokens in a request's last block so far, over to the block's new scale
    tail = cached // BLOCK * BLOCK
    row = tail[:, None] + torch.arange(BLOCK, device=rows.device)
    mine = torch.arange(len(cached), device=rows.device)
    old_page = table[mine, (tail // ps).clamp(max=table.shape[1] - 1)]
    old_block = tail % ps // BLOCK
    before = scales[old_page, :, old_block]
    scales[page, :, block] = new
    ratio = before / scales[old_page, :, old_block]
    stay = (row < cached[:, None])[:, None, :, None]
    index = (old_page[:, None, None], torch.arange(codes.shape[1], device=rows.device)[None, :, None], (row % ps)[:, None])
    kept = codes[index]
    moved = (kept.view(F8).float() * ratio[:, :, None, None]).to(F8).view(torch.uint8)
    codes[index] = torch.where(stay, moved, kept)
    codes[page, :, at % ps] = (rows / new[..., None]).to(F8).view(torch.uint8)


def _values(s, x):
    """What the pages hold, float32 [pages][heads][page][D]."""
    scales = s[x + "_scales"].repeat_interleave(BLOCK, dim=2)
    return s[x + "_pages"].float() * scales[..., None]


def _attend(scores, seen, values):
    """Softmax over the last axis where `seen`, times the values; and the scores' log-sum-exp."""
    scores = scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, values) / torch.where(total == 0, torch.ones_like(total), total)
    return out, (top + total.log()).squeeze(-1)


def _run_plain(s):
    c = s["case"]
    if c["op"] == "plan":
        return _plan_plain(s)
    dtype, kv, grp, ps = _TYPES[c["dtype"]], c["kv_heads"], c["group"], c["page"]
    dev, lens, table = s["table"].device, s["lens"].long(), s["table"].long()
    n = len(lens)
    if c["op"] in ("append", "dense"):
        begin, rows = s["begin"].long(), (s["k"] if c["op"] == "append" else s["k_out"]).shape[0]
        i = torch.arange(rows, device=dev)
        seq = torch.searchsorted(begin[1:].contiguous(), i, right=True)
        first = lens - (begin[1:] - begin[:-1])
        at = first[seq] + i - begin[seq]
    if c["op"] == "append":
        cos, sin = _angles(s)
        q, k = (_rotated(s[x], cos, sin, c) for x in "qk")
        _store(s, "k", k, seq, at, first)
        _store(s, "v", s["v"].float(), seq, at, first)
        return _appended(s, q.to(dtype), k.to(dtype) if c["keep_k"] else None)
    if c["op"] == "dense":
        out = {}
        for x in "kv":
            scale = s[x + "_scales"][table[seq, at // ps], :, at % ps // BLOCK]
            codes = s[x + "_pages"].view(torch.uint8)[table[seq, at // ps], :, at % ps].view(F8)
            s[x + "_out"].copy_(codes.float() * scale[..., None])
            out[x] = s[x + "_out"]
        return out
    q = s["q"]
    if c["op"] == "step":
        cos, sin = _angles(s)
        q, k = (_rotated(s[x], cos, sin, c) for x in "qk")
        q = q.to(dtype)
        mine = torch.arange(n, device=dev)
        _store(s, "k", k, mine, lens - 1, lens - 1)
        _store(s, "v", s["v"].float(), mine, lens - 1, lens - 1)
    k, v = (_values(s, x)[table].permute(0, 2, 1, 3, 4).reshape(n, kv, -1, D) for x in "kv")
    scores = torch.matmul(q.reshape(n, kv, grp, D).float(), k.transpose(2, 3)) * (D ** -0.5)
    seen = torch.arange(k.shape[2], device=dev) < lens[:, None]
    out, lse = _attend(scores, seen[:, None, None], v)
    got = {"out": out.reshape(n, kv * grp, D).to(dtype), "lse": lse.reshape(n, kv * grp)}
    return got if c["op"] == "decode" else {**got, **_held(s)}


# ---------------------------------------------------------------------------
# In 64 bits, from the definitions
# ---------------------------------------------------------------------------

def _turn64(x, s):
    """Channel by channel: each pair is a complex number times e^(i angle)."""
    c = s["case"]
    half = c["rot_dim"] // 2
    x = x.double().clone()
    table = s["rotation"].double()
    pos = s["positions"].long()
    for m in range(half):
        which = 0 if not c["mrope"] else 0 if m < 16 else 1 if m < 40 else 2
        p = pos[which] if c["mrope"] else pos
        unit = torch.complex(table[p, m], table[p, half + m])
        a, b = (2 * m, 2 * m + 1) if c["interleaved"] else (m, m + half)
        z = torch.complex(x[:, :, a], x[:, :, b]) * unit[:, None]
        x[:, :, a], x[:, :, b] = z.real, z.imag
    return x


def _append64(codes, scales, table, rows, first, ps):
    """One request's rows [tokens][heads][D] from its token `first` on, block by block, into codes [pages][heads][page][D]
    (64 bits, not rounded to e4m3) and scales."""
    end = first + rows.shape[0]
    block = first // BLOCK
    while block * BLOCK < end:
        lo, hi = max(first, block * BLOCK), min(end, (block + 1) * BLOCK)
        page, at = table[block * BLOCK // ps], block * BLOCK % ps
        new = rows[lo - first:hi - first]
        amax = new.abs().amax((0, 2))
        s = torch.clamp(torch.ceil(torch.log2(amax / F8_MAX)), min=-126.0)
        s = torch.where(amax > 0, 2.0 ** s, torch.full_like(s, 2.0 ** -126))
        if block * BLOCK < first:
            old = scales[page, :, at // BLOCK]
            s = torch.maximum(s, old)
            codes[page, :, at:at + lo % BLOCK] *= (old / s)[:, None, None]
        scales[page, :, at // BLOCK] = s
        codes[page, :, lo % ps:lo % ps + hi - lo] = (new / s[:, None]).transpose(0, 1)
        block += 1


def exact(case, seed):
    c = case
    if c["op"] == "plan":
        return None  # whole numbers
    s = prepare(case, seed)
    lens, ps, dev = s["lens"].tolist(), c["page"], s["table"].device
    dtype, kv = _TYPES[c["dtype"]], c["kv_heads"]
    grp = c["group"]
    held = {}
    q = s.get("q")
    if c["op"] in ("append", "step"):
        new = _lengths(c) if c["op"] == "append" else [1] * len(lens)
        q = _turn64(s["q"], s)
        k = _turn64(s["k"], s)
        for x, rows in (("k", k), ("v", s["v"].double())):
            codes, scales = s[x + "_pages"].double(), s[x + "_scales"].double()
            at = 0
            for b, t in enumerate(new):
                _append64(codes, scales, s["table"][b].long(), rows[at:at + t], lens[b] - t, ps)
                at += t
            held[x + "_pages"], held[x + "_scales"] = codes, scales
        if c["op"] == "append":
            return {"q": q, **held, **({"k": k} if c["keep_k"] else {})}
        # attention is defined on what is held: rotated queries in the rows' type, codes rounded to e4m3
        q = q.to(dtype)
    out, lse, dense = [], [], {"k": [], "v": []}
    for b, t in enumerate(lens):
        ids = s["table"][b, :-(-t // ps)].long()
        rows = {}
        for x in "kv":
            if held:
                codes, scales = held[x + "_pages"][ids].to(F8).double(), held[x + "_scales"][ids]
            else:
                codes, scales = s[x + "_pages"].view(torch.uint8)[ids].view(F8).double(), s[x + "_scales"][ids].double()
            codes = codes.view(len(ids), kv, ps // BLOCK, BLOCK, D) * scales[..., None, None]
            rows[x] = codes.view(len(ids), kv, ps, D).transpose(1, 2).reshape(-1, kv, D)[:t]
        if c["op"] == "dense":
            dense["k"].append(rows["k"])
            dense["v"].append(rows["v"])
            continue
        sc = torch.einsum("hgd,thd->hgt", q[b].double().view(kv, grp, D), rows["k"]) / math.sqrt(D)
        out.append(torch.einsum("hgt,thd->hgd", torch.softmax(sc, -1), rows["v"]).reshape(1, kv * grp, D))
        lse.append(torch.logsumexp(sc, -1).reshape(1, kv * grp))
    if c["op"] == "dense":
        return {x: torch.cat(v) for x, v in dense.items()}
    return {"out": torch.cat(out), "lse": torch.cat(lse), **held}
