"""Performance cases of the operators for caches that stay BF16 or FP16: what is timed, on which inputs, the same
results in plain torch and in 64 bits.

A case is one pass through one operator as a serving program calls it:

  append   a batch's new tokens: queries and keys rotated by their positions, keys and values stored in a paged cache
           (hg_pages_append)
  decode   attention of one new token per request over the paged cache (hg_pages_decode_attention)
  step     the same with the new token's rotation and its store in the cache (hg_pages_decode_step)
  prompt   causal (or full) attention of packed prompts, grouped heads, optionally after tokens that are cached
           already (hg_prompt_attention)

Inputs: K ~ N(0, 1) with four outlier channels 8z + 3 per KV head, Q and V ~ N(0, 1).
"""
import math

import torch

own = False  # set by the tools that measure: False computes the plain form, True calls the package

D = 128
BF16, F16 = "bf16", "f16"
_TYPES = {BF16: torch.bfloat16, F16: torch.float16}


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------

def _case(name, op, dtype, kv_heads, group, batch, longest, spread=False, context=0, page=16, token_major=False,
          rot_dim=128, interleaved=False, mrope=False, keep_k=True, causal=True):
    """`longest`: tokens of the longest request (its cached ones for decode and step, its new ones otherwise);
    `spread`: the requests' lengths run from 1 to it evenly in their logarithm, else all have it; `context`: cached
    tokens before a prompt's own; `token_major`: pages (prompts: keys and values) lie [tokens][heads], else heads
    first; `keep_k`: the rotated keys are wanted as a dense tensor too."""
    return {"name": name, "op": op, "dtype": dtype, "kv_heads": kv_heads, "group": group, "batch": batch,
            "longest": longest, "spread": spread, "context": context, "page": page, "token_major": token_major,
            "rot_dim": rot_dim, "interleaved": interleaved, "mrope": mrope, "keep_k": keep_k, "causal": causal}


def listed():
    return [
        # The smallest call: one request's new token goes into its cache.
        _case("append_token", "append", BF16, 4, 7, 1, 1, mrope=True, keep_k=False),
        # A Qwen2.5-VL-7B-shaped prompt, image and text, with three-part positions.
        _case("append_prompt", "append", BF16, 4, 7, 1, 1460, mrope=True),
        # Prompts of many lengths at once: 12 queries per KV head, half of the channels rotated as neighbours.
        _case("append_packed", "append", F16, 5, 12, 48, 4001, spread=True, page=64, token_major=True, rot_dim=64,
              interleaved=True),
        # One request with a short context: the latency of a token.
        _case("decode_short", "decode", BF16, 4, 7, 1, 321),
        # Requests of all ages side by side, 12 queries per KV head.
        _case("decode_mixed", "decode", F16, 5, 12, 37, 9001, spread=True, page=32, token_major=True),
        # A Qwen2.5-VL-7B-shaped batch generates a token: rotation, store and attention.
        _case("step_7b", "step", BF16, 4, 7, 16, 1475, mrope=True),
        # A Qwen2.5-VL-72B-shaped batch with long contexts.
        _case("decode_72b", "decode", BF16, 8, 8, 32, 8577, page=64),
        # One request with a very long context: the work lies along the cache.
        _case("decode_long", "decode", BF16, 8, 4, 1, 131073, page=128),
        # Short and long prompts packed into one call.
        _case("prompt_packed", "prompt", F16, 8, 4, 40, 2003, spread=True, token_major=True),
        # A Qwen2.5-VL-7B-shaped prompt.
        _case("prompt_7b", "prompt", BF16, 4, 7, 1, 1460),
        # The next 64 tokens of a prompt whose first 16,000 are cached: few rows, long keys.
        _case("prompt_chunk", "prompt", BF16, 4, 7, 1, 64, context=16000),
        # A Qwen2.5-VL-72B-shaped batch of long prompts.
        _case("prompt_long", "prompt", BF16, 8, 8, 2, 8576),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# A drawn case costs at most about half of the largest listed one: bytes for a cache, scores for a prompt.
_DRAW_BYTES, _DRAW_FLOPS = 6e8, 1.2e12


def draw(rng):
    op = rng.choice(["append", "decode", "decode", "step", "prompt", "prompt"])
    kv, group = rng.choice([(4, 7), (8, 8), (8, 4), (32, 1), (2, 16), (5, 12), (1, 8), (16, 2), (3, 5)])
    c = _case("", op, rng.choice([BF16, F16]), kv, group, _log(rng, 1, 64), 1, rng.random() < 0.5,
              page=rng.choice([16, 32, 64, 128]), token_major=rng.random() < 0.5,
              rot_dim=rng.choice([128, 128, 64, 32]), interleaved=rng.random() < 0.3, keep_k=rng.random() < 0.7,
              causal=rng.random() < 0.8)
    c["mrope"] = c["rot_dim"] == 128 and not c["interleaved"] and rng.random() < 0.5
    c["longest"] = _log(rng, 1, 16384) if op in ("decode", "step") else _log(rng, 1, 8192)
    if op == "prompt" and rng.random() < 0.4:
        c["context"] = _log(rng, 1, 16384)
    limit = {"prompt": ("flops", _DRAW_FLOPS)}.get(op, ("bytes", _DRAW_BYTES))
    while work(c)[limit[0]] > limit[1] or _plain_scores(c) > 2e10:
        widest = max(("batch", "longest"), key=lambda n: math.log(c[n]) / (1 if n == "longest" else 0.5))
        c[widest] = max(1, c[widest] * 3 // 4)
        c["context"] = c["context"] * 7 // 8
    del c["name"]
    return c


def _lengths(c):
    """Tokens of each request, longest last."""
    n, top = c["batch"], c["longest"]
    if not c["spread"] or n == 1:
        return [top] * n
    return [max(1, int(round(top ** (i / (n - 1))))) for i in range(n)]


def _seen(q_len, k_len, causal):
    """Keys that the rows of one prompt see, added up: row i of q_len sees keys up to i + k_len - q_len."""
    if not causal:
        return q_len * k_len
    return q_len * (k_len - q_len) + q_len * (q_len + 1) // 2


def _plain_scores(c):
    """Scores that the plain form holds at once."""
    if c["op"] != "prompt":
        return 0
    return c["batch"] * c["kv_heads"] * c["group"] * c["longest"] * (c["longest"] + c["context"])


def work(c):
    kv, hq, lens = c["kv_heads"], c["kv_heads"] * c["group"], _lengths(c)
    n, total = len(lens), sum(lens)
    row = D * 2
    if c["op"] == "append":
        # every row read once; queries, cached keys and values, and the dense keys written; a table row, a position
        # and a slot per token
        b = total * row * (2 * hq + 4 * kv + (kv if c["keep_k"] else 0))
        b += total * (c["rot_dim"] * 4 + 4 * (3 if c["mrope"] else 1) + 4)
        return {"bytes": b, "flops": total * (hq + kv) * c["rot_dim"] * 3}
    if c["op"] in ("decode", "step"):
        pages = sum(-(-t // c["page"]) for t in lens)
        b = 2 * total * kv * row + n * hq * (2 * row + 4) + 4 * pages + 4 * n
        if c["op"] == "step":
            b += n * (2 * kv * row + c["rot_dim"] * 4 + 4 * (3 if c["mrope"] else 1))
        return {"bytes": b, "flops": 4 * D * hq * total}
    keys = total + n * c["context"]
    scores = sum(_seen(t, t + c["context"], c["causal"]) for t in lens)
    return {"bytes": total * hq * (2 * row + 4) + 2 * keys * kv * row, "flops": 4 * D * hq * scores}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _keys(shape, heads_at, g, dev, dtype):
    """N(0, 1) with four outlier channels 8z + 3 per head (axis `heads_at`)."""
    heads = shape[heads_at]
    scale = torch.ones(heads, D, device=dev)
    off = torch.zeros(heads, D, device=dev)
    at = torch.rand(heads, D, generator=g, device=dev).argsort(1)[:, :4]
    scale.scatter_(1, at, 8.0)
    off.scatter_(1, at, 3.0)
    view = [1] * len(shape)
    view[heads_at], view[-1] = heads, D
    x = torch.randn(shape, generator=g, device=dev)
    return x.mul_(scale.view(view)).add_(off.view(view)).to(dtype)


def _table(length, rot_dim, dev):
    """Cosines and sines of every position: [length][rot_dim], the cosines of the rot_dim / 2 pairs first."""
    half = rot_dim // 2
    freq = 1e6 ** (-torch.arange(half, dtype=torch.float64, device=dev) / half)
    angle = torch.arange(length, dtype=torch.float64, device=dev)[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _positions(c, lens, g, dev):
    """Positions of the new tokens: one each, or three (time, height, width) as an image's patches have them."""
    if c["op"] == "step":
        first = torch.tensor([t - 1 for t in lens], dtype=torch.int32, device=dev)
    else:
        first = torch.cat([torch.arange(t, dtype=torch.int32, device=dev) for t in lens])
    if not c["mrope"]:
        return first
    patch = torch.randint(0, 36, (2, first.numel()), generator=g, device=dev, dtype=torch.int32)
    return torch.stack([first, first // 2 + patch[0], first // 3 + patch[1]])


def _sections(c):
    """Pairs that turn by each of the three positions, as Qwen2.5-VL divides its 64."""
    return (16, 24, 24) if c["mrope"] else (c["rot_dim"] // 2, 0, 0)


def prepare(case, seed):
    c, dev = case, _device()
    dtype = _TYPES[c["dtype"]]
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 7919 + 13)
    kv, hq, lens, ps = c["kv_heads"], c["kv_heads"] * c["group"], _lengths(c), c["page"]
    n, total = len(lens), sum(lens)
    s = {"case": c}
    if c["op"] == "prompt":
        keys = [t + c["context"] for t in lens]
        shape, at = ((sum(keys), kv, D), 1) if c["token_major"] else ((kv, sum(keys), D), 0)
        k = _keys(shape, at, g, dev, dtype)
        v = torch.randn(shape, generator=g, device=dev).to(dtype)
        s["q"] = torch.randn((total, hq, D), generator=g, device=dev).to(dtype)
        s["k"], s["v"] = (x if c["token_major"] else x.transpose(0, 1) for x in (k, v))
        s["q_begin"] = torch.tensor([0] + lens, dtype=torch.int32).cumsum(0, dtype=torch.int32)
        s["k_begin"] = torch.tensor([0] + keys, dtype=torch.int32).cumsum(0, dtype=torch.int32)
        s["q_begin_dev"], s["k_begin_dev"] = s["q_begin"].to(dev), s["k_begin"].to(dev)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((total, hq), device=dev)
        if own:
            import paper_2609_35800_gb300 as hg
            s["ws"] = torch.empty(hg.hg_prompt_workspace_size(), dtype=torch.uint8, device=dev)
            hg.hg_workspace_clear(s["ws"])
        return s

    # A paged cache: each request's pages, of a pool that holds some more, in no order.
    per = [-(-t // ps) for t in lens]
    pool = sum(per) + max(4, sum(per) // 16)
    order = torch.randperm(pool, generator=g, device=dev).to(torch.int32)
    table = torch.zeros(n, max(per), dtype=torch.int32, device=dev)
    row = torch.repeat_interleave(torch.arange(n, device=dev), torch.tensor(per, device=dev))
    begin = torch.tensor([0] + per, device=dev).cumsum(0)
    col = torch.arange(sum(per), device=dev) - begin[row]
    table[row, col] = order[:sum(per)]
    shape, at = ((pool, ps, kv, D), 2) if c["token_major"] else ((pool, kv, ps, D), 1)
    if c["op"] == "append":
        kp, vp = (torch.zeros(shape, dtype=dtype, device=dev) for _ in range(2))
    else:
        kp = _keys(shape, at, g, dev, dtype)
        vp = torch.randn(shape, generator=g, device=dev).to(dtype)
    # seen as [pages][heads][tokens][channels], whatever the order in memory
    s["k_pages"], s["v_pages"] = (x.transpose(1, 2) if c["token_major"] else x for x in (kp, vp))
    s["table"], s["lens"] = table, torch.tensor(lens, dtype=torch.int32, device=dev)
    if c["op"] in ("append", "step"):
        # a fused projection's output: queries, keys and values of a token side by side
        rows = total if c["op"] == "append" else n
        qkv = torch.empty((rows, hq + 2 * kv, D), dtype=dtype, device=dev)
        qkv[:, :hq] = torch.randn((rows, hq, D), generator=g, device=dev)
        qkv[:, hq:hq + kv] = _keys((rows, kv, D), 1, g, dev, dtype)
        qkv[:, hq + kv:] = torch.randn((rows, kv, D), generator=g, device=dev)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + kv], qkv[:, hq + kv:]
        s["positions"] = _positions(c, lens, g, dev)
        s["rotation"] = _table(max(lens) + 64, c["rot_dim"], dev)
    else:
        s["q"] = torch.randn((n, hq, D), generator=g, device=dev).to(dtype)
    if c["op"] == "append":
        seq = torch.repeat_interleave(torch.arange(n, device=dev), torch.tensor(lens, device=dev))
        first = torch.tensor([0] + lens, device=dev).cumsum(0)
        pos = torch.arange(total, device=dev) - first[seq]
        s["slots"] = (table[seq, pos // ps] * ps + pos % ps).to(torch.int32)
        s["q_out"] = torch.empty((total, hq, D), dtype=dtype, device=dev)
        s["k_out"] = torch.empty((total, kv, D), dtype=dtype, device=dev) if c["keep_k"] else None
    else:
        s["out"] = torch.empty((n, hq, D), dtype=dtype, device=dev)
        s["lse"] = torch.empty((n, hq), device=dev)
    if own:
        import paper_2609_35800_gb300 as hg
        s["pages"] = hg.hg_pages_create(s["k_pages"], s["v_pages"])
        if c["op"] in ("append", "step"):
            s["rot"] = hg.Rotation(s["rotation"], interleaved=c["interleaved"],
                                   sections=_sections(c) if c["mrope"] else None)
        if c["op"] in ("decode", "step"):
            s["ws"] = torch.empty(hg.hg_pages_decode_workspace_size(s["pages"], n, hq), dtype=torch.uint8, device=dev)
            hg.hg_workspace_clear(s["ws"])
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2609_35800_gb300 as hg
    c = s["case"]
    if c["op"] == "append":
        hg.hg_pages_append(s["pages"], s["q"], s["k"], s["v"], s["rot"], s["positions"], s["slots"], s["q_out"],
                           s["k_out"])
        return _appended(s, s["q_out"], s["k_out"])
    if c["op"] == "decode":
        hg.hg_pages_decode_attention(s["pages"], s["q"], s["table"], s["lens"], s["out"], s["lse"], 0.0, s["ws"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "step":
        hg.hg_pages_decode_step(s["pages"], s["q"], s["k"], s["v"], s["rot"], s["positions"], s["table"], s["lens"],
                                s["out"], s["lse"], 0.0, s["ws"])
        return {"out": s["out"], "lse": s["lse"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    hg.hg_prompt_attention(s["q"], s["k"], s["v"], s["q_begin"], s["k_begin"], s["out"], s["lse"], c["causal"], 0.0,
                           s["ws"])
    return {"out": s["out"], "lse": s["lse"]}


def _appended(s, q_out, k_out):
    out = {"q": q_out, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if k_out is not None:
        out["k"] = k_out
    return out


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
    dtype, kv, grp = _TYPES[c["dtype"]], c["kv_heads"], c["group"]
    if c["op"] == "append":
        cos, sin = _angles(s)
        q, k = (_rotated(s[x], cos, sin, c).to(dtype) for x in "qk")
        page, at = s["slots"].long() // c["page"], s["slots"].long() % c["page"]
        s["k_pages"][page, :, at] = k
        s["v_pages"][page, :, at] = s["v"]
        return _appended(s, q, k if c["keep_k"] else None)
    if c["op"] in ("decode", "step"):
        q, lens, table = s["q"], s["lens"], s["table"].long()
        n = q.shape[0]
        if c["op"] == "step":
            cos, sin = _angles(s)
            q, k = (_rotated(s[x], cos, sin, c).to(dtype) for x in "qk")
            last = lens.long() - 1
            page = table[torch.arange(n, device=last.device), last // c["page"]]
            s["k_pages"][page, :, last % c["page"]] = k
            s["v_pages"][page, :, last % c["page"]] = s["v"]
        k, v = (s[x][table].permute(0, 2, 1, 3, 4).reshape(n, kv, -1, D).float() for x in ("k_pages", "v_pages"))
        scores = torch.matmul(q.reshape(n, kv, grp, D).float(), k.transpose(2, 3)) * (D ** -0.5)
        seen = torch.arange(k.shape[2], device=lens.device) < lens[:, None]
        out, lse = _attend(scores, seen[:, None, None], v)
        got = {"out": out.reshape(n, kv * grp, D).to(dtype), "lse": lse.reshape(n, kv * grp)}
        return got if c["op"] == "decode" else {**got, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    # prompts: padded to the longest, and their rows taken out again
    qb, kb = s["q_begin_dev"].long(), s["k_begin_dev"].long()
    q_len, k_len = qb[1:] - qb[:-1], kb[1:] - kb[:-1]
    n, lq, lk = len(q_len), c["longest"], c["longest"] + c["context"]
    i, j = torch.arange(lq, device=qb.device), torch.arange(lk, device=qb.device)
    q = s["q"][(qb[:-1, None] + i).clamp_(max=s["q"].shape[0] - 1)].float()
    k, v = (s[x][(kb[:-1, None] + j).clamp_(max=s["k"].shape[0] - 1)].float() for x in "kv")
    q = q.view(n, lq, kv, grp, D).permute(0, 2, 3, 1, 4).reshape(n, kv, grp * lq, D)
    k, v = k.permute(0, 2, 1, 3), v.permute(0, 2, 1, 3)
    scores = (torch.matmul(q, k.transpose(2, 3)) * (D ** -0.5)).view(n, kv, grp, lq, lk)
    last = (i + (k_len - q_len)[:, None])[:, :, None] if c["causal"] else k_len[:, None, None] - 1
    seen = (j <= last) & (j < k_len[:, None, None])
    out, lse = _attend(scores, seen[:, None, None], v[:, :, None])
    token = torch.arange(s["q"].shape[0], device=qb.device)
    seq = torch.searchsorted(qb[1:], token, right=True)
    at = token - qb[seq]
    out = out[seq, :, :, at].reshape(-1, kv * grp, D)
    return {"out": out.to(dtype), "lse": lse[seq, :, :, at].reshape(-1, kv * grp)}


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


def _attend64(q, k, v, shown):
    """One request: q [rows][heads][128], k and v [keys][kv heads][128]; row i sees the first shown[i] keys."""
    rows, hq = q.shape[:2]
    grp = hq // k.shape[1]
    out = torch.zeros(rows, hq, D, dtype=torch.float64, device=q.device)
    lse = torch.full((rows, hq), -math.inf, dtype=torch.float64, device=q.device)
    key = torch.arange(k.shape[0], device=q.device)
    block = max(1, int(2e8 // max(1, k.shape[0])))
    for h in range(hq):
        kh, vh = k[:, h // grp].double(), v[:, h // grp].double()
        for r in range(0, rows, block):
            sc = q[r:r + block, h].double() @ kh.t() / math.sqrt(D)
            sc[key >= shown[r:r + block, None]] = -math.inf
            lse[r:r + block, h] = torch.logsumexp(sc, 1)
            out[r:r + block, h] = torch.softmax(sc, 1) @ vh
    empty = shown <= 0
    out[empty] = 0.0
    return out, lse


def exact(case, seed):
    c = case
    lens = _lengths(c)
    if c["op"] == "prompt" and 4 * D * c["kv_heads"] * c["group"] * sum(t * (t + c["context"]) for t in lens) > 8e12:
        return None  # matrix products in 64 bits take too long
    s = prepare(case, seed)
    dtype, dev = _TYPES[c["dtype"]], s["q"].device
    if c["op"] == "prompt":
        outs = []
        for b, t in enumerate(lens):
            q0, k0, k1 = int(s["q_begin"][b]), int(s["k_begin"][b]), int(s["k_begin"][b + 1])
            n = k1 - k0
            shown = torch.arange(t, device=dev) + (n - t + 1) if c["causal"] else torch.full((t,), n, device=dev)
            outs.append(_attend64(s["q"][q0:q0 + t], s["k"][k0:k1], s["v"][k0:k1], shown))
        return {"out": torch.cat([o for o, _ in outs]), "lse": torch.cat([l for _, l in outs])}
    got = {}
    q = s["q"]
    if c["op"] in ("append", "step"):
        q, k = _turn64(s["q"], s), _turn64(s["k"], s)
        kp, vp = s["k_pages"].double(), s["v_pages"].double()
        if c["op"] == "append":
            where = s["slots"].long()
        else:
            last = [t - 1 for t in lens]
            where = torch.stack([s["table"][b, t // c["page"]].long() * c["page"] + t % c["page"]
                                 for b, t in enumerate(last)])
        kp[where // c["page"], :, where % c["page"]] = k
        vp[where // c["page"], :, where % c["page"]] = s["v"].double()
        got = {"k_pages": kp, "v_pages": vp}
        if c["op"] == "append":
            return {**got, "q": q, **({"k": k} if c["keep_k"] else {})}
        # attention is defined on the rotated rows as they are held: rounded to the cache's type
        q, s["k_pages"], s["v_pages"] = q.to(dtype), kp.to(dtype), vp.to(dtype)
    outs = []
    for b, t in enumerate(lens):
        ids = s["table"][b, :-(-t // c["page"])].long()
        k, v = (s[x][ids].transpose(1, 2).reshape(-1, c["kv_heads"], D)[:t] for x in ("k_pages", "v_pages"))
        outs.append(_attend64(q[b:b + 1], k, v, torch.tensor([t], device=dev)))
    return {**got, "out": torch.cat([o for o, _ in outs]), "lse": torch.cat([l for _, l in outs])}
