"""A plan's tables, slots and positions over a 16-bit pool: prompts and single tokens stored by hg_pages_append at the slots, read
by the paged decode through the table, of requests that come, grow and end."""
import pytest
import torch

import paper_2609_35800_gb300 as hg
from attention16 import attend, check, check_turned, table, turned

pytestmark = pytest.mark.gpu
D, HEADS, HQ = 128, 2, 6
BF16 = torch.bfloat16


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("size", [16, 64])
def test_16_bit_pages_take_a_plans_slots(size):
    g = torch.Generator(device="cuda")
    g.manual_seed(size)
    n, pool, room = 4, 40, 300
    k_pages, v_pages = (torch.full((pool, HEADS, size, D), float("nan"), dtype=BF16, device="cuda") for _ in "kv")
    pages = hg.hg_pages_create(k_pages, v_pages)
    cs = table(400, D, "cuda")
    rot = hg.Rotation(cs)
    tab = torch.zeros((n, 24), dtype=torch.int32, device="cuda")
    lens, begin, counts = _ints([0] * n), _ints([0] * (n + 1)), _ints([pool, 0, 0, 0])
    free = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    ws = torch.empty(hg.hg_pages_decode_workspace_size(pages, n, HQ), dtype=torch.uint8, device="cuda")
    hg.hg_workspace_clear(ws)
    held = [[torch.zeros((0, HEADS, D), dtype=BF16, device="cuda")] * 2 for _ in range(n)]
    for new in ([40, 0, 17, 100], [1, 1, 1, 1], [1, -1, 1, 30], [0, 63, -1, 1], [1, 1, 90, 1]):
        slots, positions = (torch.full((room,), 77, dtype=torch.int32, device="cuda") for _ in range(2))
        hg.hg_pages_plan(tab, lens, _ints(new), free, counts[:1], size, lens, begin, slots, positions, counts)
        assert int(counts[hg.HG_PLAN_REFUSED]) == 0
        # rows for all there is room for: those behind the last token have no slot
        q, k, v = (torch.randn((room, h, D), generator=g, device="cuda").to(BF16) for h in (HQ, HEADS, HEADS))
        q_rot, k_rot = torch.empty_like(q), torch.empty_like(k)
        hg.hg_pages_append(pages, q, k, v, rot, positions, slots, q_rot, k_rot)
        at = 0
        for r, m in enumerate(new):
            rows = slice(at, at + max(m, 0))
            at += max(m, 0)
            if m < 0:
                held[r] = [x[:0] for x in held[r]]
            had = len(held[r][0])
            pos = torch.arange(had, had + max(m, 0), device="cuda")
            if m > 0:
                check_turned(k_rot[rows], k[rows], turned(k[rows], cs, pos, D, False, None), BF16)
            held[r] = [torch.cat([a, b]) for a, b in zip(held[r], (k_rot[rows], v[rows]))]
        lengths = [len(x[0]) for x in held]
        assert lens.tolist() == lengths and int(counts[hg.HG_PLAN_TOKENS]) == at
        for r, m in enumerate(lengths):
            ids = tab[r, :-(-m // size)].long()
            for x, got in zip(held[r], (k_pages, v_pages)):
                assert torch.equal(got[ids].transpose(1, 2).reshape(-1, HEADS, D)[:m], x)
        probe = torch.randn((n, HQ, D), generator=g, device="cuda").to(BF16)
        out, lse = torch.empty_like(probe), torch.empty((n, HQ), device="cuda")
        hg.hg_pages_decode_attention(pages, probe, tab, lens, out, lse, 0.0, ws)
        for r, m in enumerate(lengths):
            keys, values = held[r]
            ref = attend(probe[r:r + 1], keys, values, torch.tensor([m], device="cuda"), D ** -0.5)
            check(out[r:r + 1], lse[r:r + 1], ref, BF16, m, float(values.abs().max()) if m else 0.0)
    assert hg.hg_workspace_status(ws) == 0
