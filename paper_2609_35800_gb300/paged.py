"""A serving program's requests in pages of 16 or 8 bits, put together: prompts packed into one call, their keys rotated and
stored in pages, then tokens one step at a time.  Allocation and marshalling only -- every step runs in the library."""
import torch

from . import (HG_PAGES8_BLOCK, Pages, Pages8, hg_pages8_append, hg_pages8_create, hg_pages8_decode_step,
               hg_pages8_decode_workspace_size, hg_pages8_dequantize, hg_pages_append, hg_pages_create, hg_pages_decode_step,
               hg_pages_decode_workspace_size, hg_pages_plan, hg_prompt_attention, hg_prompt_workspace_size,
               hg_workspace_clear)

__all__ = ["PagedRunner", "Paged8Runner", "Pages", "Pages8"]


class PagedRunner:
    """Requests of one attention layer that share a page pool: `admit` prompts, `step` them, `release` them."""

    def __init__(self, num_pages, page_size, q_heads, kv_heads, rotation=None, dtype=torch.bfloat16, device="cuda",
                 max_batch=64, max_tokens=32768):
        self.page_size, self.q_heads, self.kv_heads = page_size, q_heads, kv_heads
        self.rotation, self.dtype, self.device = rotation, dtype, device
        self.k_pages = torch.empty(num_pages, kv_heads, page_size, 128, dtype=dtype, device=device)
        self.v_pages = torch.empty_like(self.k_pages)
        self.pages = hg_pages_create(self.k_pages, self.v_pages)
        self.free = list(range(num_pages - 1, -1, -1))
        self.owned, self.lengths = [], []  # pages and tokens of each request, on the host
        self.per_request = -(-max_tokens // page_size)
        self.table = torch.zeros(max_batch, self.per_request, dtype=torch.int32, device=device)
        self.lens = torch.zeros(max_batch, dtype=torch.int32, device=device)
        # one each: a workspace's counters lie where the other kind of call keeps its parts
        self.ws, self.prompt_ws = (torch.empty(n, dtype=torch.uint8, device=device) for n in (
            hg_pages_decode_workspace_size(self.pages, max_batch, q_heads), hg_prompt_workspace_size()))
        hg_workspace_clear(self.ws)
        hg_workspace_clear(self.prompt_ws)

    def _pages_for(self, owned, tokens):
        """The free pages that requests which own these would get next, up to these tokens each; nothing is changed."""
        need = [-(-n // self.page_size) - len(have) for n, have in zip(tokens, owned)]
        if any(n + len(have) > self.per_request for n, have in zip(need, owned)):
            raise RuntimeError("PagedRunner: a request of %d tokens, the table holds %d" % (
                max(tokens), self.per_request * self.page_size))
        if sum(need) > len(self.free):
            raise RuntimeError("PagedRunner: %d pages wanted, %d left" % (sum(need), len(self.free)))
        ids = iter(reversed(self.free))
        return [[next(ids) for _ in range(n)] for n in need]

    def _take(self, pages):
        """The pages of _pages_for are no longer free."""
        count = sum(len(ids) for ids in pages)
        del self.free[len(self.free) - count:]

    def admit(self, q, k, v, prompt_lengths, positions, k_out=None, v_out=None):
        """Prompts one after the other, q / k / v [tokens][heads][128] not yet rotated: their attention
        [tokens][q_heads][128].  k_out / v_out: where the rotated keys and the values go as dense tensors as well (a
        request that goes on in the packed cache takes hg_quantize_kv's layout from there).  Prompts that are refused (no
        page or place left, arguments that do not fit) are not admitted, none of the call's, and the others stay."""
        lens, first = list(prompt_lengths), len(self.owned)
        if first + len(lens) > self.table.shape[0]:
            raise RuntimeError("PagedRunner: more requests than the batch holds")
        if any(n < 0 for n in lens) or any(x.shape[0] != sum(lens) for x in (q, k, v)):
            raise ValueError("PagedRunner.admit: q, k and v hold %d, %d and %d rows, the prompts %d"
                             % (q.shape[0], k.shape[0], v.shape[0], sum(lens)))
        pages = self._pages_for([[]] * len(lens), lens)
        slots = [torch.empty(0, dtype=torch.int32)]
        for i, (n, ids) in enumerate(zip(lens, pages)):
            at, ids = torch.arange(n, dtype=torch.int32), torch.tensor(ids, dtype=torch.int32)
            slots.append(ids[at // self.page_size] * self.page_size + at % self.page_size)
            self.table[first + i, :len(ids)] = ids
        slots = torch.cat(slots).to(self.device)
        q_rot = torch.empty(q.shape, dtype=self.dtype, device=self.device)
        if k_out is None:
            k_out = torch.empty(k.shape, dtype=self.dtype, device=self.device)
        hg_pages_append(self.pages, q, k, v, self.rotation, positions, slots, q_rot, k_out, v_out)
        begin = torch.tensor([0] + lens).cumsum(0).to(torch.int32)
        out = torch.empty_like(q_rot)
        hg_prompt_attention(q_rot, k_out, v, begin, begin, out, None, True, 0.0, self.prompt_ws)
        self.lens[first:first + len(lens)] = torch.tensor(lens, dtype=torch.int32)
        self.owned += pages
        self.lengths += lens
        self._take(pages)
        return out

    def step(self, q, k, v, positions):
        """One new token of every request: q [requests][q_heads][128], k, v [requests][kv_heads][128].  A step that is
        refused (no page left, arguments that do not fit) leaves the requests as they were."""
        n = len(self.owned)
        if q.shape[0] != n:
            raise ValueError("PagedRunner.step: q holds %d rows, there are %d requests" % (q.shape[0], n))
        grown = [tokens + 1 for tokens in self.lengths]
        pages = self._pages_for(self.owned, grown)
        for i, ids in enumerate(pages):
            if ids:  # (past a request's length the table is not read)
                at = len(self.owned[i])
                self.table[i, at:at + len(ids)] = torch.tensor(ids, dtype=torch.int32)
        out = torch.empty(n, self.q_heads, 128, dtype=self.dtype, device=self.device)
        self.lens[:n] += 1
        try:
            hg_pages_decode_step(self.pages, q, k, v, self.rotation, positions, self.table[:n], self.lens, out, None, 0.0,
                                 self.ws)
        except BaseException:
            self.lens[:n] -= 1
            raise
        self.lengths = grown
        for owned, ids in zip(self.owned, pages):
            owned += ids
        self._take(pages)
        return out

    def release(self):
        """Every request ends; its pages are free again."""
        for pages in self.owned:
            self.free.extend(reversed(pages))
        self.owned, self.lengths = [], []
        self.lens.zero_()


class Paged8Runner:
    """Requests of one attention layer that share a pool of 8-bit pages, whose page tables are built on the GPU: `admit`
    prompts, `extend` them by further pieces, `step` them, `end` some of them.  What a call plans becomes the runner's state
    once the whole call is under way: one that is refused leaves the requests as they were."""

    def __init__(self, num_pages, page_size, q_heads, kv_heads, rotation=None, dtype=torch.bfloat16, device="cuda",
                 max_batch=64, max_tokens=32768):
        self.page_size, self.q_heads, self.kv_heads = page_size, q_heads, kv_heads
        self.rotation, self.dtype, self.device = rotation, dtype, device
        self.k_pages = torch.empty(num_pages, kv_heads, page_size, 128, dtype=torch.float8_e4m3fn, device=device)
        self.v_pages = torch.empty_like(self.k_pages)
        self.k_scales = torch.empty(num_pages, kv_heads, page_size // HG_PAGES8_BLOCK, device=device)
        self.v_scales = torch.empty_like(self.k_scales)
        self.pages = hg_pages8_create(self.k_pages, self.v_pages, self.k_scales, self.v_scales, dtype)
        self.per_request = -(-max_tokens // page_size)
        self.lengths, self.free_pages = [], num_pages  # the host's own count of what the GPU holds
        self.table = torch.zeros(max_batch, self.per_request, dtype=torch.int32, device=device)
        self.lens = torch.zeros(max_batch, dtype=torch.int32, device=device)
        self.free = torch.arange(num_pages - 1, -1, -1, dtype=torch.int32, device=device)
        self.counts = torch.tensor([num_pages, 0, 0, 0], dtype=torch.int32, device=device)
        self.ones = torch.ones(max_batch, dtype=torch.int32, device=device)
        # one each: a workspace's counters lie where the other kind of call keeps its parts
        self.ws, self.prompt_ws = (torch.empty(n, dtype=torch.uint8, device=device) for n in (
            hg_pages8_decode_workspace_size(self.pages, max_batch, q_heads), hg_prompt_workspace_size()))
        hg_workspace_clear(self.ws)
        hg_workspace_clear(self.prompt_ws)

    def _held(self, tokens):
        return sum(-(-n // self.page_size) for n in tokens)

    def _check(self, grown):
        """Pages that requests of these lengths take beyond those of the present ones; raises where there are too few."""
        if max(grown, default=0) > self.per_request * self.page_size:
            raise RuntimeError("Paged8Runner: a request of %d tokens, the table holds %d"
                               % (max(grown), self.per_request * self.page_size))
        need = self._held(grown) - self._held(self.lengths)
        if need > self.free_pages:
            raise RuntimeError("Paged8Runner: %d pages wanted, %d left" % (need, self.free_pages))
        return need

    def _plan(self, new, rooms):
        """Plans the first len(new) rows of the table: lengths, begin, positions and counts afterwards."""
        n = new.numel()
        lens, counts = torch.empty_like(self.lens[:n]), torch.empty_like(self.counts)
        begin = torch.empty(n + 1, dtype=torch.int32, device=self.device)
        slots, positions = (torch.empty(rooms, dtype=torch.int32, device=self.device) for _ in range(2))
        hg_pages_plan(self.table[:n], self.lens[:n], new, self.free, self.counts[:1], self.page_size, lens, begin, slots,
                      positions, counts)
        return lens, begin, positions, counts

    def _keep(self, lens, counts, grown, need):
        self.lens[:lens.numel()] = lens
        self.counts, self.lengths, self.free_pages = counts, grown, self.free_pages - need

    def _feed(self, q, k, v, new, grown, positions, k_out, v_out):
        """new[r] tokens come to request r, which then has grown[r]: their attention."""
        total = sum(new)
        if any(x.shape[0] != total for x in (q, k, v)):
            raise ValueError("Paged8Runner: q, k and v hold %d, %d and %d rows, the prompts %d"
                             % (q.shape[0], k.shape[0], v.shape[0], total))
        if q.shape[1:] != (self.q_heads, 128):
            raise ValueError("Paged8Runner: q is %s, the requests have %d query heads" % (list(q.shape), self.q_heads))
        need = self._check(grown)
        # everything that may fail comes before the store: a block that it stores again more coarsely stays so
        q_rot, out = (torch.empty(q.shape, dtype=self.dtype, device=self.device) for _ in range(2))
        if k_out is None:
            k_out = torch.empty(k.shape, dtype=self.dtype, device=self.device)
        if v_out is None:
            v_out = torch.empty(v.shape, dtype=self.dtype, device=self.device)
        q_begin = torch.tensor([0] + new).cumsum(0).to(torch.int32)
        cached = any(n and n != m for n, m in zip(new, grown))
        keys, values, k_begin = k_out, v_out, q_begin
        if cached:  # tokens that are there already: all of a request's from the cache
            rows = [m if n else 0 for n, m in zip(new, grown)]
            k_begin = torch.tensor([0] + rows).cumsum(0).to(torch.int32)
            begins = k_begin.to(self.device)
            keys, values = (torch.empty(self.kv_heads, sum(rows), 128, dtype=self.dtype, device=self.device).transpose(0, 1)
                            for _ in range(2))
        fed = torch.tensor(new, dtype=torch.int32, device=self.device)
        lens, begin, places, counts = self._plan(fed, total)
        hg_pages8_append(self.pages, q, k, v, self.rotation, places if positions is None else positions, begin, self.table,
                         lens, q_rot, k_out, v_out)
        if cached:
            hg_pages8_dequantize(self.pages, begins, self.table, keys, values)
        hg_prompt_attention(q_rot, keys, values, q_begin, k_begin, out, None, True, 0.0, self.prompt_ws)
        self._keep(lens, counts, grown, need)
        return out

    def admit(self, q, k, v, prompt_lengths, positions=None, k_out=None, v_out=None):
        """Prompts one after the other, q / k / v [tokens][heads][128] not yet rotated: their attention
        [tokens][q_heads][128], over the rows as they come.  positions None: each token's number in its request.  k_out /
        v_out: where the rotated keys and the values go as dense 16-bit tensors as well.  Prompts that are refused (no page
        or place left, arguments that do not fit) are not admitted, none of the call's, and the others stay."""
        lens = list(prompt_lengths)
        if any(n < 0 for n in lens):
            raise ValueError("Paged8Runner.admit: a prompt of %d tokens" % min(lens))
        if len(self.lengths) + len(lens) > self.table.shape[0]:
            raise RuntimeError("Paged8Runner: more requests than the batch holds")
        # (a new request's row of lens is 0)
        return self._feed(q, k, v, [0] * len(self.lengths) + lens, self.lengths + lens, positions, k_out, v_out)

    def extend(self, q, k, v, new_lengths, positions=None):
        """The next new_lengths[r] tokens of request r's prompt (0: none), which attend to the request's cached tokens, and
        to themselves, as the 8-bit cache holds them."""
        new = list(new_lengths)
        if len(new) != len(self.lengths) or any(n < 0 for n in new):
            raise ValueError("Paged8Runner.extend: %d lengths, there are %d requests" % (len(new), len(self.lengths)))
        return self._feed(q, k, v, new, [a + b for a, b in zip(self.lengths, new)], positions, None, None)

    def step(self, q, k, v, positions=None):
        """One new token of every request: q [requests][q_heads][128], k, v [requests][kv_heads][128].  positions None:
        each token's number in its request.  A step that is refused leaves the requests as they were."""
        n = len(self.lengths)
        if q.shape[0] != n:
            raise ValueError("Paged8Runner.step: q holds %d rows, there are %d requests" % (q.shape[0], n))
        grown = [tokens + 1 for tokens in self.lengths]
        need = self._check(grown)
        lens, _, places, counts = self._plan(self.ones[:n], n)
        out = torch.empty(n, self.q_heads, 128, dtype=self.dtype, device=self.device)
        hg_pages8_decode_step(self.pages, q, k, v, self.rotation, places if positions is None else positions, self.table[:n],
                              lens, out, None, 0.0, self.ws)
        self._keep(lens, counts, grown, need)
        return out

    def end(self, requests):
        """These requests end (by their numbers) and give their pages back; the others move up in their order."""
        n, gone = len(self.lengths), set(requests)
        if any(r < 0 or r >= n for r in gone):
            raise ValueError("Paged8Runner.end: requests %s, there are %d" % (sorted(gone), n))
        if not gone:
            return
        stay = [r for r in range(n) if r not in gone]
        new = torch.tensor([-1 if r in gone else 0 for r in range(n)], dtype=torch.int32, device=self.device)
        lens, _, _, counts = self._plan(new, 0)
        rows = torch.tensor(stay, dtype=torch.int64, device=self.device)
        self.table[:len(stay)] = self.table[rows]
        self.lens.zero_()
        self.lens[:len(stay)] = lens[rows]
        given = self._held(self.lengths[r] for r in gone)
        self.counts, self.lengths, self.free_pages = counts, [self.lengths[r] for r in stay], self.free_pages + given

    def release(self):
        """Every request ends; its pages are free again."""
        self.end(range(len(self.lengths)))
