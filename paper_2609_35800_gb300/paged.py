"""A serving program's 16-bit requests, put together: prompts packed into one call, their keys rotated and stored in
pages, then tokens one step at a time.  Allocation and marshalling only -- every step runs in the library."""
import torch

from . import (Pages, hg_pages_append, hg_pages_create, hg_pages_decode_step, hg_pages_decode_workspace_size,
               hg_prompt_attention, hg_prompt_workspace_size, hg_workspace_clear)

__all__ = ["PagedRunner", "Pages"]


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
