"""Paged8Runner: prompts, their further pieces, steps and ends put together, against what the 8-bit cache has to hold; calls
that it refuses leave the requests as they were."""
import pytest
import torch

import pages8 as ref8
import paper_2609_35800_gb300 as hg
from attention16 import ROUNDOFF, attend, table, turned
from paper_2609_35800_gb300.paged import Paged8Runner
from pages8 import BLOCK

pytestmark = pytest.mark.gpu
D, HEADS, GROUP = 128, 2, 3
HQ = HEADS * GROUP
BF16 = torch.bfloat16


class Requests:
    """A runner beside its requests' rotated keys and values.  Poisoned pages: what nobody stored shows."""

    def __init__(self, seed, num_pages, size=16, **kw):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.turns = table(500, D, "cuda")
        self.run = Paged8Runner(num_pages, size, HQ, HEADS, hg.Rotation(self.turns), **kw)
        for x in (self.run.k_pages, self.run.v_pages):
            x.view(torch.uint8).fill_(0x7f)
        for x in (self.run.k_scales, self.run.v_scales):
            x.fill_(float("nan"))
        self.num_pages, self.rows = num_pages, []  # (keys, values) of every request

    def draw(self, n):
        x = torch.randn((n, HQ + 2 * HEADS, D), generator=self.g, device="cuda").to(BF16)
        return x[:, :HQ], x[:, HQ:HQ + HEADS], x[:, HQ + HEADS:]

    def held(self, i):
        """Request i's keys and values as the cache holds them, 64 bits."""
        run, n = self.run, len(self.rows[i][0])
        ids = run.table[i, :-(-n // run.page_size)].long()
        out = []
        for codes, scales in ((run.k_pages, run.k_scales), (run.v_pages, run.v_scales)):
            x = ref8.values(codes.view(torch.uint8)[ids], scales[ids])
            out.append(x.transpose(1, 2).reshape(-1, HEADS, D)[:n])
        return out

    def stored(self):
        """The cache holds every row to e4m3's precision: half a step of its last store, and of those before it, each at
        most half as coarse in the block's range."""
        run = self.run
        for i, (k, v) in enumerate(self.rows):
            for got, want, scales in zip(self.held(i), (k, v), (run.k_scales, run.v_scales)):
                n = len(want)
                t = torch.arange(n, device="cuda")
                s = scales[run.table[i, t // run.page_size].long(), :, t % run.page_size // BLOCK].double()
                assert bool(((got - want.double()).abs() <= 2.0 ** -3 * want.double().abs() + 2.0 ** -9 * s[..., None]).all())

    def prompt_close(self, got, q, k, v, seen):
        out, _, mean, big = attend(q, k, v, seen, D ** -0.5)
        # the prompt kernel's probabilities are BF16; a rotated entry may round to either neighbour
        delta = (2.0 ** -17 + 2.0 ** -8) * big[..., None]
        tol = ROUNDOFF[BF16] * out.abs() + (ROUNDOFF[BF16] + 2 * delta) * mean * 1.01 + 2.0 ** -20
        assert bool(((got.double() - out).abs() <= tol).all())

    def feed(self, lens, first):
        """lens[j] rows come to request first + j: as new prompts where there is none."""
        fresh = first == len(self.rows)
        q, k, v = self.draw(sum(lens))
        had = [0] * len(lens) if fresh else [len(r[0]) for r in self.rows]
        pos = torch.cat([torch.arange(0)] + [torch.arange(a, a + n) for a, n in zip(had, lens)]).to(torch.int32).cuda()
        out = self.run.admit(q, k, v, lens) if fresh else self.run.extend(q, k, v, lens)
        q, k = (turned(x, self.turns, pos, D, False, None).to(BF16) for x in (q, k))
        at = 0
        for j, n in enumerate(lens):
            rows = k[at:at + n], v[at:at + n]
            if fresh:
                self.rows.append(rows)
            else:
                self.rows[j] = tuple(torch.cat([a, b]) for a, b in zip(self.rows[j], rows))
            if n:
                total = len(self.rows[first + j][0])
                keys, values = rows if all(h == 0 for h, m in zip(had, lens) if m) else [x.to(BF16) for x in self.held(first + j)]
                seen = torch.arange(total - n + 1, total + 1, device="cuda")
                self.prompt_close(out[at:at + n], q[at:at + n], keys, values, seen)
            at += n
        self.stored()

    def step(self):
        n = len(self.rows)
        q, k, v = self.draw(n)
        pos = torch.tensor([len(r[0]) for r in self.rows], dtype=torch.int32, device="cuda")
        out = self.run.step(q, k, v)
        q, k = (turned(x, self.turns, pos, D, False, None).to(BF16) for x in (q, k))
        for i in range(n):
            self.rows[i] = torch.cat([self.rows[i][0], k[i:i + 1]]), torch.cat([self.rows[i][1], v[i:i + 1]])
            keys, values = self.held(i)
            t = len(keys)
            ref = attend(q[i:i + 1], keys, values, torch.tensor([t], device="cuda"), D ** -0.5)
            ref = ref[:3] + (ref[3] * (1 + 2.0 ** 17 * 2.0 ** -8),)  # a rotated query may round to either neighbour
            ref8.check(out[i:i + 1], None, ref, BF16, t, float(self.run.v_scales[self.run.table[i, :-(-t // self.run.page_size)].long()]
                                                             .nan_to_num(0.0).max()))
        self.stored()

    def end(self, gone):
        self.run.end(gone)
        self.rows = [r for i, r in enumerate(self.rows) if i not in gone]
        self.consistent()

    def consistent(self):
        run, size = self.run, self.run.page_size
        lens = [len(r[0]) for r in self.rows]
        assert run.lengths == lens == run.lens[:len(lens)].tolist()
        assert not bool(run.lens[len(lens):].any())
        held = [p for i, n in enumerate(lens) for p in run.table[i, :-(-n // size)].tolist()]
        left = int(run.counts[0])
        assert left == run.free_pages and sorted(held + run.free[:left].tolist()) == list(range(self.num_pages))

    def state(self):
        run, lens = self.run, self.run.lengths
        table = [run.table[i, :-(-n // run.page_size)].tolist() for i, n in enumerate(lens)]
        left = int(run.counts[0])
        pages = [x.view(torch.uint8)[[p for r in table for p in r]].clone() for x in (run.k_pages, run.v_pages)]
        return (list(lens), run.lens.tolist(), table, run.free_pages, run.free[:left].tolist()), pages


def _unchanged(r, before):
    now = r.state()
    assert now[0] == before[0]
    assert all(torch.equal(a, b) for a, b in zip(now[1], before[1]))


@pytest.mark.parametrize("size", [16, 64])
def test_requests_come_and_go(size):
    r = Requests(1, 60 if size == 16 else 24, size)
    r.feed([40, 7, 16], 0)
    for _ in range(3):
        r.step()
    r.feed([21, 0, 64], 0)  # further pieces of the first and the third
    r.step()
    r.end([1])
    r.feed([33, 0, 1], 2)
    for _ in range(17):
        r.step()
    r.consistent()
    r.end([0, 3])
    r.feed([5, 5, 5], 0)
    r.step()
    r.run.release()
    r.rows = []
    r.consistent()
    r.feed([100], 0)
    r.step()
    r.consistent()


def test_refused_calls_change_nothing():
    r = Requests(2, 12, max_batch=3, max_tokens=100)
    r.feed([40, 5], 0)
    r.step()
    before = r.state()
    for lens in ([113], [10, 10], [-1]):  # past the table, past the batch
        with pytest.raises((RuntimeError, ValueError)):
            r.run.admit(*r.draw(max(0, sum(lens))), lens)
        _unchanged(r, before)
    for lens in ([80, 0], [60, 80], [1], [1, -1]):  # past the table, without pages (8 are left)
        with pytest.raises((RuntimeError, ValueError)):
            r.run.extend(*r.draw(max(0, sum(lens))), lens)
        _unchanged(r, before)
    q, k, v = r.draw(10)
    for args in ((q, k, v, [4, 5]), (q[:-1], k, v, [5, 5]), (q, k, v.half(), [5, 5]), (q, k.cpu(), v, [5, 5]),
                 (q, k, v, [5, 5], torch.zeros(9, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            r.run.extend(*args)
        _unchanged(r, before)
    q, k, v = r.draw(2)
    for args in ((q[:1], k, v), (q, k[:1], v), (q, k, v.half()), (q.cpu(), k, v), (q, k, v, torch.zeros(1, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            r.run.step(*args)
        _unchanged(r, before)
    with pytest.raises(ValueError):
        r.run.end([2])
    r.run.end([])
    _unchanged(r, before)
    r.consistent()
    for _ in range(20):
        r.step()
    r.feed([10, 10], 0)
    r.consistent()


def test_a_step_without_pages_changes_nothing():
    r = Requests(3, 5)  # the requests take all five
    r.feed([20, 16, 30], 0)
    before = r.state()
    with pytest.raises(RuntimeError):
        r.run.step(*r.draw(3))
    _unchanged(r, before)
    r.end([1])
    r.step()
    r.consistent()


def test_no_prompt_and_empty_prompts():
    r = Requests(4, 8)
    r.feed([], 0)
    r.feed([0, 17, 0], 0)
    for _ in range(2):
        r.step()
    r.feed([0, 0, 0], 0)
    assert r.run.lengths == [2, 19, 2]
    r.consistent()
