"""PagedRunner after calls that it refused: the requests go on as if the call had not been made."""
import pytest
import torch

import paper_2609_35800_gb300 as hg
from attention16 import attend, check, table, turned
from paper_2609_35800_gb300.paged import PagedRunner

pytestmark = pytest.mark.gpu
D, HEADS, GROUP = 128, 2, 3
HQ = HEADS * GROUP
BF16 = torch.bfloat16


class Requests:
    """A runner beside what its requests' caches have to hold.  Poisoned pages: what nobody stored shows."""

    def __init__(self, seed, num_pages, **kw):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.table = table(400, D, "cuda")
        self.run = PagedRunner(num_pages, 16, HQ, HEADS, hg.Rotation(self.table), **kw)
        self.run.k_pages.fill_(float("nan"))
        self.run.v_pages.fill_(float("nan"))
        self.keys, self.vals = [], []

    def rows(self, n):
        x = torch.randn((n, HQ + 2 * HEADS, D), generator=self.g, device="cuda").to(BF16)
        return x[:, :HQ], x[:, HQ:HQ + HEADS], x[:, HQ + HEADS:]

    def rotated(self, x, pos):
        return turned(x, self.table, pos, D, False, None).to(BF16)

    def compare(self, got, q, i, seen):
        ref = attend(q, self.keys[i], self.vals[i], seen, D ** -0.5)
        # a rotated entry may round to either neighbour: one unit more in every score
        ref = ref[:3] + (ref[3] + 2.0 ** 17 * 2.0 ** -8 * ref[3],)
        check(got, None, ref, BF16, len(self.keys[i]), 6.0)

    def admit(self, lens):
        q, k, v = self.rows(sum(lens))
        pos = torch.cat([torch.arange(0)] + [torch.arange(n) for n in lens]).to(torch.int32).cuda()
        out = self.run.admit(q, k, v, lens, pos)
        q, k = self.rotated(q, pos), self.rotated(k, pos)
        at = 0
        for n in lens:
            self.keys.append(k[at:at + n])
            self.vals.append(v[at:at + n])
            self.compare(out[at:at + n], q[at:at + n], len(self.keys) - 1, torch.arange(1, n + 1, device="cuda"))
            at += n

    def step(self):
        q, k, v = self.rows(len(self.keys))
        pos = torch.tensor([len(x) for x in self.keys], dtype=torch.int32, device="cuda")
        out = self.run.step(q, k, v, pos)
        q, k = self.rotated(q, pos), self.rotated(k, pos)
        for i in range(len(self.keys)):
            self.keys[i] = torch.cat([self.keys[i], k[i:i + 1]])
            self.vals[i] = torch.cat([self.vals[i], v[i:i + 1]])
            self.compare(out[i:i + 1], q[i:i + 1], i, torch.tensor([len(self.keys[i])], device="cuda"))

    def state(self):
        run = self.run
        return (list(run.free), [list(x) for x in run.owned], list(run.lengths), run.lens.tolist(),
                [run.table[i, :len(x)].tolist() for i, x in enumerate(run.owned)])


def refused_steps(r):
    """Steps whose arguments do not fit, each a call."""
    n = len(r.keys)
    q, k, v = r.rows(n)
    wide = r.rows(n + 1)
    pos = torch.tensor([len(x) for x in r.keys], dtype=torch.int32, device="cuda")
    return [(wide[0], k, v, pos), (q, wide[1], v, pos), (q[:-1], k[:-1], v[:-1], pos[:-1]), (q, k, v.half(), pos),
            (q, k, v, pos[:-1]), (q, k, v, pos.long()), (q, k, v, pos.cpu()), (q.cpu(), k, v, pos)]


@pytest.mark.parametrize("lens", [[40, 7, 16], [15, 32]])  # (16 and 32: the step takes a page)
def test_a_refused_step_changes_nothing(lens):
    r = Requests(1, 20)
    r.admit(lens)
    r.step()
    before = r.state()
    for args in refused_steps(r):
        with pytest.raises(ValueError):
            r.run.step(*args)
        assert r.state() == before
    for _ in range(18):
        r.step()
    assert r.run.lens[:len(lens)].tolist() == r.run.lengths == [n + 19 for n in lens]


def test_a_step_without_pages_changes_nothing():
    r = Requests(2, 5)  # the requests take all five
    r.admit([20, 16, 30])
    before = r.state()
    for _ in range(3):
        with pytest.raises(RuntimeError):
            r.run.step(*r.rows(3), torch.tensor([20, 16, 30], dtype=torch.int32, device="cuda"))
        assert r.state() == before
    r.run.release()
    assert sorted(r.run.free) == list(range(5))
    r.keys, r.vals = [], []
    r.admit([30, 30])
    r.step()


def test_a_step_past_the_table_changes_nothing():
    r = Requests(3, 9, max_tokens=32)
    r.admit([32, 10])
    before = r.state()
    with pytest.raises(RuntimeError):
        r.run.step(*r.rows(2), torch.tensor([32, 10], dtype=torch.int32, device="cuda"))
    assert r.state() == before


def test_refused_prompts_are_not_admitted():
    """Without pages in the middle of the call, without a place in the batch, past the table, with arguments that do not
    fit: no request of the call is there, no page is gone, and the others go on."""
    r = Requests(4, 12, max_batch=4, max_tokens=100)
    r.admit([40, 5])
    r.step()
    before = r.state()
    positions = lambda lens: torch.cat([torch.arange(n) for n in lens]).to(torch.int32).cuda()  # noqa: E731
    for lens in ([60, 90], [10, 10, 10], [113], [20, -1]):
        with pytest.raises((RuntimeError, ValueError)):
            r.run.admit(*r.rows(max(0, sum(lens))), lens, positions([max(0, n) for n in lens]))
        assert r.state() == before
    q, k, v = r.rows(30)
    for args in ((q, k, v, [20, 11], positions([20, 11])), (q, k, v, [20, 9], positions([20, 9])),
                 (q[:-1], k, v, [20, 10], positions([20, 10])), (q, k, v, [20, 10], positions([20, 9])),
                 (q, k, v.half(), [20, 10], positions([20, 10])), (q, k, v, [20, 10], positions([20, 10]).cpu()),
                 (q, k.cpu(), v, [20, 10], positions([20, 10])), (q, k, v, [20, 10], positions([20, 10]), k[:, :1]),
                 # what only the attention refuses, after the append: heads whose values are the same memory
                 (q, k, v[:, :1].expand(30, HEADS, D), [20, 10], positions([20, 10]))):
        with pytest.raises((ValueError, hg.HGError)):
            r.run.admit(*args)
        assert r.state() == before
    r.step()
    r.admit([33, 70])
    r.step()


def test_no_prompt_and_empty_prompts():
    r = Requests(5, 8)
    r.admit([])
    r.admit([0, 17, 0])
    for _ in range(2):
        r.step()
    assert r.run.lengths == [2, 19, 2]
