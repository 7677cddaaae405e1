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
        pos = torch.cat([torch.arange(n) for n in lens]).to(torch.int32).cuda()
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
