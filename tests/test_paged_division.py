"""The paged decodes' division of work, the header's own code run on the CPU: every warp of a CTA finds the same work whatever
the warps' order, every tile is some CTA's once, and no CTA gets far more than its share."""
import ctypes
import os
import re
import subprocess

import pytest

import paper_2609_35800_gb300 as hg

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(os.path.abspath(hg.__file__)), "csrc_attention")
CTAS = 304  # two for each of 152 SMs


def _source(name):
    with open(os.path.join(CSRC, name)) as f:
        return f.read()


def _number(pattern, text):
    return int(re.search(pattern, text).group(1))


class Division:
    def __init__(self, where, kernel, tile, weighs):
        text = _source("hg_pages_split.cuh")
        text = text[text.index("constexpr unsigned kAll"):text.index("// Lets the launch's page ids")]
        (where / "division.inc").write_text(text)
        kernel, header = _source(kernel), _source("hg_attention.h")
        item = re.search(r"kItemCost = (\w+)", kernel).group(1)
        self.item_cost = int(item) if item.isdigit() else _number(item + r" = (\d+)", header)
        self.join_cost = _number(r"kJoinCost = (\d+)", kernel)
        self.tile = _number(tile + r" = (\d+)", header)
        assert "kWeighsWhole = %s;" % weighs in kernel
        least = re.search(r"least_share\(int\w*(?: group)?\) \{ return ([^;]*);", kernel).group(1)
        least = [int(x) for x in re.match(r"group > 8 \? (\d+) : (\d+)$|(\d+)$", least).groups() if x] * 2
        flags = dict(TILE=self.tile, CONSUMERS=_number(r"kConsumers = (\d+)", kernel), ITEM_COST=self.item_cost,
                     JOIN_COST=self.join_cost, LEAST_MANY=least[0], LEAST_FEW=least[1], WEIGHS_WHOLE=weighs)
        self.threads = 32 * (flags["CONSUMERS"] + 1)
        so = str(where / "division.so")
        subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wno-unknown-pragmas", "-shared", "-fPIC", "-I", str(where)] +
                       ["-D%s=%s" % x for x in flags.items()] + [os.path.join(HERE, "paged_division.cpp"), "-o", so], check=True)
        self.lib = ctypes.CDLL(so)

    def cta(self, lengths, heads, cta, group=4, late=-1, ctas=CTAS):
        """What every thread of the CTA finds: (tiles, request, head, tile, first unit, its unit of the item, share, CTAs)."""
        n = len(lengths)
        out = (ctypes.c_int32 * (8 * self.threads))()
        stride = max(max(lengths, default=0), 0) // 16 + 1
        assert self.lib.divide(n, heads, group, 4, stride, (ctypes.c_int32 * n)(*lengths), ctas, cta, late, out) == 0
        return [tuple(out[8 * i:8 * i + 8]) for i in range(self.threads)]

    def tiles(self, n):
        return max(1, -(-n // self.tile))

    def whole_launch(self, lengths, heads, group=4, ctas=CTAS):
        """Every CTA's items [(request, head, first tile, tiles)], and a share."""
        work, share = [], 0
        for j in range(ctas):
            rows = self.cta(lengths, heads, j, group, ctas=ctas)
            assert all(r[0] == rows[0][0] for r in rows)
            left, b, h, t = rows[0][:4]
            if left > 0:
                assert all(r == rows[0] for r in rows)
                share = rows[0][6]
            mine = []
            while left > 0:
                n = min(left, self.tiles(lengths[b]) - t)
                mine.append((b, h, t, n))
                left, t, h = left - n, 0, h + 1
                if h == heads:
                    b, h = b + 1, 0
            work.append(mine)
        return work, share


@pytest.fixture(scope="module", params=[("hg_pages8_decode.cu", "kDecodeTile8", "true"), ("hg_pages_decode.cu", "kDecodeTile", "false")],
                ids=["8 bits", "16 bits"])
def division(request, tmp_path_factory):
    return Division(tmp_path_factory.mktemp("division"), *request.param)


BATCHES = {
    "more items than CTAs": ([8577] * 40, 8), "of mixed lengths": ([9001 - 211 * i for i in range(42)], 8),
    "one": ([131073], 4), "few": ([2000] * 4, 32), "short": ([500] * 64, 8), "empty": ([0, 5, 0, 0, 7000], 2),
    "many": ([37 * i % 4001 for i in range(300)], 3), "more than kept": ([16 * i for i in range(200)], 2), "equal": ([8577] * 32, 8),
    "a long one": ([100] * 30 + [60000], 8),
}


@pytest.mark.parametrize("late", range(4))
@pytest.mark.parametrize("batch", ["more items than CTAs", "of mixed lengths", "many", "equal"])
def test_warps_find_the_same_work_whatever_their_order(division, batch, late):
    """A warp may fall behind by any time between two barriers, while the others go on to the next use of the memory that the
    division was worked out in."""
    for cta in (0, 5, 150, CTAS - 1):
        rows = division.cta(*BATCHES[batch], cta, late=late)
        assert all(r[0] == rows[0][0] for r in rows), "tiles %s" % sorted({r[0] for r in rows})
        assert rows[0][0] == 0 or all(r == rows[0] for r in rows)


@pytest.mark.parametrize("group", [4, 12])
@pytest.mark.parametrize("batch", list(BATCHES))
def test_every_tile_is_some_ctas_once(division, batch, group):
    lengths, heads = BATCHES[batch]
    work, _ = division.whole_launch(lengths, heads, group)
    got = [(b, h, t + i) for mine in work for b, h, t, n in mine for i in range(n)]
    assert got == [(b, h, t) for b, n in enumerate(lengths) for h in range(heads) for t in range(division.tiles(n))]


FEW = {
    "a third of 3 tiles": ([180 if i % 3 == 0 else 8570 for i in range(38)], 8), "the first third short": ([180] * 13 + [8570] * 25, 8),
    "spread": ([1 + 8576 * i // 35 for i in range(36)], 8), "alike": ([8000 + 18 * i for i in range(32)], 8),
    "two lengths": ([4000, 8577] * 16, 8), "one long": ([9001] + [3000] * 29, 8), "as many as CTAs": ([8577] * 38, 8),
    "equal": ([8577] * 32, 8), "short": ([500, 1] * 15, 8),
}


@pytest.mark.parametrize("batch", list(FEW))
def test_no_more_items_than_ctas(division, batch):
    """Where whole items are taken, the fullest CTA has 1.5 shares and a join at most, whatever begins in its run; otherwise each
    has its share.  (16-bit pages: whole items by the longest alone, left as it was.)"""
    if division.tile == 32:
        pytest.skip("another rule")
    lengths, heads = FEW[batch]
    assert len(lengths) * heads <= CTAS
    work, share = division.whole_launch(lengths, heads)
    units = [sum(n + (division.item_cost if t == 0 else 0) for _, _, t, n in mine) for mine in work]
    whole = all(n == division.tiles(lengths[b]) for mine in work for b, _, _, n in mine)
    # (cut: the fixed costs of an item that a run begins with may be units of the run before)
    most = 1.5 * share + division.join_cost if whole else share + 1 + division.item_cost
    assert max(units) <= most, "%d units, a share is %d" % (max(units), share)
    if batch in ("equal", "as many as CTAs", "alike"):
        assert whole  # one item a CTA
