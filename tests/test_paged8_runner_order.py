"""Paged8Runner on the CPU, the library's calls stood in for: once a call has stored tokens, which may store a request's last
block again more coarsely, nothing that can fail is left to do but launches."""
import pytest
import torch

from paper_2609_35800_gb300 import paged

HEADS, GROUP, D, SIZE = 2, 3, 128, 16
HQ = HEADS * GROUP
CALLS = ("hg_pages8_create", "hg_pages8_decode_workspace_size", "hg_prompt_workspace_size", "hg_workspace_clear", "hg_pages_plan",
         "hg_pages8_append", "hg_pages8_dequantize", "hg_prompt_attention", "hg_pages8_decode_step")


class _Torch:
    """torch, whose calls are counted: the `fails`-th one from `count` = 0 on runs out of memory."""

    def __init__(self):
        self.count, self.fails, self.seen = 0, None, []

    def __getattr__(self, name):
        what = getattr(torch, name)
        if name not in ("empty", "empty_like", "zeros", "tensor", "arange", "ones", "cat"):
            return what

        def call(*args, **kw):
            self.count += 1
            self.seen.append(name)
            if self.count == self.fails:
                raise torch.OutOfMemoryError("no memory left")
            return what(*args, **kw)
        return call


@pytest.fixture
def runner(monkeypatch):
    calls = []

    def stand_in(name):
        def call(*args, **kw):
            calls.append(name)
            run.torch.seen.append(name)
            return 64 if name.endswith("size") else None
        return call
    for name in CALLS:
        monkeypatch.setattr(paged, name, stand_in(name))
    run = type("", (), {})()
    run.torch = _Torch()
    monkeypatch.setattr(paged, "torch", run.torch)
    run.it = paged.Paged8Runner(40, SIZE, HQ, HEADS, device="cpu", max_batch=4, max_tokens=200)
    run.calls = calls
    return run


def _rows(n, hq=HQ, heads=HEADS):
    return (torch.zeros((n, h, D), dtype=torch.bfloat16) for h in (hq, heads, heads))


def _state(run):
    return list(run.it.lengths), run.it.free_pages, run.it.lens.tolist(), id(run.it.counts)


@pytest.mark.parametrize("what", ["admit", "extend"])
def test_nothing_is_stored_by_a_call_that_runs_out_of_memory(runner, what):
    runner.it.admit(*_rows(25), [20, 5])
    before = _state(runner)
    for fails in range(1, 40):
        runner.calls.clear()
        runner.torch.count, runner.torch.fails = 0, fails
        try:
            getattr(runner.it, what)(*_rows(10), [4, 6])
        except torch.OutOfMemoryError:
            assert "hg_pages8_append" not in runner.calls, "failed at %s" % runner.torch.seen[-1]
            assert _state(runner) == before
        else:
            break
    assert runner.torch.count < fails and fails > 5
    # what came behind the store
    tail = runner.torch.seen[len(runner.torch.seen) - runner.torch.seen[::-1].index("hg_pages8_append"):]
    assert tail == (["hg_pages8_dequantize"] if what == "extend" else []) + ["hg_prompt_attention"]


@pytest.mark.parametrize("hq,heads", [(HQ + HEADS, HEADS), (HQ - 1, HEADS), (17 * HEADS, HEADS)])
@pytest.mark.parametrize("what", ["admit", "extend"])
def test_other_heads_are_refused_before_anything_is_stored(runner, what, hq, heads):
    runner.it.admit(*_rows(25), [20, 5])
    before = _state(runner)
    runner.calls.clear()
    with pytest.raises(ValueError, match="query heads"):
        getattr(runner.it, what)(*_rows(10, hq, heads), [4, 6])
    assert runner.calls == [] and _state(runner) == before
