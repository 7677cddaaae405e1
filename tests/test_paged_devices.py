"""The calls of the 16-bit caches take tensors of one device, the current one: a launch goes to no other, and an address of
another's memory would fault there.  On CPU, with tensors that only say where they are."""
import pytest
import torch

import paper_2609_35800_gb300 as hg
from paper_2609_35800_gb300 import build

A = 1 << 40  # an aligned address that nothing reads


class _Tensor:
    """A tensor on a GPU that this machine may not have."""
    is_cuda = True

    def __init__(self, index, dtype, *shape):
        self.index, self.device, self.dtype, self.shape, self.nbytes = index, "cuda:%d" % index, dtype, torch.Size(shape), 1 << 30

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return True

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def stride(self, axis=None):
        strides = [1]
        for n in reversed(self.shape[1:]):
            strides.insert(0, strides[0] * n)
        return tuple(strides) if axis is None else strides[axis]

    def data_ptr(self):
        return A


class _Library:
    """Stands for the library: a call that comes so far has passed the binding's checks."""

    def __getattr__(self, name):
        def call(*args):
            self.called = name
            return 0
        return call


BF16, I32 = torch.bfloat16, torch.int32
NAMES = {
    "append": ["q", "k", "v", "q_out", "k_out", "v_out", "slots", "positions", "the rotation's table"],
    "decode_attention": ["q", "out", "page_table", "lengths", "lse", "workspace"],
    "decode_step": ["q", "k", "v", "out", "page_table", "lengths", "lse", "workspace", "positions", "the rotation's table"],
    "prompt_attention": ["q", "k", "v", "out", "lse", "workspace"],
}


def _call(what, where, default, stream=None):
    """The call, each tensor on the device that `where` says."""
    t = lambda name, dtype, *shape: _Tensor(where.get(name, default), dtype, *shape)  # noqa: E731
    pool = _Tensor(default, BF16, 10, 4, 16, 128)
    pages = hg.Pages(None, pool, pool, hg.PageShape(0, 10, 16, 4, 128, 0, 0, 0))

    class Turn:
        pointer, positions, table = 0, 1, t("the rotation's table", torch.float32, 9, 128)
    q, k, v, out = t("q", BF16, 3, 8, 128), t("k", BF16, 3, 4, 128), t("v", BF16, 3, 4, 128), t("out", BF16, 3, 8, 128)
    pos, lse, ws = t("positions", I32, 3), t("lse", torch.float32, 3, 8), t("workspace", torch.uint8, 1 << 30)
    if what == "append":
        return hg.hg_pages_append(pages, q, k, v, Turn, pos, t("slots", I32, 3), t("q_out", BF16, 3, 8, 128),
                                  t("k_out", BF16, 3, 4, 128), t("v_out", BF16, 3, 4, 128), stream)
    if what == "prompt_attention":
        ends = torch.tensor([0, 3], dtype=I32)
        return hg.hg_prompt_attention(q, k, v, ends, ends, out, lse, True, 0.0, ws, stream)
    tail = (t("page_table", I32, 3, 5), t("lengths", I32, 3), out, lse, 0.0, ws, stream)
    if what == "decode_attention":
        return hg.hg_pages_decode_attention(pages, q, *tail)
    return hg.hg_pages_decode_step(pages, q, k, v, Turn, pos, *tail)


@pytest.fixture
def library(monkeypatch):
    stand_in = _Library()
    monkeypatch.setattr(hg, "library", lambda: stand_in)
    monkeypatch.setattr(hg._types, "device", lambda: 0, raising=False)
    monkeypatch.setattr(hg._types, "stream", lambda device: 77, raising=False)
    stand_in.called = None
    return stand_in


@pytest.mark.parametrize("what", list(NAMES))
def test_one_device(library, what):
    _call(what, {}, 0)
    assert library.called == ("hg_" if what == "prompt_attention" else "hg_pages_") + what
    library.called = None
    for name in NAMES[what]:
        if what == "prompt_attention" and name == "q":
            continue  # the others' device is q's
        with pytest.raises(ValueError, match="%s is on cuda:1, the call's tensors are on cuda:0" % name):
            _call(what, {name: 1}, 0)
    for stream in (None, 5):
        with pytest.raises(ValueError, match="the call's tensors are on cuda:1, the current device is cuda:0"):
            _call(what, {}, 1, stream)
    assert library.called is None


def test_a_pool_is_on_one_device(library):
    with pytest.raises(ValueError, match="one device"):
        hg.hg_pages_create(_Tensor(0, BF16, 10, 4, 16, 128), _Tensor(1, BF16, 10, 4, 16, 128))
    assert library.called is None


def test_the_cpus_tensors_are_refused():
    build.build()
    pages = hg.Pages(None, torch.zeros(10, 4, 16, 128, dtype=BF16), None, hg.PageShape(0, 10, 16, 4, 128, 0, 0, 0))
    q, k, i = torch.zeros(3, 8, 128, dtype=BF16), torch.zeros(3, 4, 128, dtype=BF16), torch.zeros(3, dtype=I32)
    with pytest.raises(ValueError, match="must be a CUDA tensor"):
        hg.hg_pages_append(pages, q, k, k, None, None, i, q)
    with pytest.raises(ValueError, match="must be a CUDA tensor"):
        hg.hg_prompt_attention(q, k, k, i[:2], i[:2], q, None, True, 0.0, i)
