"""Refusals of the paged and prompt attention entry points, on CPU: the C ABI's (status codes, nothing enqueued) and
the Python binding's (ValueError before the library is entered)."""
import ctypes
import os
import re
import struct

import pytest
import torch

import paper_2609_35800_gb300 as hg
from paper_2609_35800_gb300 import build

OK, INVALID, ALIGN, UNSUPPORTED, WS_SMALL = 0, 1, 2, 3, 4
A = 1 << 40  # an aligned address that nothing reads


@pytest.fixture(scope="module")
def lib():
    build.build()
    return hg.library()


def _shape(**kw):
    d = dict(dtype=0, num_pages=10, page_size=16, num_kv_heads=4, head_dim=128, page_stride=0, head_stride=0, token_stride=0)
    d.update(kw)
    return hg.PageShape(**d)


def _create(lib, k=A, v=A, **kw):
    h = ctypes.c_void_p()
    st = lib.hg_pages_create(ctypes.byref(_shape(**kw)), k, v, ctypes.byref(h))
    if st == OK:
        lib.hg_pages_destroy(h)
    return st


@pytest.mark.parametrize("kw,status", [
    (dict(), OK),
    (dict(dtype=1, page_size=256, num_kv_heads=64), OK),
    (dict(page_stride=4 * 16 * 128, head_stride=128, token_stride=4 * 128), OK),
    (dict(dtype=2), INVALID), (dict(dtype=-1), INVALID),
    (dict(num_pages=0), INVALID), (dict(num_kv_heads=0), INVALID), (dict(page_size=0), INVALID),
    (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED), (dict(page_size=512), UNSUPPORTED),
    (dict(head_dim=64), UNSUPPORTED), (dict(num_kv_heads=65), UNSUPPORTED),
    (dict(num_pages=1 << 27), UNSUPPORTED),
    (dict(page_stride=-8), INVALID),
    (dict(page_stride=8192, head_stride=2048, token_stride=64), INVALID),
    (dict(page_stride=8192, head_stride=64, token_stride=128), INVALID),
    (dict(page_stride=64, head_stride=2048, token_stride=128), INVALID),
    (dict(page_stride=8196, head_stride=2048, token_stride=128), ALIGN),
    (dict(page_stride=1 << 38, head_stride=2048, token_stride=128), UNSUPPORTED),
    (dict(k=A + 8), ALIGN), (dict(v=A + 2), ALIGN), (dict(k=None), INVALID), (dict(v=None), INVALID),
])
def test_create(lib, kw, status):
    assert _create(lib, **kw) == status


def test_create_null(lib):
    h = ctypes.c_void_p()
    assert lib.hg_pages_create(None, A, A, ctypes.byref(h)) == INVALID
    assert lib.hg_pages_create(ctypes.byref(_shape()), A, A, None) == INVALID
    lib.hg_pages_destroy(None)


@pytest.fixture(scope="module")
def pages(lib):
    h = ctypes.c_void_p()
    assert lib.hg_pages_create(ctypes.byref(_shape()), A, A, ctypes.byref(h)) == OK
    yield h
    lib.hg_pages_destroy(h)


def _rows(data=A, token=512, head=128):
    return (data, token, head)


def _io(*rows):
    return struct.pack("=%dq" % (3 * len(rows)), *(x for r in rows for x in r))


def _rotation(table=A, table_len=100, rot_dim=128, interleaved=0, sections=(0, 0, 0)):
    raw = hg._Rotation(table, table_len, rot_dim, interleaved, (ctypes.c_int32 * 3)(*sections))
    return raw


NONE = (0, 0, 0)


@pytest.mark.parametrize("kw,status", [
    (dict(tokens=0), OK),
    (dict(tokens=0, slots=None), OK),
    (dict(tokens=-1), INVALID), (dict(heads=-1), INVALID), (dict(heads=1025), UNSUPPORTED),
    (dict(slots=None), INVALID), (dict(slots=A + 2), ALIGN),
    (dict(k=NONE), INVALID), (dict(v=NONE), INVALID), (dict(q=NONE), INVALID), (dict(q_out=NONE), INVALID),
    (dict(k=_rows(A + 8)), ALIGN), (dict(v=_rows(token=513)), ALIGN), (dict(q=_rows(head=-128)), INVALID),
    (dict(k_out=_rows(A + 4)), ALIGN), (dict(v_out=_rows(token=1 << 38)), INVALID),
    (dict(rotation=dict(table=None)), INVALID), (dict(rotation=dict(table=A + 4)), ALIGN),
    (dict(rotation=dict(), positions=None), INVALID), (dict(rotation=dict(), positions=A + 1), ALIGN),
    (dict(rotation=dict(table_len=0)), INVALID), (dict(rotation=dict(interleaved=2)), INVALID),
    (dict(rotation=dict(rot_dim=0)), UNSUPPORTED), (dict(rotation=dict(rot_dim=24)), UNSUPPORTED),
    (dict(rotation=dict(rot_dim=144)), UNSUPPORTED),
    (dict(rotation=dict(sections=(16, 24, 23))), INVALID), (dict(rotation=dict(sections=(-8, 48, 24))), INVALID),
    (dict(rotation=dict(sections=(20, 20, 24))), UNSUPPORTED),
    (dict(pages=None), INVALID), (dict(io=None), INVALID),
])
def test_append(lib, pages, kw, status):
    d = dict(pages=pages, tokens=3, heads=8, q=_rows(), k=_rows(), v=_rows(), q_out=_rows(), k_out=NONE, v_out=NONE,
             rotation=None, positions=A, slots=A)
    d.update(kw)
    io = d["io"] if "io" in d else _io(d["q"], d["k"], d["v"], d["q_out"], d["k_out"], d["v_out"])
    rot = None if d["rotation"] is None else ctypes.byref(_rotation(**d["rotation"]))
    assert lib.hg_pages_append(d["pages"], d["tokens"], d["heads"], io, rot, d["positions"], d["slots"], None) == status


@pytest.mark.parametrize("step", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), OK),
    (dict(batch=-1), INVALID), (dict(heads=0), INVALID), (dict(heads=6), INVALID), (dict(heads=68), UNSUPPORTED),
    (dict(batch=(1 << 20) + 1), UNSUPPORTED),
    (dict(pages=None), INVALID), (dict(io=None), INVALID), (dict(table=None), INVALID), (dict(lengths=None), INVALID),
    (dict(table=A + 2), ALIGN), (dict(lengths=A + 1), ALIGN), (dict(lse=A + 2), ALIGN),
    (dict(stride=-1), INVALID), (dict(stride=1 << 28), UNSUPPORTED),
    (dict(q=NONE), INVALID), (dict(out=NONE), INVALID), (dict(q=_rows(A + 8)), ALIGN), (dict(out=_rows(head=132)), ALIGN),
    (dict(scale=float("nan")), INVALID),
    (dict(ws=None), INVALID), (dict(ws=A + 8), ALIGN), (dict(ws_bytes=-1), WS_SMALL),
])
def test_decode(lib, pages, step, kw, status):
    need = ctypes.c_size_t()
    assert lib.hg_pages_decode_workspace_size(pages, 3, 8, ctypes.byref(need)) == OK
    d = dict(pages=pages, batch=3, heads=8, q=_rows(), k=_rows(), v=_rows(), out=_rows(), table=A, stride=5, lengths=A,
             lse=None, scale=0.0, ws=A, ws_bytes=0)
    d.update(kw)
    io = d["io"] if "io" in d else _io(d["q"], d["k"], d["v"], d["out"])
    tail = (d["table"], d["stride"], d["lengths"], d["lse"], d["scale"], d["ws"], need.value + d["ws_bytes"], None)
    if step:
        got = lib.hg_pages_decode_step(d["pages"], d["batch"], d["heads"], io, None, None, *tail)
    else:
        got = lib.hg_pages_decode_attention(d["pages"], d["batch"], d["heads"], io, *tail)
    assert got == status


def test_decode_step_needs_its_token(lib, pages):
    need = ctypes.c_size_t()
    lib.hg_pages_decode_workspace_size(pages, 3, 8, ctypes.byref(need))
    tail = (A, 5, A, None, 0.0, A, need.value, None)
    for rows, status in (((_rows(), NONE, _rows(), _rows()), INVALID), ((_rows(), _rows(), _rows(A + 2), _rows()), ALIGN)):
        assert lib.hg_pages_decode_step(pages, 3, 8, _io(*rows), None, None, *tail) == status
    rot = _rotation(rot_dim=20)
    rows = _io(_rows(), _rows(), _rows(), _rows())
    assert lib.hg_pages_decode_step(pages, 3, 8, rows, ctypes.byref(rot), A, *tail) == UNSUPPORTED


def test_decode_workspace_size(lib, pages):
    n = ctypes.c_size_t()
    f = lib.hg_pages_decode_workspace_size
    assert f(pages, 3, 8, None) == INVALID
    assert f(None, 3, 8, ctypes.byref(n)) == INVALID
    assert f(pages, -1, 8, ctypes.byref(n)) == INVALID
    assert f(pages, 3, 7, ctypes.byref(n)) == INVALID
    assert f(pages, 3, 68, ctypes.byref(n)) == UNSUPPORTED
    sizes = []
    for batch in (0, 1, 8, 100):
        assert f(pages, batch, 8, ctypes.byref(n)) == OK
        sizes.append(n.value)
    assert sizes == sorted(sizes) and sizes[0] >= 512


@pytest.mark.parametrize("kw,status", [
    (dict(count=0), OK), (dict(q_begin=(5, 5, 5)), OK), (dict(count=0, ws=None), OK),
    (dict(dtype=2), INVALID), (dict(count=-1), INVALID), (dict(hq=0), INVALID), (dict(hkv=0), INVALID),
    (dict(hq=6), INVALID), (dict(hq=68), UNSUPPORTED), (dict(hq=65, hkv=65), UNSUPPORTED),
    (dict(q_begin=None), INVALID), (dict(k_begin=None), INVALID),
    (dict(q_begin=(0, 5, 4)), INVALID), (dict(k_begin=(0, 9, 8)), INVALID), (dict(q_begin=(-1, 5, 6)), INVALID),
    (dict(causal=2), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(io=None), INVALID), (dict(q=NONE), INVALID), (dict(k=NONE), INVALID), (dict(v=NONE), INVALID), (dict(out=NONE), INVALID),
    (dict(k=_rows(A + 8)), ALIGN), (dict(v=_rows(token=129)), ALIGN), (dict(out=_rows(head=-8)), INVALID),
    (dict(lse=A + 2), ALIGN), (dict(ws=None), INVALID), (dict(ws=A + 8), ALIGN), (dict(ws_bytes=-1), WS_SMALL),
    (dict(k=_rows(head=0)), UNSUPPORTED), (dict(q=_rows(token=64)), UNSUPPORTED),  # rows that share memory
    (dict(k=_rows(head=0), ws=None), UNSUPPORTED),
])
def test_prompt(lib, kw, status):
    need = ctypes.c_size_t()
    assert lib.hg_prompt_workspace_size(None) == INVALID
    assert lib.hg_prompt_workspace_size(ctypes.byref(need)) == OK
    d = dict(dtype=0, count=2, hq=8, hkv=4, q=_rows(), k=_rows(), v=_rows(), out=_rows(), q_begin=(0, 5, 9),
             k_begin=(0, 5, 9), lse=None, causal=1, scale=0.0, ws=A, ws_bytes=0)
    d.update(kw)
    io = d["io"] if "io" in d else _io(d["q"], d["k"], d["v"], d["out"])
    ints = lambda x: None if x is None else (ctypes.c_int32 * len(x))(*x)  # noqa: E731
    assert lib.hg_prompt_attention(d["dtype"], d["count"], d["hq"], d["hkv"], io, ints(d["q_begin"]), ints(d["k_begin"]),
                                   d["lse"], d["causal"], d["scale"], d["ws"], need.value + d["ws_bytes"], None) == status


# -- the binding's own checks ------------------------------------------------------------------------------------------

def _raises(fn, what):
    with pytest.raises(ValueError) as e:
        fn()
    assert what in str(e.value), str(e.value)


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


@pytest.fixture
def pool(lib, pages):
    return hg.Pages(None, _t(10, 4, 16, 128), None, _shape())


def test_binding_create(lib):
    p = _t(10, 4, 16, 128)
    _raises(lambda: hg.hg_pages_create(p, p), "CUDA")
    _raises(lambda: hg.hg_pages_create(p, p[:9]), "of one type")
    _raises(lambda: hg.hg_pages_create(p, p.half()), "of one type")
    _raises(lambda: hg.hg_pages_create(p.float(), p.float()), "bfloat16 or float16")
    _raises(lambda: hg.hg_pages_create(p, _t(10, 16, 4, 128).transpose(1, 2)), "same strides")
    _raises(lambda: hg.Rotation(torch.zeros(4, 128, dtype=torch.float64)), "float32")
    _raises(lambda: hg.Rotation(torch.zeros(4, 128)), "CUDA")


def test_binding_append(pool):
    q, k, i = _t(3, 8, 128), _t(3, 4, 128), torch.zeros(3, dtype=torch.int32)
    f = hg.hg_pages_append
    _raises(lambda: f(pool, q, k, k, None, None, i, q), "must be a CUDA tensor")
    _raises(lambda: f(pool, q, k, k, None, None, i), "needs q_out")
    _raises(lambda: f(pool, q[:2], k, k, None, None, i, q), "q is")
    _raises(lambda: f(pool, None, k[:, :3], k, None, None, i), "k is")
    _raises(lambda: f(pool, None, k.half(), k, None, None, i), "k is")
    _raises(lambda: f(pool, None, _t(3, 128, 4).transpose(1, 2), k, None, None, i), "dense channels")


def test_binding_decode_and_prompt(pool):
    q, k, i = _t(3, 8, 128), _t(3, 4, 128), torch.zeros(3, dtype=torch.int32)
    _raises(lambda: hg.hg_pages_decode_attention(pool, q, i, i, q, None, 0.0, i), "must be a CUDA tensor")
    _raises(lambda: hg.hg_pages_decode_attention(pool, q.half(), i, i, q, None, 0.0, i), "q is")
    _raises(lambda: hg.hg_pages_decode_step(pool, q, k[:2], k, None, None, i, i, q, None, 0.0, i), "must be a CUDA tensor")
    _raises(lambda: hg._decode_table("f", i, i, 3), "page_table must be")
    _raises(lambda: hg._ints("f", "x", i, 4), "holds 3 entries")
    _raises(lambda: hg._ints("f", "x", i.long(), 3), "contiguous int32")
    _raises(lambda: hg._ints("f", "x", i, 3), "must be a CUDA tensor")
    _raises(lambda: hg._lse("f", torch.zeros(3, 8, dtype=torch.float64), 3, 8), "lse must be")
    _raises(lambda: hg._lse("f", torch.zeros(3, 8), 3, 8), "CUDA")
    _raises(lambda: hg.hg_prompt_attention(q.float(), k, k, i, i, q, None, True, 0.0, i), "bfloat16 or float16")
    _raises(lambda: hg.hg_prompt_attention(q, k, k, i, i, q, None, True, 0.0, i), "CUDA tensor")
    _raises(lambda: hg._workspace("f", i), "workspace must be a CUDA tensor")
    _raises(lambda: hg._workspace("f", None), "workspace must be a tensor")


class _Turn:
    """Stands for a Rotation of three positions a token; the checks come before its table is read."""
    pointer, positions = 0, 3


@pytest.mark.parametrize("shape", [(3, 64), (64, 3), (3, 4), (5, 3), (192,), (4, 5), (1, 15), (15, 1)])
def test_three_positions_have_the_calls_own_layout(shape):
    """Positions are read as [3][tokens]: a buffer of more tokens, or one of tokens first, holds enough entries, elsewhere."""
    positions = torch.zeros(shape, dtype=torch.int32)
    _raises(lambda: hg._rotated_by("f", _Turn, positions, 5), "f: positions are %s, the call takes [3][5]" % list(shape))


@pytest.mark.parametrize("shape", [(3, 5), (15,)])
def test_three_positions_as_the_call_takes_them(shape):
    _raises(lambda: hg._rotated_by("f", _Turn, torch.zeros(shape, dtype=torch.int32), 5), "must be a CUDA tensor")
    _raises(lambda: hg._rotated_by("f", _Turn, torch.zeros(shape), 5), "contiguous int32")


class _Table:
    """A table on no GPU in particular: the rotation keeps its address."""
    dtype, is_cuda, shape = torch.float32, True, (10, 128)
    dim = staticmethod(lambda: 2)
    is_contiguous = staticmethod(lambda: True)
    data_ptr = staticmethod(lambda: A)


@pytest.mark.parametrize("sections,positions", [(None, 1), ((0, 0, 0), 1), ((16, 24, 24), 3), ((0, 0, 64), 3)])
def test_positions_of_a_rotation(sections, positions):
    """Sections that are all 0 are one position a token, in the library and in the binding."""
    rotation = hg.Rotation(_Table, sections=sections)
    assert rotation.positions == positions
    assert tuple(rotation.raw.sections) == (sections or (0, 0, 0))


@pytest.mark.parametrize("before", [0, 255, 256, 600])
def test_prompts_are_planned_before_the_first_launch(lib, before):
    """2^30 tokens of 64 heads are more than one launch numbers: refused as such, whatever comes before them."""
    need = ctypes.c_size_t()
    assert lib.hg_prompt_workspace_size(ctypes.byref(need)) == OK
    q_begin = list(range(before + 1)) + [before + (1 << 30)]
    k_begin = list(range(before + 2))
    ints = lambda x: (ctypes.c_int32 * len(x))(*x)  # noqa: E731
    io = _io(*[_rows(token=64 * 128)] * 4)
    got = lib.hg_prompt_attention(0, before + 1, 64, 64, io, ints(q_begin), ints(k_begin), None, 1, 0.0, A, need.value, None)
    assert got == UNSUPPORTED


@pytest.mark.parametrize("batch,heads,page_size", [(1 << 10, 4, 16), (1 << 17, 64, 16), (1 << 20, 2, 32)])
def test_decode_takes_tables_up_to_the_headers_limit(lib, batch, heads, page_size):
    """Of a table that the header allows only the workspace, which is too small, is refused."""
    text = open(os.path.join(build.INCLUDE, "headguard.h")).read()
    more = int(re.search(r"table_stride \* page_size / 32[\s*]*\+[\s*]*(\d+)", text).group(1))
    h = ctypes.c_void_p()
    assert lib.hg_pages_create(ctypes.byref(_shape(num_kv_heads=heads, page_size=page_size)), A, A, ctypes.byref(h)) == OK
    try:
        tiles = (1 << 31) // (batch * heads) - more  # the first number of tiles that is not allowed
        for over in (False, True):
            stride = max(0, (tiles if over else tiles - 1) * 32 // page_size)
            if over and stride * page_size // 32 < tiles:
                stride += 1
            if stride * page_size >= 1 << 31:
                continue
            got = lib.hg_pages_decode_attention(h, batch, heads, _io(_rows(), NONE, NONE, _rows()), A, stride, A, None, 0.0, A,
                                                0, None)
            assert got == (UNSUPPORTED if over else WS_SMALL)
    finally:
        lib.hg_pages_destroy(h)
