"""Refusals of the 8-bit paged cache's and the page plan's entry points, on CPU: the C ABI's (status codes, nothing
enqueued) and the Python binding's (ValueError before the library is entered)."""
import ctypes
import struct

import pytest
import torch

import paper_2609_35800_gb300 as hg
from paper_2609_35800_gb300 import build

OK, INVALID, ALIGN, UNSUPPORTED, WS_SMALL = 0, 1, 2, 3, 4
A = 1 << 40  # an aligned address that nothing reads
NONE = (0, 0, 0)


@pytest.fixture(scope="module")
def lib():
    build.build()
    return hg.library()


def _shape(**kw):
    d = dict(dtype=0, num_pages=10, page_size=16, num_kv_heads=4, head_dim=128, page_stride=0, head_stride=0, token_stride=0)
    d.update(kw)
    return hg.PageShape(**d)


@pytest.mark.parametrize("kw,status", [
    (dict(), OK), (dict(dtype=1, page_size=256, num_kv_heads=64), OK),
    (dict(page_stride=4 * 16 * 128, head_stride=128, token_stride=4 * 128), OK),
    (dict(dtype=2), INVALID), (dict(num_pages=0), INVALID), (dict(num_kv_heads=0), INVALID), (dict(page_size=0), INVALID),
    (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED), (dict(page_size=512), UNSUPPORTED),
    (dict(head_dim=64), UNSUPPORTED), (dict(num_kv_heads=65), UNSUPPORTED), (dict(num_pages=1 << 27), UNSUPPORTED),
    (dict(page_stride=-16), INVALID), (dict(page_stride=8192, head_stride=2048, token_stride=64), INVALID),
    (dict(page_stride=8192 + 8, head_stride=2048, token_stride=128), ALIGN),  # 8 bytes are no 16
    (dict(page_stride=1 << 38, head_stride=2048, token_stride=128), UNSUPPORTED),
    (dict(k=A + 8), ALIGN), (dict(v=A + 1), ALIGN), (dict(ks=A + 2), ALIGN), (dict(vs=A + 1), ALIGN),
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(ks=None), INVALID), (dict(vs=None), INVALID),
])
def test_create(lib, kw, status):
    kw = dict(kw)
    ptr = [kw.pop(n, A) for n in ("k", "v", "ks", "vs")]
    h = ctypes.c_void_p()
    got = lib.hg_pages8_create(ctypes.byref(_shape(**kw)), *ptr, ctypes.byref(h))
    if got == OK:
        lib.hg_pages8_destroy(h)
    assert got == status


def test_create_null(lib):
    h = ctypes.c_void_p()
    assert lib.hg_pages8_create(None, A, A, A, A, ctypes.byref(h)) == INVALID
    assert lib.hg_pages8_create(ctypes.byref(_shape()), A, A, A, A, None) == INVALID
    lib.hg_pages8_destroy(None)


@pytest.fixture(scope="module")
def pages(lib):
    h = ctypes.c_void_p()
    assert lib.hg_pages8_create(ctypes.byref(_shape()), A, A, A, A, ctypes.byref(h)) == OK
    yield h
    lib.hg_pages8_destroy(h)


def _rows(data=A, token=512, head=128):
    return (data, token, head)


def _io(*rows):
    return struct.pack("=%dq" % (3 * len(rows)), *(x for r in rows for x in r))


def _rotation(table=A, table_len=100, rot_dim=128, interleaved=0, sections=(0, 0, 0)):
    return hg._Rotation(table, table_len, rot_dim, interleaved, (ctypes.c_int32 * 3)(*sections))


@pytest.mark.parametrize("kw,status", [
    (dict(tokens=0), OK), (dict(tokens=0, begin=None), OK), (dict(requests=0, begin=None, table=None), OK),
    (dict(tokens=-1), INVALID), (dict(requests=-1), INVALID), (dict(heads=-1), INVALID), (dict(heads=1025), UNSUPPORTED),
    (dict(tokens=(1 << 30) + 1), UNSUPPORTED), (dict(requests=(1 << 28) + 1), UNSUPPORTED),
    (dict(begin=None), INVALID), (dict(table=None), INVALID), (dict(lengths=None), INVALID), (dict(stride=-1), INVALID),
    (dict(begin=A + 2), ALIGN), (dict(table=A + 1), ALIGN), (dict(lengths=A + 3), ALIGN), (dict(stride=1 << 28), UNSUPPORTED),
    (dict(k=NONE), INVALID), (dict(v=NONE), INVALID), (dict(q=NONE), INVALID), (dict(q_out=NONE), INVALID),
    (dict(k=_rows(A + 8)), ALIGN), (dict(v=_rows(token=513)), ALIGN), (dict(q=_rows(head=-128)), INVALID),
    (dict(k_out=_rows(A + 4)), ALIGN), (dict(v_out=_rows(token=1 << 38)), INVALID),
    (dict(rotation=dict(table=None)), INVALID), (dict(rotation=dict(), positions=None), INVALID),
    (dict(rotation=dict(rot_dim=24)), UNSUPPORTED), (dict(rotation=dict(sections=(16, 24, 23))), INVALID),
    (dict(pages=None), INVALID), (dict(io=None), INVALID),
])
def test_append(lib, pages, kw, status):
    d = dict(pages=pages, tokens=3, requests=2, heads=8, q=_rows(), k=_rows(), v=_rows(), q_out=_rows(), k_out=NONE, v_out=NONE,
             rotation=None, positions=A, begin=A, table=A, stride=5, lengths=A)
    d.update(kw)
    io = d["io"] if "io" in d else _io(d["q"], d["k"], d["v"], d["q_out"], d["k_out"], d["v_out"])
    rot = None if d["rotation"] is None else ctypes.byref(_rotation(**d["rotation"]))
    assert lib.hg_pages8_append(d["pages"], d["tokens"], d["requests"], d["heads"], io, rot, d["positions"], d["begin"],
                                d["table"], d["stride"], d["lengths"], None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(rows=0), OK), (dict(requests=0), OK),
    (dict(rows=-1), INVALID), (dict(requests=-1), INVALID), (dict(rows=(1 << 30) + 1), UNSUPPORTED),
    (dict(begin=None), INVALID), (dict(table=None), INVALID), (dict(stride=-1), INVALID), (dict(stride=1 << 28), UNSUPPORTED),
    (dict(begin=A + 2), ALIGN), (dict(table=A + 1), ALIGN),
    (dict(k=None, v=None), INVALID), (dict(k=NONE, v=NONE), INVALID), (dict(k=_rows(A + 8)), ALIGN), (dict(k=None, v=_rows(token=4)), ALIGN),
    (dict(v=_rows(head=-8)), INVALID), (dict(pages=None), INVALID),
])
def test_dequantize(lib, pages, kw, status):
    d = dict(pages=pages, rows=3, requests=2, begin=A, table=A, stride=5, k=_rows(), v=_rows())
    d.update(kw)
    k, v = (None if d[x] is None else _io(d[x]) for x in "kv")
    assert lib.hg_pages8_dequantize(d["pages"], d["rows"], d["requests"], d["begin"], d["table"], d["stride"], k, v, None) == status


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
    assert lib.hg_pages8_decode_workspace_size(pages, 3, 8, ctypes.byref(need)) == OK
    d = dict(pages=pages, batch=3, heads=8, q=_rows(), k=_rows(), v=_rows(), out=_rows(), table=A, stride=5, lengths=A,
             lse=None, scale=0.0, ws=A, ws_bytes=0)
    d.update(kw)
    io = d["io"] if "io" in d else _io(d["q"], d["k"], d["v"], d["out"])
    tail = (d["table"], d["stride"], d["lengths"], d["lse"], d["scale"], d["ws"], need.value + d["ws_bytes"], None)
    if step:
        got = lib.hg_pages8_decode_step(d["pages"], d["batch"], d["heads"], io, None, None, *tail)
    else:
        got = lib.hg_pages8_decode_attention(d["pages"], d["batch"], d["heads"], io, *tail)
    assert got == status


def test_decode_step_needs_its_token(lib, pages):
    need = ctypes.c_size_t()
    lib.hg_pages8_decode_workspace_size(pages, 3, 8, ctypes.byref(need))
    tail = (A, 5, A, None, 0.0, A, need.value, None)
    for rows, status in (((_rows(), NONE, _rows(), _rows()), INVALID), ((_rows(), _rows(), _rows(A + 2), _rows()), ALIGN)):
        assert lib.hg_pages8_decode_step(pages, 3, 8, _io(*rows), None, None, *tail) == status
    rows = _io(_rows(), _rows(), _rows(), _rows())
    assert lib.hg_pages8_decode_step(pages, 3, 8, rows, ctypes.byref(_rotation(rot_dim=20)), A, *tail) == UNSUPPORTED


def test_decode_workspace_size(lib, pages):
    n, m = ctypes.c_size_t(), ctypes.c_size_t()
    f = lib.hg_pages8_decode_workspace_size
    assert f(pages, 3, 8, None) == INVALID
    assert f(None, 3, 8, ctypes.byref(n)) == INVALID
    assert f(pages, -1, 8, ctypes.byref(n)) == INVALID
    assert f(pages, 3, 7, ctypes.byref(n)) == INVALID
    assert f(pages, 3, 68, ctypes.byref(n)) == UNSUPPORTED
    h = ctypes.c_void_p()
    assert lib.hg_pages_create(ctypes.byref(_shape()), A, A, ctypes.byref(h)) == OK
    for batch in (0, 1, 8, 100):  # one workspace serves both kinds of pool
        assert f(pages, batch, 8, ctypes.byref(n)) == OK
        assert lib.hg_pages_decode_workspace_size(h, batch, 8, ctypes.byref(m)) == OK
        assert n.value == m.value
    lib.hg_pages_destroy(h)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), INVALID), (dict(size=0), INVALID), (dict(stride=-1), INVALID), (dict(capacity=-1), INVALID),
    (dict(tokens=-1), INVALID), (dict(batch=16385), UNSUPPORTED), (dict(size=8), UNSUPPORTED), (dict(size=48), UNSUPPORTED),
    (dict(size=512), UNSUPPORTED), (dict(stride=1 << 27), UNSUPPORTED), (dict(tokens=(1 << 30) + 1), UNSUPPORTED),
    (dict(batch=16384, stride=1 << 17), UNSUPPORTED),
    (dict(table=None), INVALID), (dict(cached=None), INVALID), (dict(new=None), INVALID), (dict(free=None), INVALID),
    (dict(count=None), INVALID), (dict(lengths=None), INVALID), (dict(begin=None), INVALID), (dict(slots=None), INVALID),
    (dict(counts=None), INVALID),
] + [({x: A + 2}, ALIGN) for x in ("table", "cached", "new", "free", "count", "lengths", "begin", "slots", "positions", "counts")])
def test_plan(lib, kw, status):
    d = dict(batch=3, size=16, table=A, stride=5, cached=A, new=A, free=A, capacity=9, count=A, tokens=20, lengths=A, begin=A,
             slots=A, positions=None, counts=A)
    d.update(kw)
    assert lib.hg_pages_plan(*(d[x] for x in ("batch", "size", "table", "stride", "cached", "new", "free", "capacity", "count",
                                              "tokens", "lengths", "begin", "slots", "positions", "counts")), None) == status


# -- the binding's own checks ------------------------------------------------------------------------------------------

def _raises(fn, what):
    with pytest.raises(ValueError) as e:
        fn()
    assert what in str(e.value), str(e.value)


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


@pytest.fixture
def pool(pages):
    c, s = _t(10, 4, 16, 128, dtype=torch.uint8), _t(10, 4, 1, dtype=torch.float32)
    pages8 = hg.Pages8(None, c, c, s, s, _shape(), torch.bfloat16)
    pages8.device = 0
    return pages8


def test_binding_create(lib):
    c, s = _t(10, 4, 32, 128, dtype=torch.float8_e4m3fn), _t(10, 4, 2, dtype=torch.float32)
    f = hg.hg_pages8_create
    _raises(lambda: f(c, c, s, s), "CUDA")
    _raises(lambda: f(c, c, s, s, torch.float32), "bfloat16 or float16")
    _raises(lambda: f(c, c[:9], s, s), "of one type")
    _raises(lambda: f(c, c.view(torch.uint8), s, s), "of one type")
    _raises(lambda: f(c.to(torch.bfloat16), c.to(torch.bfloat16), s, s), "float8_e4m3fn or uint8")
    _raises(lambda: f(c, c.transpose(1, 2).contiguous().transpose(1, 2), s, s), "same strides")
    _raises(lambda: f(c, c, s[:, :, :1], s), "scales must be")
    _raises(lambda: f(c, c, s, s.double()), "scales must be")


def test_binding_append_and_dequantize(pool):
    q, k, i, tab = _t(3, 8, 128), _t(3, 4, 128), torch.zeros(3, dtype=torch.int32), torch.zeros((2, 5), dtype=torch.int32)
    f = hg.hg_pages8_append
    _raises(lambda: f(pool, q, k, k, None, None, i, tab, i, q), "must be a CUDA tensor")
    _raises(lambda: f(pool, q, k, k, None, None, i, tab, i), "needs q_out")
    _raises(lambda: f(pool, q[:2], k, k, None, None, i, tab, i, q), "q is")
    _raises(lambda: f(pool, None, k.half(), k, None, None, i, tab, i), "k is")
    _raises(lambda: f(pool, None, _t(3, 128, 4).transpose(1, 2), k, None, None, i, tab, i), "dense channels")
    _raises(lambda: hg.hg_pages8_dequantize(pool, i, tab, None), "neither")
    _raises(lambda: hg.hg_pages8_dequantize(pool, i, tab, k.half()), "k_out is")
    _raises(lambda: hg.hg_pages8_dequantize(pool, i, tab, None, q), "v_out is")
    _raises(lambda: hg.hg_pages8_dequantize(pool, i, tab, k), "must be a CUDA tensor")
    _raises(lambda: hg._requests("f", i, tab[:1], 0), "page_table must be [2]")
    _raises(lambda: hg._requests("f", i.long(), tab, 0), "begin must be contiguous int32")
    _raises(lambda: hg._requests("f", i, tab, 0), "begin must be a CUDA tensor")


def test_binding_decode(pool):
    q, k, i = _t(3, 8, 128), _t(3, 4, 128), torch.zeros(3, dtype=torch.int32)
    _raises(lambda: hg.hg_pages8_decode_attention(pool, q, i, i, q, None, 0.0, i), "must be a CUDA tensor")
    _raises(lambda: hg.hg_pages8_decode_attention(pool, q.half(), i, i, q, None, 0.0, i), "q is")
    _raises(lambda: hg.hg_pages8_decode_step(pool, q, k[:2], k, None, None, i, i, q, None, 0.0, i), "must be a CUDA tensor")


def test_binding_plan(lib):
    i, tab = torch.zeros(3, dtype=torch.int32), torch.zeros((3, 5), dtype=torch.int32)
    f = hg.hg_pages_plan
    _raises(lambda: f(tab[:2], i, i, i, i, 16, i, i, i, None, i), "page_table must be [3]")
    _raises(lambda: f(i, i, i, i, i, 16, i, i, i, None, i), "page_table must be [3]")
    _raises(lambda: f(tab.long(), i, i, i, i, 16, i, i, i, None, i), "contiguous int32")
    _raises(lambda: f(tab, i, i, i, i, 16, i, i, i, None, i), "CUDA")


class _Tensor:
    """A tensor on a GPU that this machine may not have."""
    is_cuda = True

    def __init__(self, index, dtype, *shape):
        self.index, self.device, self.dtype, self.shape, self.nbytes = index, "cuda:%d" % index, dtype, shape, 99
        self.size = torch.Size(shape)

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return True

    def numel(self):
        return self.size.numel()

    def stride(self):
        return 128 * self.shape[1], 128, 1

    def data_ptr(self):
        return A


def test_one_device(monkeypatch):
    """A launch goes to the current device: tensors of another are refused, as are those of several."""
    rows, ints, floats = (_Tensor(1, d, *s) for d, s in ((torch.bfloat16, (3, 4, 128)), (torch.int32, (3,)), (torch.float32, (3, 4))))
    assert hg._rows_on("f", "x", rows, 3, 4, torch.bfloat16, 1) == (A, 512, 128)
    assert hg._ints_on("f", "x", ints, 3, 1) == A and hg._lse_on("f", floats, 3, 4, 1) == A
    assert hg._workspace_on("f", floats, 1) == (A, 99) and hg._lse_on("f", None, 3, 4, 1) is None
    what = "x is on cuda:1, the call's tensors are on cuda:0"
    _raises(lambda: hg._rows_on("f", "x", rows, 3, 4, torch.bfloat16, 0), what)
    _raises(lambda: hg._ints_on("f", "x", ints, 3, 0), what)
    _raises(lambda: hg._lse_on("f", floats, 3, 4, 0), "lse is on cuda:1")
    _raises(lambda: hg._workspace_on("f", floats, 0), "workspace is on cuda:1")

    class Turn:
        pointer, positions, table = 5, 1, floats
    assert hg._rotated_on("f", Turn, ints, 3, 1) == (5, A)
    _raises(lambda: hg._rotated_on("f", Turn, ints, 3, 0), "the rotation's table is on cuda:1")
    _raises(lambda: hg._rotated_on("f", Turn, None, 3, 1), "f: the rotation needs positions")
    monkeypatch.setattr(hg._types, "device", lambda: 0, raising=False)
    monkeypatch.setattr(hg._types, "stream", lambda device: 77 + device, raising=False)
    assert hg._stream_on("f", None, 0) == 77 and hg._stream_on("f", 5, 0) == 5
    _raises(lambda: hg._stream_on("f", None, 1), "the call's tensors are on cuda:1, the current device is cuda:0")


@pytest.mark.parametrize("shape", [(3, 64), (64, 3), (5, 3), (192,), (1, 15)])
def test_three_positions_have_the_calls_own_layout(shape):
    class Turn:
        pointer, positions, table = 0, 3, _Tensor(0, torch.float32, 9, 128)
    _raises(lambda: hg._rotated_on("f", Turn, torch.zeros(shape, dtype=torch.int32), 5, 0),
            "f: positions are %s, the call takes [3][5]" % list(shape))
