"""HeadGuard mixed-precision KV cache for GB300 -- Python binding of the C ABI.

Thin ctypes marshalling over ``libheadguard.so`` (declared in
``include/headguard.h``): every function here has the C entry point's name,
converts its arguments (torch tensors -> device pointers, streams -> handles)
and raises :class:`HGError` on a non-zero status (and ValueError, before the
call, when a tensor argument is not a dense CUDA tensor holding the bytes the
call reads or writes through it; the calls of the 16-bit caches also take
strided rows of dense channels).  All computation happens in
the library's CUDA kernels; there is no Python or CPU fallback, and importing
the compute functions without the built library raises.
"""
import ctypes
import os
import struct

from . import build as _build

__all__ = [
    "HGError", "Shape", "QuantConfig", "HeadRegions", "Cache",
    "HG_BASE_MINMAX_TOKEN", "HG_BASE_KIVI", "HG_BASE_AKVQ_HADAMARD",
    "HG_HEAD_QUANTIZED", "HG_HEAD_KEYS_ONLY", "HG_HEAD_PROTECTED",
    "hg_cache_layout", "hg_cache_create", "hg_cache_destroy", "hg_cache_head_regions",
    "hg_cache_appended", "hg_cache_reset_appended", "hg_quantize_kv", "hg_dequantize_kv",
    "hg_append_kv", "hg_decode_workspace_size", "hg_workspace_clear", "hg_workspace_status",
    "hg_check_bounded_wait", "hg_select_heads",
    "hg_decode_attention",
    "hg_decode_step", "hg_decode_attention_noalloc", "hg_cache_image_bits_per_elem",
    "hg_status_string",
    "HG_DTYPE_BF16", "HG_DTYPE_F16", "PageShape", "Pages", "Rotation",
    "hg_pages_create", "hg_pages_destroy", "hg_pages_append", "hg_pages_decode_workspace_size",
    "hg_pages_decode_attention", "hg_pages_decode_step", "hg_prompt_workspace_size", "hg_prompt_attention",
    "library", "library_path",
]

HG_BASE_MINMAX_TOKEN = 0
HG_BASE_KIVI = 1
HG_BASE_AKVQ_HADAMARD = 2
HG_HEAD_QUANTIZED = 0
HG_HEAD_KEYS_ONLY = 1
HG_HEAD_PROTECTED = 2
HG_DTYPE_BF16 = 0
HG_DTYPE_F16 = 1
NONE_OFFSET = (1 << 64) - 1

STATUS = {
    0: "HG_OK", 1: "HG_ERR_INVALID_ARG", 2: "HG_ERR_ALIGNMENT", 3: "HG_ERR_UNSUPPORTED",
    4: "HG_ERR_WORKSPACE_TOO_SMALL", 5: "HG_ERR_CAPACITY", 6: "HG_ERR_CUDA",
    7: "HG_ERR_ARENA_TOO_SMALL",
}


class HGError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__("%s: %s (%s)" % (where, STATUS.get(status, status),
                                          hg_status_string(status)))


class Shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "batch", "num_layers", "num_kv_heads", "num_q_heads", "head_dim", "seq_len",
        "img_start", "img_len", "max_new_tokens")]


class QuantConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "base", "bits", "keys_only", "kivi_group_tokens", "kivi_group_channels",
        "kivi_residual", "meta_bits", "salient_permille")]


class HeadRegions(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("head_class", "nq", "bf16_prefill",
                                                "bf16_capacity")] +
                [(n, ctypes.c_uint64) for n in ("kb", "vb", "kq", "kqm", "vq", "vqm", "kimg",
                                                 "kb_bstride", "kq_bstride", "kqm_bstride",
                                                 "vq_bstride", "vqm_bstride", "kimg_bstride",
                                                 "sal", "sal_bstride")] +
                [(n, ctypes.c_int32) for n in ("n_coded", "n_salient")])


class PageShape(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("dtype", "num_pages", "page_size", "num_kv_heads", "head_dim")] +
                [(n, ctypes.c_int64) for n in ("page_stride", "head_stride", "token_stride")])


class _Rotation(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("table_len", ctypes.c_int32), ("rot_dim", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("sections", ctypes.c_int32 * 3)]


_lib = None


def library_path():
    return _build.LIB


def library():
    """Load libheadguard.so (it must have been built by build.build())."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.LIB
    if not os.path.exists(path):
        raise RuntimeError("libheadguard.so is not built (%s); run "
                           "paper_2609_35800_gb300.build.build() first" % path)
    L = ctypes.CDLL(path)
    P, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    st = ctypes.c_int
    sigs = {
        "hg_cache_layout": ([P, P, P, ctypes.POINTER(sz)], st),
        "hg_cache_create": ([P, P, P, P, sz, ctypes.POINTER(P)], st),
        "hg_cache_destroy": ([P], None),
        "hg_cache_head_regions": ([P, i32, i32, ctypes.POINTER(HeadRegions)], st),
        "hg_cache_appended": ([P, i32], i32),
        "hg_cache_reset_appended": ([P], st),
        "hg_quantize_kv": ([P, i32, i32, P, P, P], st),
        "hg_dequantize_kv": ([P, i32, i32, P, P, i32, P], st),
        "hg_append_kv": ([P, i32, i32, P, P, P], st),
        "hg_decode_workspace_size": ([P, i32, ctypes.POINTER(sz)], st),
        "hg_workspace_clear": ([P, sz, P], st),
        "hg_workspace_status": ([P, ctypes.POINTER(ctypes.c_uint32), P], st),
        "hg_check_bounded_wait": ([P, ctypes.c_uint32, P], st),
        "hg_select_heads": ([P, P, i32, i32, i32, i32, P], st),
        "hg_decode_attention": ([P, i32, i32, P, P, ctypes.c_float, P, sz, P], st),
        "hg_decode_step": ([P, i32, i32, P, P, P, P, ctypes.c_float, P, sz, P], st),
        "hg_decode_attention_noalloc": ([P, i32, i32, P, P, ctypes.c_float, P], st),
        "hg_cache_image_bits_per_elem": ([P, ctypes.POINTER(ctypes.c_double)], st),
        "hg_pages_create": ([P, P, P, ctypes.POINTER(P)], st),
        "hg_pages_destroy": ([P], None),
        "hg_pages_append": ([P, i32, i32, P, P, P, P, P], st),
        "hg_pages_decode_workspace_size": ([P, i32, i32, ctypes.POINTER(sz)], st),
        "hg_pages_decode_attention": ([P, i32, i32, P, P, i32, P, P, ctypes.c_float, P, sz, P], st),
        "hg_pages_decode_step": ([P, i32, i32, P, P, P, P, i32, P, P, ctypes.c_float, P, sz, P], st),
        "hg_prompt_workspace_size": ([ctypes.POINTER(sz)], st),
        "hg_prompt_attention": ([i32, i32, i32, i32, P, P, P, P, i32, ctypes.c_float, P, sz, P], st),
        "hg_status_string": ([st], ctypes.c_char_p),
    }
    for name, (args, res) in sigs.items():
        f = getattr(L, name)
        f.argtypes = args
        f.restype = res
    _lib = L
    return L


def _check(status, where):
    if status != 0:
        raise HGError(status, where)


def _devs(where, *specs):
    """Addresses of device buffer arguments, each given as (x, nbytes, name).
    A torch tensor must be dense and hold at least `nbytes` bytes (the extent
    the library reads or writes through it) -- checked for every argument
    first -- and live on a CUDA device; an int is taken as a raw device
    address whose extent the caller vouches for, None as a null pointer
    (which the library rejects)."""
    out = []
    for x, nbytes, _ in specs:
        if x is None or isinstance(x, int):
            out.append(x)
        elif x.is_cuda and x.is_contiguous() and x.nbytes >= nbytes:
            out.append(x.data_ptr())
        else:
            _refuse(where, specs)
    return out


def _refuse(where, specs):
    """Raise for the first argument that _devs does not take."""
    for x, nbytes, name in specs:
        if x is None or isinstance(x, int):
            continue
        if not x.is_contiguous():
            raise ValueError("%s: %s must be contiguous" % (where, name))
        have = x.numel() * x.element_size()
        if have < nbytes:
            raise ValueError("%s: %s holds %d bytes, the call touches %d"
                             % (where, name, have, nbytes))
    for x, _, name in specs:
        if x is not None and not isinstance(x, int) and not x.is_cuda:
            raise ValueError("%s: %s must be a CUDA tensor" % (where, name))


def _extent(cache, *dims, elem=2):
    """Bytes of a dense [dims...][head_dim] array of `elem`-byte entries."""
    n = elem * cache.shape.head_dim
    for d in dims:
        n *= int(d) if d > 0 else 0
    return n


def _stream(stream):
    """cudaStream_t handle: a torch.cuda.Stream, an int, or None (current torch stream)."""
    if stream is None:
        import torch
        if torch.cuda.is_initialized():
            try:  # the handle alone, without a Stream object around it; not part of torch's public interface
                return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
            except AttributeError:
                pass
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _mask_bytes(mask):
    import numpy as np
    m = np.ascontiguousarray(np.asarray(mask, dtype=np.uint8))
    return m, m.ctypes.data_as(ctypes.c_void_p)


class Cache:
    """Owning handle of an hg_cache descriptor (the arena stays caller-owned)."""

    def __init__(self, handle, arena, shape, config, mask):
        self.handle = handle
        self.arena = arena
        self.shape = shape
        self.config = config
        self.mask = mask

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.hg_cache_destroy(self.handle)
            self.handle = None


def hg_status_string(status):
    return library().hg_status_string(int(status)).decode()


def hg_cache_layout(shape, config, head_mask):
    m, mp = _mask_bytes(head_mask)
    out = ctypes.c_size_t(0)
    _check(library().hg_cache_layout(ctypes.byref(shape), ctypes.byref(config), mp,
                                     ctypes.byref(out)), "hg_cache_layout")
    return out.value


def hg_cache_create(shape, config, head_mask, arena, arena_bytes=None):
    """Create the descriptor of a cache stored in `arena` (a device tensor or address)."""
    m, mp = _mask_bytes(head_mask)
    if arena_bytes is None:
        arena_bytes = arena.numel() * arena.element_size()
    h = ctypes.c_void_p()
    ap, = _devs("hg_cache_create", (arena, arena_bytes, "arena"))
    _check(library().hg_cache_create(ctypes.byref(shape), ctypes.byref(config), mp, ap,
                                     arena_bytes, ctypes.byref(h)), "hg_cache_create")
    return Cache(h, arena, shape, config, m.copy())


def hg_cache_destroy(cache):
    if cache.handle:
        library().hg_cache_destroy(cache.handle)
        cache.handle = None


def hg_cache_head_regions(cache, layer, head):
    out = HeadRegions()
    _check(library().hg_cache_head_regions(cache.handle, layer, head, ctypes.byref(out)),
           "hg_cache_head_regions")
    return out


def hg_cache_appended(cache, layer):
    return library().hg_cache_appended(cache.handle, layer)


def hg_cache_reset_appended(cache):
    _check(library().hg_cache_reset_appended(cache.handle), "hg_cache_reset_appended")


def hg_quantize_kv(cache, layer_begin, k_list, v_list, stream=None):
    n = len(k_list)
    if len(v_list) != n:
        raise ValueError("hg_quantize_kv: %d key and %d value tensors" % (n, len(v_list)))
    sh = cache.shape
    need = _extent(cache, sh.batch, sh.num_kv_heads, sh.seq_len)
    ptrs = []
    for x in (*k_list, *v_list):
        if x is None or isinstance(x, int):
            ptrs.append((x or 0) & 0xffffffffffffffff)  # any integer, as ctypes takes one for a pointer
        elif x.is_cuda and x.is_contiguous() and x.nbytes >= need:
            ptrs.append(x.data_ptr())
        else:
            _refuse("hg_quantize_kv", [(k, need, "k[%d]" % i) for i, k in enumerate(k_list)] +
                    [(v, need, "v[%d]" % i) for i, v in enumerate(v_list)])
    # two arrays of n pointers, as bytes
    _check(library().hg_quantize_kv(cache.handle, layer_begin, n, struct.pack("%dQ" % n, *ptrs[:n]),
                                    struct.pack("%dQ" % n, *ptrs[n:]), _stream(stream)), "hg_quantize_kv")


def hg_dequantize_kv(cache, layer_begin, layer_count, k_out, v_out, out_fp32, stream=None):
    """Reconstruct layers [layer_begin, +layer_count) into k_out / v_out
    [layer_count][B][H_kv][T + appended][128] (fp32 or BF16)."""
    sh = cache.shape
    t = sh.seq_len + max(hg_cache_appended(cache, layer_begin), 0)
    need = _extent(cache, layer_count, sh.batch, sh.num_kv_heads, t, elem=4 if out_fp32 else 2)
    kp, vp = _devs("hg_dequantize_kv", (k_out, need, "k_out"), (v_out, need, "v_out"))
    _check(library().hg_dequantize_kv(cache.handle, layer_begin, layer_count, kp, vp,
                                      1 if out_fp32 else 0, _stream(stream)), "hg_dequantize_kv")


def hg_append_kv(cache, layer_begin, layer_count, k_new, v_new, stream=None):
    sh = cache.shape
    need = _extent(cache, layer_count, sh.batch, sh.num_kv_heads)
    kp, vp = _devs("hg_append_kv", (k_new, need, "k_new"), (v_new, need, "v_new"))
    _check(library().hg_append_kv(cache.handle, layer_begin, layer_count, kp, vp,
                                  _stream(stream)), "hg_append_kv")


def hg_decode_workspace_size(cache, layer_count):
    out = ctypes.c_size_t(0)
    _check(library().hg_decode_workspace_size(cache.handle, layer_count, ctypes.byref(out)),
           "hg_decode_workspace_size")
    return out.value


def hg_workspace_clear(workspace, nbytes=None, stream=None):
    """Zero a decode workspace; workspace None clears the status word of the
    allocation-free entry point's scratch on the current device."""
    if workspace is None:
        nbytes = 0
    elif nbytes is None:
        nbytes = workspace.numel() * workspace.element_size()
    wp, = _devs("hg_workspace_clear", (workspace, nbytes, "workspace"))
    _check(library().hg_workspace_clear(wp, nbytes, _stream(stream)), "hg_workspace_clear")


def hg_workspace_status(workspace, stream=None):
    """Status word of a decode workspace (waits for the stream); 0 = healthy.
    workspace None: the status word of the allocation-free entry point's scratch
    on the current device."""
    out = ctypes.c_uint32(0)
    wp, = _devs("hg_workspace_status", (workspace, 4, "workspace"))
    _check(library().hg_workspace_status(wp, ctypes.byref(out), _stream(stream)),
           "hg_workspace_status")
    return out.value


def hg_check_bounded_wait(word, rounds, stream=None):
    """Run the bounded-wait self-check into the device word `word` (see the header)."""
    wp, = _devs("hg_check_bounded_wait", (word, 4, "word"))
    _check(library().hg_check_bounded_wait(wp, int(rounds), _stream(stream)),
           "hg_check_bounded_wait")


def hg_select_heads(g_scores, o_scores, num_layers, num_q_heads, num_kv_heads, k=-1):
    """Protected-head mask (numpy uint8 [num_layers][num_kv_heads]) from host
    per-query-head scores [num_layers][num_q_heads] (see the header)."""
    import numpy as np
    g = np.ascontiguousarray(np.asarray(g_scores, dtype=np.float32))
    o = np.ascontiguousarray(np.asarray(o_scores, dtype=np.float32))
    mask = np.zeros((num_layers, num_kv_heads), dtype=np.uint8)
    _check(library().hg_select_heads(g.ctypes.data_as(ctypes.c_void_p), o.ctypes.data_as(ctypes.c_void_p),
                                     num_layers, num_q_heads, num_kv_heads, int(k),
                                     mask.ctypes.data_as(ctypes.c_void_p)), "hg_select_heads")
    return mask


def hg_decode_attention(cache, layer_begin, layer_count, q, out, softmax_scale, workspace,
                        workspace_bytes=None, stream=None):
    if workspace_bytes is None:
        workspace_bytes = workspace.nbytes
    sh = cache.shape
    need = _extent(cache, layer_count, sh.batch, sh.num_q_heads)
    qp, op, wp = _devs("hg_decode_attention", (q, need, "q"), (out, need, "out"),
                       (workspace, workspace_bytes, "workspace"))
    _check(library().hg_decode_attention(cache.handle, layer_begin, layer_count, qp, op,
                                         float(softmax_scale), wp, workspace_bytes,
                                         _stream(stream)), "hg_decode_attention")


def hg_decode_step(cache, layer_begin, layer_count, q, k_new, v_new, out, softmax_scale, workspace,
                   workspace_bytes=None, stream=None):
    """Append the step's K/V and run decode attention including it, in one launch."""
    if workspace_bytes is None:
        workspace_bytes = workspace.nbytes
    sh = cache.shape
    per = _extent(cache, layer_count, sh.batch)
    nq, nkv = per * sh.num_q_heads, per * sh.num_kv_heads
    qp, kp, vp, op, wp = _devs("hg_decode_step", (q, nq, "q"), (k_new, nkv, "k_new"),
                               (v_new, nkv, "v_new"), (out, nq, "out"),
                               (workspace, workspace_bytes, "workspace"))
    _check(library().hg_decode_step(cache.handle, layer_begin, layer_count, qp, kp, vp, op,
                                    float(softmax_scale), wp, workspace_bytes, _stream(stream)),
           "hg_decode_step")


def hg_decode_attention_noalloc(cache, layer_begin, layer_count, q, out, softmax_scale,
                                stream=None):
    """Decode attention with the library's static 32 MiB scratch as workspace (no allocation)."""
    sh = cache.shape
    need = _extent(cache, layer_count, sh.batch, sh.num_q_heads)
    qp, op = _devs("hg_decode_attention_noalloc", (q, need, "q"), (out, need, "out"))
    _check(library().hg_decode_attention_noalloc(cache.handle, layer_begin, layer_count, qp, op,
                                                 float(softmax_scale), _stream(stream)),
           "hg_decode_attention_noalloc")


def hg_cache_image_bits_per_elem(cache):
    out = ctypes.c_double(0)
    _check(library().hg_cache_image_bits_per_elem(cache.handle, ctypes.byref(out)),
           "hg_cache_image_bits_per_elem")
    return out.value


# ---------------------------------------------------------------------------
# Caches that stay 16-bit: page pools, append, paged decode, prompts
# ---------------------------------------------------------------------------


class _Types:
    """The torch types that the calls below compare with, looked up at the first call (the package itself can be
    imported without torch)."""

    def __getattr__(self, name):
        import torch
        self.code = {torch.bfloat16: HG_DTYPE_BF16, torch.float16: HG_DTYPE_F16}
        self.int32, self.float32 = torch.int32, torch.float32
        return self.__dict__[name]


_types = _Types()
_pack18, _pack12 = struct.Struct("=18q").pack, struct.Struct("=12q").pack  # hg_append_io, hg_attention_io


class Pages:
    """Owning handle of an hg_pages descriptor (the pool's tensors stay the caller's)."""

    def __init__(self, handle, k_pages, v_pages, shape):
        self.handle = handle
        self.k_pages = k_pages
        self.v_pages = v_pages
        self.shape = shape
        self.dtype = k_pages.dtype

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.hg_pages_destroy(self.handle)
            self.handle = None


class Rotation:
    """Position rotation of queries and keys: `table` float32 [positions][rot_dim] on the GPU, cosines of the
    rot_dim / 2 pairs, then sines; `sections`: the pairs that turn by each of a token's three positions (None: one
    position a token).  A call's positions are then [3][tokens], else [tokens].  See hg_rotation."""

    def __init__(self, table, interleaved=False, sections=None):
        import torch
        if table.dim() != 2 or table.dtype != torch.float32 or not table.is_contiguous():
            raise ValueError("Rotation: table must be a contiguous float32 [positions][rot_dim]")
        if not table.is_cuda:
            raise ValueError("Rotation: table must be a CUDA tensor")
        self.table = table
        self.positions = 3 if sections is not None and any(sections) else 1  # (all 0: one, as in hg_rotation)
        self.raw = _Rotation(table.data_ptr(), table.shape[0], table.shape[1], int(interleaved),
                             (ctypes.c_int32 * 3)(*(sections or (0, 0, 0))))
        self.pointer = ctypes.addressof(self.raw)


def _rows(where, name, x, tokens, heads, dtype):
    """(address, token stride, head stride) of a tensor seen as [tokens][heads][128] with dense channels."""
    if x.dtype is dtype and x.shape == (tokens, heads, 128) and x.is_cuda:
        ts, hs, cs = x.stride()
        if cs == 1:
            # a stride that is never taken may be anything in torch
            return x.data_ptr(), ts if tokens > 1 else 0, hs if heads > 1 else 0
    if x.shape != (tokens, heads, 128) or x.dtype != dtype:
        raise ValueError("%s: %s is %s %s, the call takes %s [%d][%d][128]"
                         % (where, name, x.dtype, list(x.shape), dtype, tokens, heads))
    if x.stride(2) != 1:
        raise ValueError("%s: %s must have dense channels" % (where, name))
    raise ValueError("%s: %s must be a CUDA tensor" % (where, name))


_NO_ROWS = (0, 0, 0)
_Int = ctypes.c_int32


def _ints(where, name, x, need, cuda=True):
    """Address of a dense int32 tensor of at least `need` entries."""
    if x.dtype is _types.int32 and x.is_contiguous() and x.numel() >= need and x.is_cuda is cuda:
        return x.data_ptr()
    if x.dtype != _types.int32 or not x.is_contiguous():
        raise ValueError("%s: %s must be contiguous int32" % (where, name))
    if x.numel() < need:
        raise ValueError("%s: %s holds %d entries, the call reads %d" % (where, name, x.numel(), need))
    raise ValueError("%s: %s must be a %s tensor" % (where, name, "CUDA" if cuda else "CPU"))


def _lse(where, x, tokens, heads):
    if x is None:
        return None
    if x.dtype is _types.float32 and x.shape == (tokens, heads) and x.is_contiguous() and x.is_cuda:
        return x.data_ptr()
    if x.dtype != _types.float32 or x.shape != (tokens, heads) or not x.is_contiguous():
        raise ValueError("%s: lse must be contiguous float32 [%d][%d]" % (where, tokens, heads))
    raise ValueError("%s: lse must be a CUDA tensor" % where)


def _rotated_by(where, rotation, positions, tokens):
    if rotation is None:
        return None, None
    parts = rotation.positions
    if parts > 1 and positions.shape != (parts, tokens) and positions.shape != (parts * tokens,):
        # (their distance is the call's tokens: a longer row would be read from the wrong places)
        raise ValueError("%s: positions are %s, the call takes [%d][%d]" % (where, list(positions.shape), parts, tokens))
    return rotation.pointer, _ints(where, "positions", positions, parts * tokens)


def hg_pages_create(k_pages, v_pages):
    """Descriptor of the page pool whose keys and values are these tensors, each seen as
    [pages][kv heads][page size][128] (any strides: pages that lie [tokens][heads] are passed transposed)."""
    if k_pages.dim() != 4 or k_pages.shape != v_pages.shape or k_pages.dtype != v_pages.dtype:
        raise ValueError("hg_pages_create: k_pages and v_pages must be [pages][heads][tokens][128] of one type")
    if k_pages.dtype not in _types.code:
        raise ValueError("hg_pages_create: pages must be bfloat16 or float16")
    n, heads, size, dim = k_pages.shape
    # the stride of an axis of length 1 is never taken: a dense one stands for it
    strides = [tuple(s if d > 1 else dim for s, d in zip(x.stride(), x.shape)) for x in (k_pages, v_pages)]
    if strides[0] != strides[1] or k_pages.stride(3) != 1:
        raise ValueError("hg_pages_create: k_pages and v_pages must have the same strides and dense channels")
    if not (k_pages.is_cuda and v_pages.is_cuda):
        raise ValueError("hg_pages_create: k_pages and v_pages must be CUDA tensors")
    shape = PageShape(_types.code[k_pages.dtype], n, size, heads, dim, *strides[0][:3])
    h = ctypes.c_void_p()
    _check(library().hg_pages_create(ctypes.byref(shape), k_pages.data_ptr(), v_pages.data_ptr(), ctypes.byref(h)),
           "hg_pages_create")
    return Pages(h, k_pages, v_pages, shape)


def hg_pages_destroy(pages):
    if pages.handle:
        library().hg_pages_destroy(pages.handle)
        pages.handle = None


def hg_pages_append(pages, q, k, v, rotation, positions, slots, q_out=None, k_out=None, v_out=None, stream=None):
    """Rotate q and k ([tokens][heads][128], any token and head strides; q None: no queries) and store k and v at
    `slots` (int32, page * page size + place; negative: nowhere).  The rotated rows also go to q_out and, where
    given, k_out; v to v_out."""
    w, d = "hg_pages_append", pages.dtype
    n, heads, hq = k.shape[0], pages.shape.num_kv_heads, 0 if q is None else q.shape[1]
    if q is not None and q_out is None:
        raise ValueError("hg_pages_append: q needs q_out")
    io = _pack18(*(_rows(w, "q", q, n, hq, d) if hq else _NO_ROWS), *_rows(w, "k", k, n, heads, d),
                     *_rows(w, "v", v, n, heads, d), *(_rows(w, "q_out", q_out, n, hq, d) if hq else _NO_ROWS),
                     *(_NO_ROWS if k_out is None else _rows(w, "k_out", k_out, n, heads, d)),
                     *(_NO_ROWS if v_out is None else _rows(w, "v_out", v_out, n, heads, d)))
    rp, pp = _rotated_by(w, rotation, positions, n)
    _check(library().hg_pages_append(pages.handle, n, hq, io, rp, pp, _ints(w, "slots", slots, n), _stream(stream)), w)


def hg_pages_decode_workspace_size(pages, batch, num_q_heads):
    out = ctypes.c_size_t(0)
    _check(library().hg_pages_decode_workspace_size(pages.handle, batch, num_q_heads, ctypes.byref(out)),
           "hg_pages_decode_workspace_size")
    return out.value


def _decode_table(where, page_table, lengths, batch):
    if page_table.dim() != 2 or page_table.shape[0] < batch:
        raise ValueError("%s: page_table must be [%d][pages]" % (where, batch))
    per = page_table.shape[1]
    return _ints(where, "page_table", page_table, batch * per), per, _ints(where, "lengths", lengths, batch)


def _workspace(where, x):
    if x is None or isinstance(x, int):
        raise ValueError("%s: workspace must be a tensor" % where)
    if x.is_cuda and x.is_contiguous():
        return x.data_ptr(), x.nbytes
    _refuse(where, [(x, 0, "workspace")])


def hg_pages_decode_attention(pages, q, page_table, lengths, out, lse, softmax_scale, workspace, stream=None):
    """Attention of one token per request (q, out [batch][heads][128]) over the first lengths[b] tokens of its pages
    page_table[b]; lse float32 [batch][heads] or None."""
    w, d = "hg_pages_decode_attention", pages.dtype
    n, hq = q.shape[0], q.shape[1]
    io = _pack12(*_rows(w, "q", q, n, hq, d), 0, 0, 0, 0, 0, 0, *_rows(w, "out", out, n, hq, d))
    tp, ts, lp = _decode_table(w, page_table, lengths, n)
    _check(library().hg_pages_decode_attention(pages.handle, n, hq, io, tp, ts, lp, _lse(w, lse, n, hq),
                                               softmax_scale, *_workspace(w, workspace), _stream(stream)), w)


def hg_pages_decode_step(pages, q, k, v, rotation, positions, page_table, lengths, out, lse, softmax_scale, workspace,
                         stream=None):
    """One decode step: q and the new token's k rotated, k and v stored as token lengths[b] - 1 of request b, attention
    over its lengths[b] tokens."""
    w, d = "hg_pages_decode_step", pages.dtype
    n, hq, heads = q.shape[0], q.shape[1], pages.shape.num_kv_heads
    io = _pack12(*_rows(w, "q", q, n, hq, d), *_rows(w, "k", k, n, heads, d),
                     *_rows(w, "v", v, n, heads, d), *_rows(w, "out", out, n, hq, d))
    rp, pp = _rotated_by(w, rotation, positions, n)
    tp, ts, lp = _decode_table(w, page_table, lengths, n)
    _check(library().hg_pages_decode_step(pages.handle, n, hq, io, rp, pp, tp, ts, lp, _lse(w, lse, n, hq),
                                          softmax_scale, *_workspace(w, workspace), _stream(stream)), w)


def hg_prompt_workspace_size():
    out = ctypes.c_size_t(0)
    _check(library().hg_prompt_workspace_size(ctypes.byref(out)), "hg_prompt_workspace_size")
    return out.value


def hg_prompt_attention(q, k, v, q_begin, k_begin, out, lse, causal, softmax_scale, workspace, stream=None):
    """Attention of packed prompts: q, out [tokens][heads][128], k, v [keys][kv heads][128] (any token and head
    strides); prompt i has the rows q_begin[i]..q_begin[i + 1] and the keys k_begin[i]..k_begin[i + 1] (CPU int32
    tensors [prompts + 1]); lse float32 [tokens][heads] or None."""
    w, d = "hg_prompt_attention", q.dtype
    code = _types.code.get(d)
    if code is None:
        raise ValueError("%s: q must be bfloat16 or float16" % w)
    n, hq, _ = q.shape
    nk, heads, _ = k.shape
    count = q_begin.numel() - 1
    io = _pack12(*_rows(w, "q", q, n, hq, d), *_rows(w, "k", k, nk, heads, d),
                     *_rows(w, "v", v, nk, heads, d), *_rows(w, "out", out, n, hq, d))
    qb, kb = _ints(w, "q_begin", q_begin, 1, False), _ints(w, "k_begin", k_begin, count + 1, False)
    q_end, k_end = _Int.from_address(qb + 4 * count).value, _Int.from_address(kb + 4 * count).value
    if q_end > n or k_end > nk:
        raise ValueError("%s: the prompts end at %d and %d, q and k hold %d and %d rows" % (w, q_end, k_end, n, nk))
    _check(library().hg_prompt_attention(code, count, hq, heads, io, qb, kb, _lse(w, lse, n, hq), 1 if causal else 0,
                                         softmax_scale, *_workspace(w, workspace), _stream(stream)), w)
