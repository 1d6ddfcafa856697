"""ctypes binding of the 4-bit key-value cache (the C ABI in include/treespark_kv.h).

The steps of a target's pass over draft trees that lie between ts_tree_mask and ts_verify: pages and
slots for the trees' rows (plan), their keys and values into the cache (append), attention over context
and tree (attention), and, after the verdict, the accepted rows kept (accept); read gives rows of the cache
back as numbers.  Argument marshalling only, as in binding.py: tensors are int32, float32, bfloat16 or
uint8 on one GPU, and a call that does not fit raises before anything is launched.

    pool = kv.Pool(num_pages, R, max_blocks, page_size)
    cache = kv.empty_cache(layers, num_pages, page_size, heads, head_dim)
    ...                                                     # each round:
    slot, granted = kv.plan(pool, length, n, cap)           # n: nodes of each request's tree
    for layer in range(layers):
        kv.append(cache, k, v, slot, layer=layer)           # k, v [R * cap][heads][head_dim]
        out, _ = kv.attention(cache, q, length, granted, pool.table, mask=mask, layer=layer)
    length = kv.accept(cache, length, granted, pool.table, path_nodes, path_len)

A call runs on the tensors' device, on its current stream or the given one.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding
from .binding import TS_BF16, TS_F32, TS_MAX_D, TreeSparkError, _check  # noqa: F401

EXPORTED = ("ts_kv_block_bytes", "ts_kv_plan", "ts_kv_append", "ts_kv_read", "ts_kv_attention_workspace_size",
            "ts_kv_attention", "ts_kv_accept")
PAGE_SIZES = (16, 32, 64, 128, 256)
HEAD_DIMS = (64, 128, 256)


class CacheStruct(ctypes.Structure):
    """ts_kv_cache."""
    _fields_ = [("pages", ctypes.c_void_p), ("layer_stride", ctypes.c_int64), ("page_stride", ctypes.c_int64),
                ("layers", ctypes.c_int32), ("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


_lib = None


def lib():
    """The HIP library with the cache's entry points declared; raises if it has not been built."""
    global _lib
    if _lib is None:
        L = binding.lib()
        P, I32, I64, SZ, F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
        L.ts_kv_block_bytes.argtypes = [I32, I32]
        L.ts_kv_block_bytes.restype = SZ
        L.ts_kv_plan.argtypes = [P, P, I32, I32, I32, I32, I32, P, P, P, P, P, P, P]
        L.ts_kv_plan.restype = I32
        L.ts_kv_append.argtypes = [P, I32, P, P, I32, I64, I64, P, I32, P]
        L.ts_kv_append.restype = I32
        L.ts_kv_read.argtypes = [P, I32, I32, P, I32, P, P, I32, P]
        L.ts_kv_read.restype = I32
        L.ts_kv_attention_workspace_size.argtypes = [P, I32, I32, I32, I32]
        L.ts_kv_attention_workspace_size.restype = SZ
        L.ts_kv_attention.argtypes = [P, I32, P, I32, I64, I32, P, P, I32, I32, P, I32, P, F, P, P, P, SZ, P]
        L.ts_kv_attention.restype = I32
        L.ts_kv_accept.argtypes = [P, P, P, I32, P, I32, P, P, P, P]
        L.ts_kv_accept.restype = I32
        _lib = L
    return _lib


_I32 = torch.int32


def _int32(name, t, shape, device):
    """The address of a contiguous int32 tensor of that shape on that GPU (host tensors are on device -1)."""
    if t.dtype is _I32 and t.shape == shape and t.get_device() == device >= 0 and t.is_contiguous():
        return t.data_ptr()
    where = f"cuda:{device}" if device >= 0 else "a GPU"
    raise ValueError(f"{name}: a contiguous int32 tensor {list(shape)} on {where} is needed, got {t.dtype} "
                     f"{list(t.shape)} on {t.device}")


def _public_stream(device):
    return torch.cuda.current_stream(device).cuda_stream


# the handle of a device's current stream; the short way takes 0.1 us of the 1.2 us of the public one
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _public_stream)


def _call(function, device, *args):
    """Calls a C entry on the device's current stream, with the device current."""
    handle = _current_stream(device)
    if torch.cuda.current_device() == device:
        rc = function(*args, handle)
    else:
        with torch.cuda.device(device):
            rc = function(*args, handle)
    if rc:
        _check(rc)


def _on(stream, device):
    """The given stream as the current one: what a call allocates or fills is then in that stream's order too."""
    if stream.device_index != device:
        raise ValueError(f"the stream is of cuda:{stream.device_index}, the tensors are on cuda:{device}")
    return torch.cuda.stream(stream)


class Cache:
    """A cache over pages [layers][num_pages][bytes], a uint8 GPU tensor with contiguous pages of at least
    heads * block_bytes(page_size, head_dim) bytes (layers and pages may have any strides that are multiples
    of 16)."""

    def __init__(self, pages, page_size, heads, head_dim):
        if pages.dim() != 3 or pages.dtype is not torch.uint8 or not pages.is_cuda or pages.stride(2) != 1:
            raise ValueError("pages: a uint8 tensor [layers][num_pages][bytes] on a GPU is needed")
        block = block_bytes(page_size, head_dim)
        if pages.shape[2] < heads * block:
            raise ValueError(f"pages of {pages.shape[2]} bytes hold no {heads} heads of {block}")
        self.pages, self.device = pages, pages.get_device()
        self.struct = CacheStruct(pages.data_ptr(), pages.stride(0), pages.stride(1), pages.shape[0], pages.shape[1],
                                  page_size, heads, head_dim)
        self._ref = ctypes.byref(self.struct)
        self._row = (heads, head_dim)
        self._sizes = {}  # workspace bytes by sizes

    @property
    def layers(self):
        return self.struct.layers

    @property
    def num_pages(self):
        return self.struct.num_pages

    @property
    def page_size(self):
        return self.struct.page_size

    @property
    def heads(self):
        return self.struct.heads

    @property
    def head_dim(self):
        return self.struct.head_dim

    def ref(self):
        return self._ref


def block_bytes(page_size, head_dim):
    """ts_kv_block_bytes; raises for sizes a cache cannot have."""
    n = lib().ts_kv_block_bytes(page_size, head_dim)
    if n == 0:
        raise ValueError(f"page_size {page_size} of {PAGE_SIZES} and head_dim {head_dim} of {HEAD_DIMS} are needed")
    return n


def empty_cache(layers, num_pages, page_size, heads, head_dim, device="cuda"):
    """A Cache in new memory."""
    pages = torch.zeros((layers, num_pages, heads * block_bytes(page_size, head_dim)), dtype=torch.uint8, device=device)
    return Cache(pages, page_size, heads, head_dim)


class Pool:
    """The free pages and the requests' block tables: free_pages [num_pages], free_count [1], held [R], table
    [R][max_blocks], int32 on one GPU (given, or new with every page free)."""

    def __init__(self, num_pages, R, max_blocks, page_size, device="cuda", free_pages=None, free_count=None, held=None,
                 table=None):
        given = (free_pages, free_count, held, table)
        if all(t is None for t in given):
            free_pages = torch.arange(num_pages, dtype=torch.int32, device=device)
            free_count = torch.full((1,), num_pages, dtype=torch.int32, device=device)
            held = torch.zeros((R,), dtype=torch.int32, device=device)
            table = torch.full((R, max_blocks), -1, dtype=torch.int32, device=device)
        elif any(t is None for t in given):
            raise ValueError("free_pages, free_count, held and table are given together")
        self.num_pages, self.R, self.max_blocks, self.page_size = num_pages, R, max_blocks, page_size
        self._tensors = free_pages, free_count, held, table
        self.device = d = free_pages.get_device()
        self._addr = (_int32("free_pages", free_pages, (num_pages,), d), _int32("free_count", free_count, (1,), d),
                      _int32("held", held, (R,), d), _int32("table", table, (R, max_blocks), d))

    # read-only: a plan goes by the tensors that the pool was made with
    free_pages = property(lambda self: self._tensors[0])
    free_count = property(lambda self: self._tensors[1])
    held = property(lambda self: self._tensors[2])
    table = property(lambda self: self._tensors[3])


def plan(pool: Pool, length, n, cap, slots=True, out=None, stream=None):
    """ts_kv_plan: pages for the rows 0..n[q] behind length[q] tokens of every request.  Returns (slot [R][cap],
    granted [R]), int32; slot is None with slots=False (only the pages).  out = (slot, granted) reuses tensors, a slot of
    None there as with slots=False."""
    if stream is not None:
        with _on(stream, pool.device):
            return plan(pool, length, n, cap, slots, out)
    R, d = pool.R, pool.device
    a_len, a_n = _int32("length", length, (R,), d), _int32("n", n, (R,), d)
    if out is None:
        slot = n.new_empty((R, cap)) if slots else None
        granted = n.new_empty((R,))
    else:
        slot, granted = out if slots else (None, out[1])
        _int32("granted", granted, (R,), d)
        if slot is not None:
            _int32("slot", slot, (R, cap), d)
    free_pages, free_count, held, table = pool._addr
    _call(lib().ts_kv_plan, d, a_len, a_n, R, cap, pool.page_size, pool.num_pages, pool.max_blocks, free_pages,
          free_count, held, table, slot.data_ptr() if slot is not None else None, granted.data_ptr())
    return slot, granted


def _rows(name, t, cache):
    """Row stride of keys or values [rows][heads][head_dim] (or [R][cap][heads][head_dim])."""
    sh, st = t.shape, t.stride()
    heads, D = cache._row
    if len(sh) not in (3, 4) or sh[-1] != D or sh[-2] != heads or t.get_device() != cache.device:
        raise ValueError(f"{name}: [rows][{heads}][{D}] on cuda:{cache.device} is needed, got {list(sh)} on {t.device}")
    if st[-1] != 1 or (st[-2] != D and heads > 1):
        raise ValueError(f"{name}: the heads of a row must be contiguous, got strides {st}")
    return _row_stride(name, sh[:-2], st, heads * D)


def _row_stride(name, sh, st, width):
    """Elements from a row to the next of rows laid out as sh, [rows] or [R][cap]."""
    if len(sh) == 2 and sh[1] > 1:
        if sh[0] > 1 and st[0] != st[1] * sh[1]:
            raise ValueError(f"{name}: rows must be evenly spaced, got strides {st}")
        return st[1]
    return st[0] if sh[0] > 1 else width


def append(cache: Cache, k, v, slot, layer=0, stream=None):
    """ts_kv_append: rows' keys and values k, v [rows][heads][head_dim] (float32 or bfloat16; rows may be apart,
    as in a projection's output that holds both) into a layer of the cache, at slot (int32, one per row)."""
    if stream is not None:
        with _on(stream, cache.device):
            return append(cache, k, v, slot, layer)
    s_k, s_v = _rows("k", k, cache), _rows("v", v, cache)
    rows = slot.numel()
    if k.dtype is not v.dtype or k.shape != v.shape:
        raise ValueError("k and v must have one dtype and as many rows")
    if k.numel() != rows * cache._row[0] * cache._row[1]:
        raise ValueError(f"{rows} slots for keys {list(k.shape)}")
    _call(lib().ts_kv_append, cache.device, cache._ref, layer, k.data_ptr(), v.data_ptr(), binding._dtype_code(k),
          s_k, s_v, _int32("slot", slot, slot.shape, cache.device), rows)


def read(cache: Cache, slot, layer=0, layers=None, dtype=None, out=None, stream=None):
    """ts_kv_read: the rows at slot as (k, v) [layers][rows][heads][head_dim], of `layers` layers from `layer` on
    (None: all that follow).  out = (k, v) reuses tensors, either of which may be None; without it rows that have no
    slot are zero.  dtype: float32 or bfloat16 (the default)."""
    if stream is not None:
        with _on(stream, cache.device):
            return read(cache, slot, layer, layers, dtype, out)
    layers = cache.struct.layers - layer if layers is None else layers
    rows, d = slot.numel(), cache.device
    shape = (layers, rows) + cache._row
    a_slot = _int32("slot", slot, slot.shape, d)
    if out is None:
        out = tuple(torch.zeros(shape, dtype=dtype or torch.bfloat16, device=slot.device) for _ in range(2))
    k, v = out
    one = k if k is not None else v
    if one is None:
        return out
    for t in out:
        if t is not None and (t.shape != shape or t.get_device() != d or not t.is_contiguous() or t.dtype is not one.dtype):
            raise ValueError(f"out: contiguous tensors {list(shape)} of one dtype on cuda:{d} are needed")
    _call(lib().ts_kv_read, d, cache._ref, layer, layers, a_slot, rows, k.data_ptr() if k is not None else None,
          v.data_ptr() if v is not None else None, binding._dtype_code(one))
    return k, v


def attention_workspace_size(cache: Cache, R, cap, q_heads, dtype):
    """ts_kv_attention_workspace_size for queries of a torch dtype."""
    key = R, cap, q_heads, dtype
    size = cache._sizes.get(key)
    if size is None:
        with torch.cuda.device(cache.device):
            size = lib().ts_kv_attention_workspace_size(cache._ref, R, cap, q_heads,
                                                        TS_BF16 if dtype is torch.bfloat16 else TS_F32)
        cache._sizes[key] = size
    return size


def attention(cache: Cache, q, length, n, table, mask=None, scale=None, layer=0, out=None, lse=None, workspace=None,
              stream=None):
    """ts_kv_attention.  q [R][cap][q_heads][head_dim] (float32 or bfloat16; rows may be apart), length and n [R], table
    [R][max_blocks], mask the [R][cap][W] words of binding.tree_mask or None for chains (causal).  scale: head_dim
    ** -0.5 by default.  Returns (out, lse): out like q, contiguous; lse float32 [R][cap][q_heads] if given, else None.
    Rows past n[q] of given tensors are left as they were; those of a new out are zero."""
    if stream is not None:
        with _on(stream, cache.device):
            return attention(cache, q, length, n, table, mask, scale, layer, out, lse, workspace)
    d, sh, st = cache.device, q.shape, q.stride()
    if len(sh) != 4 or sh[3] != cache._row[1] or q.get_device() != d:
        raise ValueError(f"q: [R][cap][q_heads][{cache._row[1]}] on cuda:{d} is needed, got {list(sh)} on {q.device}")
    R, cap, q_heads, D = sh
    if st[3] != 1 or (st[2] != D and q_heads > 1):
        raise ValueError(f"q: the heads of a row must be contiguous, got strides {st}")
    stride = _row_stride("q", sh[:2], st, q_heads * D)
    dtype = binding._dtype_code(q)
    if table.dim() != 2:
        raise ValueError("table: [R][max_blocks] is needed")
    max_blocks = table.shape[1]
    if out is None:
        out = torch.zeros(sh, dtype=q.dtype, device=q.device)
    elif out.shape != sh or out.dtype is not q.dtype or out.get_device() != d or not out.is_contiguous():
        raise ValueError(f"out: a contiguous {q.dtype} tensor {list(sh)} on cuda:{d} is needed")
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != sh[:3] or lse.get_device() != d
                            or not lse.is_contiguous()):
        raise ValueError(f"lse: a contiguous float32 tensor {list(sh[:3])} on cuda:{d} is needed")
    if workspace is None:
        workspace = torch.empty(max(attention_workspace_size(cache, R, cap, q_heads, q.dtype), 1), dtype=torch.uint8,
                                device=q.device)
    elif workspace.get_device() != d or workspace.dtype is not torch.uint8 or not workspace.is_contiguous():
        raise ValueError(f"workspace: a contiguous uint8 tensor on cuda:{d} is needed")
    _call(lib().ts_kv_attention, d, cache._ref, layer, q.data_ptr(), dtype, stride, q_heads,
          _int32("length", length, (R,), d),
          _int32("n", n, (R,), d), R, cap, _int32("table", table, (R, max_blocks), d), max_blocks,
          None if mask is None else _int32("mask", mask, (R, cap, (cap + 31) // 32), d),
          D ** -0.5 if scale is None else scale, out.data_ptr(), lse.data_ptr() if lse is not None else None,
          workspace.data_ptr(), workspace.numel())
    return out, lse


def accept(cache: Cache, length, n, table, path_nodes, path_len, new_length=None, stream=None):
    """ts_kv_accept: the accepted paths' rows, in every layer, moved behind the contexts.  path_nodes [R][16] and
    path_len [R] as binding.verify returns them (numpy arrays are copied to the GPU) or int32 GPU tensors.  Returns
    the new lengths [R]."""
    if stream is not None:
        with _on(stream, cache.device):
            return accept(cache, length, n, table, path_nodes, path_len, new_length)
    d = cache.device
    if table.dim() != 2:
        raise ValueError("table: [R][max_blocks] is needed")
    R, max_blocks = table.shape
    if not isinstance(path_nodes, torch.Tensor):
        path_nodes = torch.from_numpy(path_nodes).to(table.device)
    if not isinstance(path_len, torch.Tensor):
        path_len = torch.from_numpy(path_len).to(table.device)
    if new_length is None:
        new_length = length.new_empty((R,))
    _call(lib().ts_kv_accept, d, cache._ref, _int32("length", length, (R,), d), _int32("n", n, (R,), d), R,
          _int32("table", table, (R, max_blocks), d), max_blocks, _int32("path_nodes", path_nodes, (R, TS_MAX_D), d),
          _int32("path_len", path_len, (R,), d), _int32("new_length", new_length, (R,), d))
    return new_length
