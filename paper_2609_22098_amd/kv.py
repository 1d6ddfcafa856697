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
"""
from __future__ import annotations

import ctypes

from . import binding
from .binding import TS_BF16, TS_F32, TS_MAX_D, TreeSparkError, _check, _torch  # noqa: F401

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


def _int32(name, t, shape, device):
    """The address of a contiguous int32 tensor of that shape on that GPU."""
    if t.dtype is not _torch().int32 or tuple(t.shape) != shape or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous int32 tensor {list(shape)} on cuda:{device} is needed, "
                         f"got {t.dtype} {list(t.shape)} on {t.device}")
    return t.data_ptr()


class _On:
    """The device's current or the given stream, with the device current during the call."""

    __slots__ = ("device", "stream", "before")

    def __init__(self, device, stream):
        cuda = _torch().cuda
        if stream is None:
            stream = cuda.current_stream(device)
        elif stream.device_index != device:
            raise ValueError(f"the stream is of cuda:{stream.device_index}, the tensors are on cuda:{device}")
        self.device, self.stream = device, stream.cuda_stream

    def __enter__(self):
        cuda = _torch().cuda
        self.before = cuda.current_device()
        if self.before != self.device:
            cuda.set_device(self.device)
        return self.stream

    def __exit__(self, *_):
        if self.before != self.device:
            _torch().cuda.set_device(self.before)


class Cache:
    """A cache over pages [layers][num_pages][bytes], a uint8 GPU tensor with contiguous pages of at least
    heads * block_bytes(page_size, head_dim) bytes (layers and pages may have any strides that are multiples
    of 16)."""

    def __init__(self, pages, page_size, heads, head_dim):
        torch = _torch()
        if pages.dim() != 3 or pages.dtype is not torch.uint8 or not pages.is_cuda or pages.stride(2) != 1:
            raise ValueError("pages: a uint8 tensor [layers][num_pages][bytes] on a GPU is needed")
        block = block_bytes(page_size, head_dim)
        if pages.shape[2] < heads * block:
            raise ValueError(f"pages of {pages.shape[2]} bytes hold no {heads} heads of {block}")
        self.pages, self.device = pages, pages.get_device()
        self.struct = CacheStruct(pages.data_ptr(), pages.stride(0), pages.stride(1), pages.shape[0], pages.shape[1],
                                  page_size, heads, head_dim)
        self._ref = ctypes.byref(self.struct)

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
    torch = _torch()
    pages = torch.zeros((layers, num_pages, heads * block_bytes(page_size, head_dim)), dtype=torch.uint8, device=device)
    return Cache(pages, page_size, heads, head_dim)


class Pool:
    """The free pages and the requests' block tables: free_pages [num_pages], free_count [1], held [R], table
    [R][max_blocks], int32 on one GPU (given, or new with every page free)."""

    def __init__(self, num_pages, R, max_blocks, page_size, device="cuda", free_pages=None, free_count=None, held=None,
                 table=None):
        torch = _torch()
        given = (free_pages, free_count, held, table)
        if all(t is None for t in given):
            free_pages = torch.arange(num_pages, dtype=torch.int32, device=device)
            free_count = torch.full((1,), num_pages, dtype=torch.int32, device=device)
            held = torch.zeros((R,), dtype=torch.int32, device=device)
            table = torch.full((R, max_blocks), -1, dtype=torch.int32, device=device)
        elif any(t is None for t in given):
            raise ValueError("free_pages, free_count, held and table are given together")
        self.num_pages, self.R, self.max_blocks, self.page_size = num_pages, R, max_blocks, page_size
        self.free_pages, self.free_count, self.held, self.table = free_pages, free_count, held, table
        self.device = d = free_pages.get_device()
        self._addr = (_int32("free_pages", free_pages, (num_pages,), d), _int32("free_count", free_count, (1,), d),
                      _int32("held", held, (R,), d), _int32("table", table, (R, max_blocks), d))


def plan(pool: Pool, length, n, cap, slots=True, out=None, stream=None):
    """ts_kv_plan: pages for the rows 0..n[q] behind length[q] tokens of every request.  Returns (slot [R][cap],
    granted [R]), int32; slot is None with slots=False (only the pages).  out = (slot, granted) reuses tensors."""
    torch = _torch()
    R, d = pool.R, pool.device
    a_len, a_n = _int32("length", length, (R,), d), _int32("n", n, (R,), d)
    if out is None:
        slot = torch.empty((R, cap), dtype=torch.int32, device=length.device) if slots else None
        granted = torch.empty((R,), dtype=torch.int32, device=length.device)
    else:
        slot, granted = out
        _int32("granted", granted, (R,), d)
        if slot is not None:
            _int32("slot", slot, (R, cap), d)
    free_pages, free_count, held, table = pool._addr
    with _On(d, stream) as s:
        _check(lib().ts_kv_plan(a_len, a_n, R, cap, pool.page_size, pool.num_pages, pool.max_blocks, free_pages, free_count,
                                held, table, slot.data_ptr() if slot is not None else None, granted.data_ptr(), s))
    return slot, granted


def _rows(name, t, cache):
    """Address and row stride of keys or values [rows][heads][head_dim] (or [R][cap][heads][head_dim])."""
    s = cache.struct
    if t.shape[-2:] != (s.heads, s.head_dim) or t.dim() not in (3, 4) or t.get_device() != cache.device:
        raise ValueError(f"{name}: [rows][{s.heads}][{s.head_dim}] on cuda:{cache.device} is needed, got {list(t.shape)} "
                         f"on {t.device}")
    st = t.stride()
    if st[-1] != 1 or st[-2] != s.head_dim or (t.dim() == 4 and st[0] != st[1] * t.shape[1]):
        raise ValueError(f"{name}: the heads of a row must be contiguous and rows evenly spaced, got strides {st}")
    return t.data_ptr(), st[-3]


def append(cache: Cache, k, v, slot, layer=0, stream=None):
    """ts_kv_append: rows' keys and values k, v [rows][heads][head_dim] (float32 or bfloat16; rows may be apart,
    as in a projection's output that holds both) into a layer of the cache, at slot (int32, one per row)."""
    a_k, s_k = _rows("k", k, cache)
    a_v, s_v = _rows("v", v, cache)
    if k.dtype is not v.dtype or k.shape[:-2] != v.shape[:-2]:
        raise ValueError("k and v must have one dtype and as many rows")
    rows = slot.numel()
    if k.shape[:-2].numel() != rows:
        raise ValueError(f"{rows} slots for {k.shape[:-2].numel()} rows")
    a_slot = _int32("slot", slot, tuple(slot.shape), cache.device)
    with _On(cache.device, stream) as s:
        _check(lib().ts_kv_append(cache.ref(), layer, a_k, a_v, binding._dtype_code(k), s_k, s_v, a_slot, rows, s))


def read(cache: Cache, slot, layer=0, layers=None, dtype=None, out=None, stream=None):
    """ts_kv_read: the rows at slot as (k, v) [layers][rows][heads][head_dim], of `layers` layers from `layer` on
    (None: all that follow).  out = (k, v) reuses tensors, either of which may be None; without it rows that have no
    slot are zero.  dtype: float32 or bfloat16 (the default)."""
    torch = _torch()
    c = cache.struct
    layers = c.layers - layer if layers is None else layers
    rows = slot.numel()
    shape = (layers, rows, c.heads, c.head_dim)
    if out is None:
        out = tuple(torch.zeros(shape, dtype=dtype or torch.bfloat16, device=slot.device) for _ in range(2))
    k, v = out
    one = k if k is not None else v
    for t in out:
        if t is not None and (tuple(t.shape) != shape or t.get_device() != cache.device or not t.is_contiguous()
                              or t.dtype is not one.dtype):
            raise ValueError(f"out: contiguous tensors {list(shape)} of one dtype on cuda:{cache.device} are needed")
    if one is None:
        return out
    a_slot = _int32("slot", slot, tuple(slot.shape), cache.device)
    with _On(cache.device, stream) as s:
        _check(lib().ts_kv_read(cache.ref(), layer, layers, a_slot, rows, k.data_ptr() if k is not None else None,
                                v.data_ptr() if v is not None else None, binding._dtype_code(one), s))
    return k, v


def attention_workspace_size(cache: Cache, R, cap, q_heads, dtype):
    """ts_kv_attention_workspace_size for queries of a torch dtype."""
    code = TS_BF16 if dtype is _torch().bfloat16 else TS_F32
    with _On(cache.device, None):
        return lib().ts_kv_attention_workspace_size(cache.ref(), R, cap, q_heads, code)


def attention(cache: Cache, q, length, n, table, mask=None, scale=None, layer=0, out=None, lse=None, workspace=None,
              stream=None):
    """ts_kv_attention.  q [R][cap][q_heads][head_dim] (float32 or bfloat16; rows may be apart), length and n [R], table
    [R][max_blocks], mask the [R][cap][W] words of binding.tree_mask or None for chains (causal).  scale: head_dim
    ** -0.5 by default.  Returns (out, lse): out like q, contiguous; lse float32 [R][cap][q_heads] if given, else None.
    Rows past n[q] of given tensors are left as they were; those of a new out are zero."""
    torch = _torch()
    c, d = cache.struct, cache.device
    if q.dim() != 4 or q.shape[3] != c.head_dim or q.get_device() != d:
        raise ValueError(f"q: [R][cap][q_heads][{c.head_dim}] on cuda:{d} is needed, got {list(q.shape)} on {q.device}")
    R, cap, q_heads, D = q.shape
    st = q.stride()
    if st[3] != 1 or (st[2] != D and q_heads > 1) or (st[0] != st[1] * cap and R > 1):
        raise ValueError(f"q: the heads of a row must be contiguous and rows evenly spaced, got strides {st}")
    dtype = binding._dtype_code(q)
    if table.dim() != 2:
        raise ValueError("table: [R][max_blocks] is needed")
    max_blocks = table.shape[1]
    a_table = _int32("table", table, (R, max_blocks), d)
    a_len, a_n = _int32("length", length, (R,), d), _int32("n", n, (R,), d)
    a_mask = _int32("mask", mask, (R, cap, (cap + 31) // 32), d) if mask is not None else None
    if out is None:
        out = torch.zeros((R, cap, q_heads, D), dtype=q.dtype, device=q.device)
    elif out.shape != q.shape or out.dtype is not q.dtype or out.get_device() != d or not out.is_contiguous():
        raise ValueError(f"out: a contiguous {q.dtype} tensor {list(q.shape)} on cuda:{d} is needed")
    if lse is not None and (lse.dtype is not torch.float32 or tuple(lse.shape) != (R, cap, q_heads)
                            or lse.get_device() != d or not lse.is_contiguous()):
        raise ValueError(f"lse: a contiguous float32 tensor {[R, cap, q_heads]} on cuda:{d} is needed")
    with _On(d, stream) as s:
        if workspace is None:
            size = lib().ts_kv_attention_workspace_size(cache.ref(), R, cap, q_heads, dtype)
            with torch.cuda.stream(stream or torch.cuda.current_stream(d)):  # freed memory is reused in its order
                workspace = torch.empty((max(size, 1),), dtype=torch.uint8, device=q.device)
        elif workspace.get_device() != d or workspace.dtype is not torch.uint8 or not workspace.is_contiguous():
            raise ValueError(f"workspace: a contiguous uint8 tensor on cuda:{d} is needed")
        _check(lib().ts_kv_attention(cache.ref(), layer, q.data_ptr(), dtype, st[1] if cap > 1 or R > 1 else q_heads * D, q_heads,
                                     a_len, a_n, R, cap, a_table, max_blocks, a_mask,
                                     D ** -0.5 if scale is None else scale, out.data_ptr(),
                                     lse.data_ptr() if lse is not None else None, workspace.data_ptr(),
                                     workspace.numel(), s))
    return out, lse


def accept(cache: Cache, length, n, table, path_nodes, path_len, new_length=None, stream=None):
    """ts_kv_accept: the accepted paths' rows, in every layer, moved behind the contexts.  path_nodes [R][16] and
    path_len [R] as binding.verify returns them (numpy arrays are copied to the GPU) or int32 GPU tensors.  Returns
    the new lengths [R]."""
    torch = _torch()
    d = cache.device
    if table.dim() != 2:
        raise ValueError("table: [R][max_blocks] is needed")
    R, max_blocks = table.shape
    if not isinstance(path_nodes, torch.Tensor):
        path_nodes = torch.from_numpy(path_nodes).to(table.device)
    if not isinstance(path_len, torch.Tensor):
        path_len = torch.from_numpy(path_len).to(table.device)
    if new_length is None:
        new_length = torch.empty((R,), dtype=torch.int32, device=table.device)
    with _On(d, stream) as s:
        _check(lib().ts_kv_accept(cache.ref(), _int32("length", length, (R,), d), _int32("n", n, (R,), d), R,
                                  _int32("table", table, (R, max_blocks), d), max_blocks,
                                  _int32("path_nodes", path_nodes, (R, TS_MAX_D), d), _int32("path_len", path_len, (R,), d),
                                  _int32("new_length", new_length, (R,), d), s))
    return new_length
