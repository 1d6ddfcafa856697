"""The cache's C ABI on the host: exports, sizes and refusals (nothing is launched), and the binding's checks."""
import ctypes
import os
import re

import numpy as np
import pytest

from paper_2609_22098_amd import binding as b
from paper_2609_22098_amd import kv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x1000  # a non-null address that is never dereferenced


def test_library_exports_every_declared_symbol():
    txt = open(os.path.join(ROOT, "include", "treespark_kv.h")).read()
    declared = sorted(set(re.findall(r"^(?:size_t|int32_t)\s+(ts_\w+)\s*\(", txt, re.M)))
    assert sorted(kv.EXPORTED) == declared and len(declared) == 7
    for name in declared:
        assert hasattr(kv.lib(), name), name


def test_block_bytes():
    for page in kv.PAGE_SIZES:
        for D in kv.HEAD_DIMS:
            assert kv.block_bytes(page, D) == 2 * page * (D // 2 + D // 32)
    for page, D in ((0, 64), (8, 64), (48, 64), (512, 64), (16, 32), (16, 96), (16, 0), (-16, 64), (16, 512)):
        assert kv.lib().ts_kv_block_bytes(page, D) == 0
        with pytest.raises(ValueError):
            kv.block_bytes(page, D)


def _cache(**kw):
    f = dict(pages=FAKE, layer_stride=1 << 20, page_stride=8704 * 2, layers=2, num_pages=10, page_size=64, heads=2,
             head_dim=128)
    f.update(kw)
    return kv.CacheStruct(*[f[name] for name, _ in kv.CacheStruct._fields_])


BAD_CACHES = [(dict(pages=None), b.TS_EINVAL), (dict(pages=FAKE + 8), b.TS_EINVAL), (dict(layers=0), b.TS_EINVAL),
              (dict(num_pages=0), b.TS_EINVAL), (dict(heads=0), b.TS_EINVAL), (dict(page_size=48), b.TS_EUNSUPPORTED),
              (dict(page_size=8), b.TS_EUNSUPPORTED), (dict(head_dim=96), b.TS_EUNSUPPORTED),
              (dict(page_stride=8704 * 2 - 16), b.TS_EINVAL), (dict(page_stride=8704 * 2 + 8), b.TS_EINVAL),
              (dict(layer_stride=16), b.TS_EINVAL), (dict(layer_stride=(1 << 20) + 8), b.TS_EINVAL),
              (dict(page_stride=-8704 * 2), b.TS_EINVAL), (dict(num_pages=1 << 25), b.TS_EUNSUPPORTED),
              (dict(layers=1 << 16), b.TS_EUNSUPPORTED)]


def _append(c, layer=0, k=FAKE, v=FAKE, dtype=b.TS_BF16, ks=256, vs=256, slot=FAKE, rows=3):
    return kv.lib().ts_kv_append(ctypes.byref(c) if c else None, layer, k, v, dtype, ks, vs, slot, rows, None)


def _read(c, layer=0, layers=1, slot=FAKE, rows=3, k=FAKE, v=FAKE, dtype=b.TS_BF16):
    return kv.lib().ts_kv_read(ctypes.byref(c) if c else None, layer, layers, slot, rows, k, v, dtype, None)


def _attention(c, layer=0, q=FAKE, dtype=b.TS_BF16, qs=512, hq=4, length=FAKE, n=FAKE, R=2, cap=5, table=FAKE, blocks=8,
               mask=FAKE, scale=0.1, out=FAKE, lse=FAKE, ws=FAKE, wsb=1 << 40):
    return kv.lib().ts_kv_attention(ctypes.byref(c) if c else None, layer, q, dtype, qs, hq, length, n, R, cap, table,
                                    blocks, mask, scale, out, lse, ws, wsb, None)


def _accept(c, length=FAKE, n=FAKE, R=2, table=FAKE, blocks=8, nodes=FAKE, plen=FAKE, new=FAKE + 64):
    return kv.lib().ts_kv_accept(ctypes.byref(c) if c else None, length, n, R, table, blocks, nodes, plen, new, None)


@pytest.mark.parametrize("call", [_append, _read, _attention, _accept])
def test_bad_caches_are_refused(call):
    assert call(None) == b.TS_EINVAL
    for change, code in BAD_CACHES:
        assert call(_cache(**change)) == code, change
        assert kv.lib().ts_last_error()


def test_append_and_read_refusals():
    c = _cache()
    for kw in (dict(layer=-1), dict(layer=2), dict(k=None), dict(v=None), dict(slot=None), dict(dtype=2), dict(rows=-1),
               dict(ks=255), dict(ks=248), dict(vs=260), dict(k=FAKE + 8), dict(v=FAKE + 4)):
        assert _append(c, **kw) == b.TS_EINVAL, kw
    assert _append(c, dtype=b.TS_F32, ks=258, vs=256) == b.TS_EINVAL
    assert _append(c, rows=0, k=None, v=None, slot=None) == b.TS_OK
    for kw in (dict(layer=-1), dict(layer=2), dict(layer=1, layers=2), dict(layers=0), dict(slot=None), dict(dtype=-1),
               dict(rows=-1), dict(k=FAKE + 8), dict(v=FAKE + 8)):
        assert _read(c, **kw) == b.TS_EINVAL, kw
    assert _read(c, rows=0) == b.TS_OK and _read(c, k=None, v=None) == b.TS_OK


def test_attention_refusals():
    c = _cache()
    for kw in (dict(layer=2), dict(layer=-1), dict(q=None), dict(length=None), dict(n=None), dict(table=None),
               dict(out=None), dict(dtype=5), dict(hq=3), dict(hq=0), dict(hq=-2), dict(R=-1), dict(cap=0),
               dict(cap=b.lib().ts_tree_mask_words(1) + 4096), dict(blocks=0), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(qs=511), dict(qs=516), dict(q=FAKE + 8), dict(out=FAKE + 8)):
        assert _attention(c, **kw) == b.TS_EINVAL, kw
    assert _attention(c, mask=None, cap=(1 << 20) + 1) == b.TS_EINVAL
    assert _attention(c, R=65537) == b.TS_EUNSUPPORTED
    assert _attention(c, R=65536, mask=None, cap=1 << 14) == b.TS_EUNSUPPORTED  # rows * heads reach 2^31
    assert _attention(c, blocks=(1 << 24) + 1) == b.TS_EUNSUPPORTED
    assert _attention(c, R=0, q=None) == b.TS_OK


def test_sizes_past_the_kernels_counters_are_refused():
    """Groups whose places in the line of work could pass 64 bits, threads past a launch's 32, pages past 31; a scale
    that is infinite in base 2; outputs on top of inputs."""
    c = _cache()
    assert _attention(c, hq=514, qs=514 * 128) == b.TS_EUNSUPPORTED
    assert kv.lib().ts_kv_attention_workspace_size(ctypes.byref(c), 2, 5, 514, b.TS_BF16) == 0
    assert kv.lib().ts_kv_attention_workspace_size(ctypes.byref(c), 2, 5, 512, b.TS_BF16) > 0
    assert _attention(c, scale=3e38) == b.TS_EINVAL
    assert _attention(c, q=FAKE, out=FAKE) == b.TS_EINVAL
    big = _cache(heads=1024, head_dim=256, page_size=16, page_stride=1024 * 16 * 272)
    big.layer_stride = 10 * big.page_stride
    width = 1024 * 256
    assert _append(big, ks=width, vs=width, rows=(1 << 16) + 1) == b.TS_EUNSUPPORTED
    assert _read(big, rows=(1 << 16) + 1) == b.TS_EUNSUPPORTED
    for same in ("n", "plen"):
        assert _accept(c, **{same: FAKE + 64}) == b.TS_EINVAL
    assert kv.lib().ts_kv_plan(FAKE, FAKE, 65536, 1, 16, (1 << 27) - 1, (1 << 15) - 1, *[FAKE] * 6, None) == b.TS_EUNSUPPORTED


def test_attention_workspace():
    """A function of sizes alone, which a call refuses to go below; 0 for what it would refuse."""
    c, L = _cache(), kv.lib()

    def size(R=2, cap=5, hq=4, dtype=b.TS_BF16, c=c):
        return L.ts_kv_attention_workspace_size(ctypes.byref(c), R, cap, hq, dtype)

    assert 0 < size(R=1) <= size() <= size(R=60000) and size() <= size(cap=500)
    assert size(hq=3) == size(cap=0) == size(R=-1) == size(dtype=4) == size(c=_cache(head_dim=80)) == 0
    for R, cap, hq, dtype in ((2, 5, 4, b.TS_BF16), (1, 1, 2, b.TS_F32), (70, 65, 8, b.TS_BF16), (1, 4096, 4, b.TS_F32)):
        n = size(R, cap, hq, dtype)
        kw = dict(R=R, cap=cap, hq=hq, dtype=dtype, qs=hq * 128)
        assert _attention(c, wsb=n - 1, **kw) == b.TS_ENOSPACE
        assert _attention(c, wsb=n, ws=None, **kw) == b.TS_EINVAL and _attention(c, wsb=n, ws=FAKE + 8, **kw) == b.TS_EINVAL


def test_accept_refusals():
    c = _cache()
    for kw in (dict(length=None), dict(n=None), dict(table=None), dict(nodes=None), dict(plen=None), dict(new=None),
               dict(R=-1), dict(blocks=0), dict(new=FAKE)):
        assert _accept(c, **kw) == b.TS_EINVAL, kw
    assert _accept(c, R=65537) == b.TS_EUNSUPPORTED
    assert _accept(c, R=0, nodes=None) == b.TS_OK


def test_plan_refusals():
    def call(length=FAKE, n=FAKE, R=2, cap=5, page=16, pages=10, blocks=4, free=FAKE, count=FAKE, held=FAKE, table=FAKE,
             slot=FAKE, granted=FAKE):
        return kv.lib().ts_kv_plan(length, n, R, cap, page, pages, blocks, free, count, held, table, slot, granted, None)

    for name in ("length", "n", "free", "count", "held", "table", "granted"):
        assert call(**{name: None}) == b.TS_EINVAL, name
    for kw in (dict(R=-1), dict(cap=0), dict(cap=(1 << 20) + 1), dict(pages=0), dict(blocks=0)):
        assert call(**kw) == b.TS_EINVAL, kw
    for kw in (dict(page=17), dict(page=0), dict(R=65537), dict(pages=1 << 27), dict(blocks=(1 << 26) + 1),
               dict(R=65536, blocks=1 << 15), dict(R=65536, cap=1 << 15)):
        assert call(**kw) == b.TS_EUNSUPPORTED, kw
    assert call(R=0, length=None) == b.TS_OK


def test_binding_refuses_what_is_not_on_a_gpu():
    torch = pytest.importorskip("torch")
    i32 = torch.zeros((2,), dtype=torch.int32)
    with pytest.raises(ValueError):
        kv.Cache(torch.zeros((1, 4, 8704), dtype=torch.uint8), 64, 1, 128)
    with pytest.raises(ValueError):
        kv.Pool(4, 2, 8, 16, device="cpu", held=i32)


def test_plain_quantisation_by_hand():
    """The oracle's rounding at borders: ties to the even code, the scale's step between 7 and 8."""
    import kv_ref
    x = np.zeros((1, 32))
    x[0, :9] = [6, 5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -5]
    code, byte = kv_ref.quantise(x)
    assert byte[0, 0] == 127
    assert list(kv_ref.VALUES[code[0, :9]]) == [6, 4, 4, 2, 2, 1, 1, 0, -4]
    for top, want in ((7.0, 127), (7.0000005, 128), (3.5, 126), (0.0, 2), (1e-45, 2), (3.4e38, 252)):
        x[0, :] = 0
        x[0, 3] = top
        assert kv_ref.quantise(x)[1][0, 0] == want, top
