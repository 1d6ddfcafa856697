"""The cache's binding on the host: what must never reach the library (which a stub stands in for)."""
import pytest

from paper_2609_22098_amd import kv

torch = pytest.importorskip("torch")


class _Library:
    """Stands in for the library and counts the calls that reach it."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def entry(*args):
            self.calls.append((name, args))
            return 0
        return entry


@pytest.fixture
def library(monkeypatch):
    stub = _Library()
    monkeypatch.setattr(kv, "lib", lambda: stub)
    monkeypatch.setattr(kv, "_current_stream", lambda device: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    return stub


def _given(R=2, pages=6, blocks=4):
    i32 = dict(dtype=torch.int32)
    return dict(free_pages=torch.arange(pages, **i32), free_count=torch.full((1,), pages, **i32),
                held=torch.zeros((R,), **i32), table=torch.full((R, blocks), -1, **i32))


def test_a_pool_on_the_host_is_refused(library):
    """Host tensors agree among themselves about their device; a pool of them never gets as far as a plan."""
    length = n = torch.zeros((2,), dtype=torch.int32)
    for make in (lambda: kv.Pool(6, 2, 4, 16, device="cpu"), lambda: kv.Pool(6, 2, 4, 16, **_given())):
        with pytest.raises(ValueError):
            kv.plan(make(), length, n, 3)
    assert not library.calls


def test_no_address_is_taken_of_a_host_tensor(library):
    """Not even where a device of -1, which host tensors report, is asked for."""
    with pytest.raises(ValueError):
        kv._int32("n", torch.zeros((2,), dtype=torch.int32), (2,), -1)


def _pool(monkeypatch):
    """A pool whose tensors pass for GPU tensors."""
    monkeypatch.setattr(kv, "_int32", lambda name, t, shape, device: f"{name} {list(t.shape)}")
    return kv.Pool(6, 2, 4, 16, **_given())


def test_a_plan_without_slots_writes_none(library, monkeypatch):
    """slots=False asks for pages alone, also where tensors are given; a slot of None among those says the same."""
    pool = _pool(monkeypatch)
    length = n = torch.zeros((2,), dtype=torch.int32)
    slot, granted = torch.zeros((2, 3), dtype=torch.int32), torch.zeros((2,), dtype=torch.int32)
    for slots, out, want in ((False, (slot, granted), None), (False, (None, granted), None), (True, (None, granted), None),
                             (True, (slot, granted), slot), (False, None, None)):
        got = kv.plan(pool, length, n, 3, slots=slots, out=out)
        assert got[0] is want and (out is None or got[1] is granted)
        name, args = library.calls[-1]
        assert name == "ts_kv_plan" and args[11] == (None if want is None else slot.data_ptr())
    assert kv.plan(pool, length, n, 3)[0].shape == (2, 3) and library.calls[-1][1][11]


def test_no_workspace_for_sizes_that_a_call_refuses():
    """R * cap * q_heads of 2^31 and more; one row less has a size."""
    import ctypes
    from paper_2609_22098_amd import binding as b
    c = kv.CacheStruct(0x1000, 1 << 20, 8704 * 2, 2, 10, 64, 2, 128)

    def size(R, cap, hq):
        return kv.lib().ts_kv_attention_workspace_size(ctypes.byref(c), R, cap, hq, b.TS_BF16)

    assert size(65536, 1 << 13, 4) == 0 and size(65536, (1 << 13) - 1, 4) > 0
    assert size(2048, 1 << 20, 2) == 0 and size(1023, 1 << 20, 2) > 0


def test_accepted_lengths_go_to_none_of_the_inputs():
    """Every layer reads the tables and the paths while the new lengths are written."""
    import ctypes
    from paper_2609_22098_amd import binding as b
    c = kv.CacheStruct(0x1000, 1 << 20, 8704 * 2, 2, 10, 64, 2, 128)
    arrays = [0x1000, 0x2000, 0x3000, 0x4000, 0x5000]  # len, n, table, path_nodes, path_len; never dereferenced
    length, n, table, nodes, count = arrays
    for new in arrays:
        assert kv.lib().ts_kv_accept(ctypes.byref(c), length, n, 1, table, 1, nodes, count, new, None) == b.TS_EINVAL
