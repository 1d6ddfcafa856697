"""The 4-bit cache's kernels against plain numpy in 64 bits (kv_ref): planning, rows in and out, attention, the
accepted rows, and a whole round of them."""
import numpy as np
import pytest

import kv_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "GPU tests need a GPU"
    from paper_2609_22098_amd import kv
    kv.lib()
    return t


def _dev(torch, a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a).astype(dtype)).cuda()


# ---------------------------------------------------------------- plan


@pytest.mark.parametrize("R,cap,page,blocks,rounds,spare", [
    (1, 1, 16, 4, 4, 9), (1, 65, 64, 40, 4, 60), (5, 33, 16, 12, 8, 40), (64, 65, 64, 9, 4, 300), (70, 7, 32, 6, 4, 200),
    (200, 5, 16, 5, 4, 700), (1500, 3, 16, 3, 3, 3000), (2100, 2, 16, 4, 3, 4000), (3, 2049, 128, 40, 3, 60)])
def test_plan_rounds(torch, R, cap, page, blocks, rounds, spare):
    """Several rounds on one pool: lengths that grow and shrink, requests that leave, tables and pools that are too
    small; every array equals the literal walk's."""
    from paper_2609_22098_amd import kv
    rng = np.random.default_rng(R * 1000 + cap)
    pool = kv.Pool(spare, R, blocks, page)
    free, held, table = list(range(spare)), np.zeros(R, np.int64), np.full((R, blocks), -1, np.int64)
    for r in range(rounds):
        length = rng.integers(0, blocks * page + 3, R)
        n = rng.integers(-1, cap + 2, R)
        gone = rng.random(R) < 0.3
        length[gone], n[gone] = 0, -1
        if r == 1:
            n[:] = -3
        if r == 0:
            length //= 3
        slot, granted = kv.plan(pool, _dev(torch, length), _dev(torch, n), cap, slots=(r != 2))
        want_slot, want_granted = kv_ref.plan(length, n, cap, page, blocks, free, held, table)
        assert np.array_equal(granted.cpu().numpy(), want_granted)
        if r != 2:
            assert np.array_equal(slot.cpu().numpy(), want_slot)
        assert np.array_equal(pool.held.cpu().numpy(), held) and np.array_equal(pool.table.cpu().numpy(), table)
        count = int(pool.free_count)
        assert count == len(free) and np.array_equal(pool.free_pages.cpu().numpy()[:count], free)


def test_plan_gives_back_what_it_took(torch):
    """Taking pages and giving them back at once restores the stack, order and all."""
    from paper_2609_22098_amd import kv
    rng = np.random.default_rng(0)
    pool = kv.Pool(500, 40, 16, 16)
    length = _dev(torch, rng.integers(0, 100, 40))
    kv.plan(pool, length, _dev(torch, np.full(40, -1)), 65, slots=False)
    before = [t.clone() for t in (pool.free_pages, pool.free_count, pool.held, pool.table)]
    kv.plan(pool, length, _dev(torch, rng.integers(0, 65, 40)), 65)
    assert int(pool.free_count) < int(before[1])
    kv.plan(pool, length, _dev(torch, np.full(40, -1)), 65, slots=False)
    for a, b in zip((pool.free_pages, pool.free_count, pool.held, pool.table), before):
        assert torch.equal(a[: int(before[1])] if a is pool.free_pages else a,
                           b[: int(before[1])] if a is pool.free_pages else b)


def test_plan_counts_out_of_range(torch):
    """Lengths, counts and page ids that no round leaves behind are cut to their range; nothing else is touched."""
    from paper_2609_22098_amd import kv
    pool = kv.Pool(8, 3, 4, 16)
    pool.free_count.fill_(99)       # read as 8
    pool.free_pages[7] = 1 << 20    # the page on top does not exist
    pool.held[2] = -5               # read as 0
    slot, granted = kv.plan(pool, _dev(torch, [-7, 2**31 - 1, 0]), _dev(torch, [3, 0, 2**31 - 1]), 20)
    assert granted.tolist() == [3, -1, 19]
    assert slot[0].tolist() == [-1] * 20          # its only page is the one that does not exist
    assert slot[1].tolist() == [-1] * 20
    assert slot[2].tolist() == list(range(96, 112)) + list(range(80, 84))
    assert int(pool.free_count) == 5 and pool.held.tolist() == [1, 0, 2]


# ---------------------------------------------------------------- rows in and out


def _rows(rng, rows, heads, D):
    """Values over many magnitudes, with groups of zeros, of one value, on the borders of rounding and scale."""
    x = rng.standard_normal((rows, heads, D)) * 2.0 ** rng.integers(-30, 30, (rows, heads, 1))
    g = x.reshape(-1, 32)
    g[0] = 0
    g[1 % len(g)] = 0
    g[1 % len(g), 7] = -3e-39
    g[2 % len(g)] = np.tile([6, 5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25], 4) * np.where(np.arange(32) % 3, 1, -1)
    g[3 % len(g)] = 7 * 2.0 ** -5
    g[4 % len(g), 0] = 3.3e38
    return g.reshape(x.shape).astype(np.float32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,heads,D,page", [(1, 1, 64, 16), (5, 3, 128, 64), (33, 2, 256, 32), (7, 1, 64, 256),
                                               (130, 5, 128, 16), (9, 8, 64, 128)])
def test_rows_in_and_out(torch, dtype, rows, heads, D, page):
    """Every value read back is the one that the format's rule gives, in both dtypes; rows without a slot are
    neither written nor read; rows of not-a-numbers mark their own head alone."""
    from paper_2609_22098_amd import kv
    rng = np.random.default_rng(rows)
    pages = -(-rows // page) + 3
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    both = torch.from_numpy(np.concatenate([_rows(rng, rows, heads, D), _rows(rng, rows, heads, D)], 1)).to(t)
    if rows > 4:
        both[1, 0, 5] = float("nan")
        both[2, 2 * heads - 1, 0] = float("inf")
        both[3, heads, D - 1] = -float("inf")
    cache = kv.empty_cache(2, pages, page, heads, D)
    slot = rng.permutation(pages * page)[:rows].astype(np.int32)
    if rows > 4:
        slot[4] = [-1, pages * page, 2**31 - 1, -(2**31)][rows % 4]
    dev = both.cuda()
    kv.append(cache, dev[:, :heads], dev[:, heads:], _dev(torch, slot), layer=1)
    want_k, want_v = kv_ref.rounded(both[:, :heads].double().numpy(), both[:, heads:].double().numpy())
    for out_t in (torch.float32, torch.bfloat16):
        k, v = (torch.full((2, rows, heads, D), 77.0, dtype=out_t, device="cuda") for _ in "kv")
        kv.read(cache, _dev(torch, slot), out=(k, v))
        k2, _ = kv.read(cache, _dev(torch, slot), layer=1, out=(torch.full_like(k[1:], 77.0), None))
        there = (slot >= 0) & (slot < pages * page)
        for got, want in ((k, want_k), (v, want_v)):
            assert np.array_equal(got[1].cpu().double().numpy()[there], want[there], equal_nan=True)
            assert (got[0][torch.from_numpy(there).cuda()] == 0).all()   # the other layer is as it was
            assert (got[:, torch.from_numpy(~there).cuda()] == 77).all()
        assert torch.equal(k2[0].nan_to_num(5.0), k[1].nan_to_num(5.0))


def test_rows_keep_their_neighbours(torch):
    """Writing one slot changes that token's bytes only, in its layer and page."""
    from paper_2609_22098_amd import kv
    cache = kv.empty_cache(3, 4, 16, 2, 64)
    cache.pages.random_(0, 256)
    before = cache.pages.clone()
    x = torch.randn((1, 2, 64), device="cuda")
    kv.append(cache, x, x, _dev(torch, [2 * 16 + 5]), layer=1)
    changed = torch.nonzero(cache.pages != before).cpu().numpy()
    assert len(changed) and set(map(tuple, changed[:, :2])) == {(1, 2)}
    inside = set()
    for h in range(2):
        base = h * 16 * 68
        for at, size in ((5 * 32, 32), (512 + 5 * 2, 2), (544 + 5 * 32, 32), (1056 + 5 * 2, 2)):
            inside |= set(range(base + at, base + at + size))
    assert set(changed[:, 2]) <= inside


# ---------------------------------------------------------------- attention


class Case:
    """A batch: cache, tables with scattered pages, queries, masks, and the oracle's answer."""

    def __init__(self, torch, lens, ns, cap, hq, heads, D, page, dtype, mask, seed=0, layers=1, reach=0, kscale=1.0):
        from paper_2609_22098_amd import kv
        rng = np.random.default_rng(seed)
        self.lens, self.ns, self.cap, self.D, self.dtype = np.array(lens), np.array(ns), cap, D, dtype
        R = len(lens)
        self.rows = np.maximum(np.minimum(self.ns, cap - 1), -1) + 1
        need = -(-(self.lens + self.rows) // page)
        pages = int(need.sum()) + 2
        ids = rng.permutation(pages)
        self.blocks = max(int(need.max()), -(-reach // page))  # a table that names more tokens than there are
        self.table = np.full((R, self.blocks), -1, np.int64)
        at = 0
        for q in range(R):
            self.table[q, :need[q]] = ids[at:at + need[q]]
            at += need[q]
        ref = kv_ref.Cache(pages, page, heads, D)
        shape = (pages * page, heads, D)
        k = rng.standard_normal(shape) * kscale
        k[..., rng.integers(0, D, 3)] *= 6
        ref.k, ref.v = kv_ref.rounded(k, rng.standard_normal(shape))
        self.ref = ref
        self.t = torch.float32 if dtype == "f32" else torch.bfloat16
        self.q = torch.from_numpy(rng.standard_normal((R, cap, hq, D))).to(self.t)
        self.words = (cap + 31) // 32
        self.mask = None
        if mask:
            self.mask = np.zeros((R, cap, self.words), np.uint32)
            for q in range(R):
                parent = [-1] + [int(rng.integers(max(0, i - 4), i)) for i in range(1, max(self.rows[q], 1))]
                self.mask[q, :self.rows[q]] = kv_ref.tree_bits(parent, self.rows[q], self.words)
        self.scale = D ** -0.5
        self.layers, self.layer = layers, layers - 1

    def run(self, torch, kvq=None, **kw):
        from paper_2609_22098_amd import kv
        R, cap, hq, D = self.q.shape
        packed = kv_ref.pack(self.ref, 1)
        pages = torch.zeros((self.layers,) + packed.shape[1:], dtype=torch.uint8, device="cuda")
        pages[self.layer] = torch.from_numpy(packed[0].copy()).cuda()
        cache = kv.Cache(pages, self.ref.page, self.ref.k.shape[1], D)
        out = torch.full((R, cap, hq, D), 99.0, dtype=self.t, device="cuda")
        lse = torch.full((R, cap, hq), 99.0, device="cuda")
        mask = None if self.mask is None else torch.from_numpy(self.mask.view(np.int32)).cuda()
        q = self.q.cuda() if kvq is None else kvq
        kv.attention(cache, q, _dev(torch, self.lens), _dev(torch, self.ns), _dev(torch, self.table), mask=mask,
                     scale=self.scale, layer=self.layer, out=out, lse=lse, **kw)
        torch.cuda.synchronize()
        return out, lse

    def rows_of(self, q, tokens):
        """Keys and values of a request's positions; those without a page are not-a-number."""
        pos = np.arange(tokens)
        block = pos // self.ref.page
        page = np.where(block < self.blocks, self.table[q, np.minimum(block, self.blocks - 1)], -1)
        bad = (page < 0) | (page * self.ref.page >= len(self.ref.k))
        slot = np.where(bad, 0, page * self.ref.page + pos % self.ref.page)
        k, v = self.ref.k[slot].copy(), self.ref.v[slot].copy()
        k[bad] = np.nan
        v[bad] = 0
        return k, v

    def check(self, torch, **kw):
        out, lse = self.run(torch, **kw)
        got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
        query = self.q.double().numpy()
        half = 2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -24  # half a step of the output, relative
        worst = sums = norm = 0.0
        for q in range(len(self.lens)):
            rows, length = int(self.rows[q]), int(self.lens[q])
            assert (got[q, rows:] == 99).all() and (gl[q, rows:] == 99).all()
            if not rows:
                continue
            total = length + rows
            k, v = self.rows_of(q, total)
            see = kv_ref.sees(length, rows, total, None if self.mask is None else self.mask[q])
            want, wl, mass, mag = kv_ref.attention(query[q, :rows], k, v, see, self.scale)
            # A score is a sum of D products of at most mag in all.  The matrix unit aligns products of one
            # instruction to the largest: measured on random operands, 2.1e-5 of the sum of magnitudes is the
            # most that it drops (2^-15 allowed); fp32 sums drop D 2^-24 of it at most and far less in fact.
            # An error d of the scores moves out by at most (e^2d - 1) * mass and lse by d.  Sums of T fp32
            # weights add T 2^-24 at most, the exponential 2^-22, a weight rounded to bf16 half a step.
            d = mag * ((2.0 ** -15) if self.dtype == "bf16" else 2.0 ** -22)
            small = (total + 16) * 2.0 ** -24 + 2.0 ** -22
            weight = (half if self.dtype == "bf16" else 0.0) + small
            bound = half * np.abs(want) + (np.expm1(2 * d)[..., None] + weight) * mass + 1e-30
            nan = np.isnan(want)
            assert np.array_equal(np.isnan(got[q, :rows]), nan)
            e = np.where(nan, 0, np.abs(got[q, :rows] - want) - bound)
            assert e.max() <= 0, (q, e.max(), np.unravel_index(e.argmax(), e.shape))
            inf = np.isinf(wl)
            assert np.array_equal(np.isnan(gl[q, :rows]), np.isnan(wl)) and (gl[q, :rows][inf] == wl[inf]).all()
            fin = np.isfinite(wl)
            el = np.abs(gl[q, :rows] - np.where(fin, wl, 0)) - (d + small + 2.0 ** -22 * np.where(fin, np.abs(wl), 0))
            assert (el[fin] <= 0).all(), (q, el[fin].max())
            diff = np.where(nan, 0, got[q, :rows] - want)
            sums, norm = sums + (diff ** 2).sum(), norm + np.where(nan, 0, want ** 2).sum()
            worst = max(worst, float(np.abs(diff).max(initial=0)))
        # and as a whole: bf16 rounds outputs and weights, each within half a step, about uniformly, so that
        # both together stay under half a step in the 2-norm; f32 sums of up to some thousand terms walk
        # at random to sqrt(T) 2^-24
        if norm:
            rel = (sums / norm) ** 0.5
            assert rel <= (2.0 ** -8 if self.dtype == "bf16" else 4e-6), rel
        return out, lse


SHAPES = [  # lens, n, cap, hq, heads, D, page
    ([0], [0], 1, 1, 1, 64, 16),
    ([1], [0], 1, 4, 1, 128, 16),
    ([15, 16, 17, 0, 63, 64, 65], [0] * 7, 1, 8, 2, 128, 16),
    ([300, 1000, 5], [0, 0, 0], 1, 7, 1, 64, 64),
    ([130, 0, 77], [8, 3, 0], 9, 6, 2, 128, 32),
    ([40, 511, 0, 9], [32, -1, 32, 64], 33, 12, 12, 64, 16),
    ([700, 257], [64, 31], 65, 8, 2, 128, 64),
    ([513], [64], 65, 5, 1, 128, 128),
    ([100, 31], [70, 129], 130, 3, 3, 256, 32),
    ([2000, 3], [16, 2], 17, 16, 2, 256, 64),
    ([90, 400], [199, 150], 200, 4, 2, 64, 256),
    ([1200], [255], 256, 8, 1, 128, 16),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", [True, False])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attention(torch, shape, mask, dtype):
    """Chains and trees over contexts of no token to some thousand, groups of every kind, pages that end inside
    a tile, requests that sit out, counts above the capacity; tables that name few tokens, more, and many (the
    work is then cut otherwise, into tiles of other sizes)."""
    lens, n, cap, hq, heads, D, page = SHAPES[shape]
    for reach in (0, 1200, 17000):
        Case(torch, lens, n, cap, hq, heads, D, page, dtype, mask, seed=shape, layers=1 + shape % 2, reach=reach).check(torch)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,hi,cap,hq,heads,D,page", [(300, 90, 1, 2, 1, 64, 16), (300, 70, 5, 8, 2, 64, 64), (520, 40, 3, 44, 1, 128, 32),
                                                      (1, 20000, 1, 4, 1, 128, 64), (2, 9000, 1, 1, 1, 256, 16), (1, 6000, 40, 8, 1, 128, 64),
                                                      (3, 2500, 7, 4, 2, 256, 128)])
def test_attention_cuts(torch, R, hi, cap, hq, heads, D, page, dtype):
    """More requests than a workgroup has threads; a context that is cut into more pieces than a wave has lanes."""
    rng = np.random.default_rng(R + hi)
    lens, n = rng.integers(0, hi + 1, R), rng.integers(-1, cap, R)
    lens[0], n[0] = hi, cap - 1
    Case(torch, lens, n, cap, hq, heads, D, page, dtype, cap > 1, seed=R, reach=17000).check(torch)


def test_attention_scale_of_zero(torch):
    """Every visible token has the same weight; hidden ones still have none."""
    for dtype in ("bf16", "f32"):
        for reach in (0, 17000):
            c = Case(torch, [70, 0], [39, 3], 40, 4, 2, 128, 16, dtype, True, seed=12, reach=reach)
            c.scale = 0.0
            c.check(torch)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 7, 65, 140])
def test_attention_sees_nothing(torch, rows, dtype):
    """Rows whose mask leaves nothing, with and without a context, and masks with bits past the rows."""
    c = Case(torch, [0, 37, 0], [rows - 1] * 3, rows + 40, 4, 2, 128, 16, dtype, True, seed=5, reach=1500 * (rows % 3))
    c.mask[0, : rows // 2 + 1] = 0
    c.mask[1, ::2] = 0
    c.mask[:, :, (rows + 31) // 32:] = 0xFFFFFFFF  # nodes that do not exist
    if rows % 32:
        c.mask[:, :, rows // 32] |= np.uint32((0xFFFFFFFF << (rows % 32)) & 0xFFFFFFFF)
    out, lse = c.check(torch)
    assert (out[0, 0] == 0).all() and torch.isneginf(lse[0, 0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [2, 66])
def test_attention_not_a_number(torch, rows, dtype):
    """A stored not-a-number reaches the rows that see it and no other; bytes behind a request's last row
    (unwritten memory) reach none."""
    c = Case(torch, [50, 21], [rows - 1] * 2, rows, 6, 2, 64, 32, dtype, True, seed=9, reach=17000 * (rows % 4 == 2))
    c.mask[:] = 0
    for i in range(rows):
        c.mask[:, i, i // 32] |= np.uint32(1 << (i % 32))
    c.mask[:, 0, 0] |= 2                       # row 0 sees rows 0 and 1; row 1 only itself
    t = 50 + 1
    slot = c.table[0, t // 32] * 32 + t % 32
    c.ref.k[slot, 1] = np.nan
    c.ref.v[slot, 1] = 0
    out, _ = c.check(torch)
    assert torch.isnan(out[0, 0, 3:]).all() and not torch.isnan(out[0, 0, :3]).any()
    assert torch.isnan(out[0, 1, 3:]).all() and not torch.isnan(out[0, 2:]).any() and not torch.isnan(out[1]).any()


def test_attention_unwritten_bytes(torch):
    """Every byte of the cache that holds no row of the request set to 255, infinite scales among them."""
    from paper_2609_22098_amd import kv
    for rows, dtype in ((1, "bf16"), (40, "bf16"), (3, "f32")):
        c = Case(torch, [21, 70], [rows - 1] * 2, rows, 4, 2, 128, 64, dtype, False, seed=2)
        c.ref.k[:], c.ref.v[:] = c.ref.k, c.ref.v
        used = np.zeros(len(c.ref.k), bool)
        for q in range(2):
            pos = np.arange(c.lens[q] + rows)
            used[c.table[q, pos // 64] * 64 + pos % 64] = True
        packed = torch.from_numpy(kv_ref.pack(c.ref)[0].copy()).view(-1, 2, 64 * 136)
        for at, size in ((0, 64), (64 * 64, 4), (64 * 68, 64), (64 * 132, 4)):
            part = packed[:, :, at:at + 64 * size].unflatten(2, (64, size))
            part[~torch.from_numpy(used).view(-1, 64)[:, None, :].expand(-1, 2, -1)] = 255 if size == 64 else 254
        cache = kv.Cache(packed.reshape(1, len(packed), -1).cuda(), 64, 2, 128)
        out, _ = kv.attention(cache, c.q.cuda(), _dev(torch, c.lens), _dev(torch, c.ns), _dev(torch, c.table))
        want, _ = c.run(torch)
        assert torch.equal(out[:, :rows], want[:, :rows])


@pytest.mark.parametrize("rows", [1, 30, 70])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_without_pages(torch, rows, dtype):
    """Positions past the table and page ids that do not exist read as not-a-number, in the rows that see them."""
    c = Case(torch, [100, 64, 10], [rows - 1] * 3, rows, 4, 1, 128, 16, dtype, False, seed=3, reach=40 * rows)
    c.table[0, 2] = len(c.ref.k) // 16       # a page that does not exist
    c.table[1, (64 + rows - 1) // 16] = -1   # the last rows' page is missing
    out, _ = c.check(torch)
    assert torch.isnan(out[0, :rows]).all() and not torch.isnan(out[2, :rows]).any()
    c.table[0, 2] = c.table[0, 1]
    c.lens[2] = 2**31 - 1                    # far past the table
    out, lse = c.run(torch)
    assert torch.isnan(out[2, :rows]).all() and torch.isnan(lse[2, :rows]).all() and not torch.isnan(out[0, :rows]).any()


def test_attention_strides(torch):
    """Queries inside a projection's wider rows, layers inside pages, on another stream, with a given workspace."""
    from paper_2609_22098_amd import kv
    for dtype in ("bf16", "f32"):
        c = Case(torch, [33, 150], [4, 2], 5, 4, 2, 64, 16, dtype, True, seed=4)
        want, _ = c.run(torch)
        wide = torch.randn((2, 5, 11, 64), device="cuda").to(c.t)
        wide[:, :, 3:7] = c.q.cuda()
        packed = torch.from_numpy(kv_ref.pack(c.ref)[0].copy()).cuda()
        pages = torch.randint(0, 256, (len(packed), 3, packed.shape[1] + 32), dtype=torch.uint8, device="cuda")
        pages[:, 1, : packed.shape[1]] = packed
        cache = kv.Cache(pages.transpose(0, 1)[:, :, : packed.shape[1]], 16, 2, 64)
        assert cache.layers == 3
        s = torch.cuda.Stream()
        mask = torch.from_numpy(c.mask.view(np.int32)).cuda()
        args = [_dev(torch, a) for a in (c.lens, c.ns, c.table)]
        ws = torch.empty(max(1, kv.attention_workspace_size(cache, 2, 5, 4, c.t)), dtype=torch.uint8, device="cuda")
        s.wait_stream(torch.cuda.current_stream())
        out, _ = kv.attention(cache, wide[:, :, 3:7], *args, mask=mask, layer=1, workspace=ws, stream=s,
                              out=torch.full_like(want, 99.0))
        s.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_scores(torch, dtype, D):
    """Queries whose elements lie 2^14 apart and whose rows lie 2^120 apart, on one token each: the log-sum-exp is then
    the score itself.  Off by at most what the header states; in fp32 by D + 8 roundings of the sum of magnitudes."""
    from paper_2609_22098_amd import kv
    rng = np.random.default_rng(D)
    R, hq, heads = 48, 6, 2
    ref = kv_ref.Cache(R, 16, heads, D)
    ref.k, ref.v = kv_ref.rounded(rng.standard_normal((R * 16, heads, D)) * 2.0 ** rng.integers(-20, 20, (R * 16, heads, 1)),
                                  rng.standard_normal((R * 16, heads, D)))
    cache = kv.Cache(torch.from_numpy(kv_ref.pack(ref, 1).copy()).cuda(), 16, heads, D)
    q = rng.standard_normal((R, 1, hq, D)) * 2.0 ** rng.integers(-14, 1, (R, 1, hq, D)) * 2.0 ** rng.integers(-60, 60, (R, 1, hq, 1))
    q[0] = 0
    q[1] *= 2.0 ** -50
    q[2, ..., :-1] = 0
    q = torch.from_numpy(q).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    scale = 0.3
    lse = torch.full((R, 1, hq), 99.0, device="cuda")
    zero = _dev(torch, np.zeros(R))
    out, _ = kv.attention(cache, q.cuda(), zero, zero, _dev(torch, np.arange(R)[:, None]), scale=scale, lse=lse)
    x = q.double().numpy()[:, 0].reshape(R, heads, hq // heads, D)
    k = ref.k[::16][:, :, None]
    want = scale * (x * k).sum(-1).reshape(R, hq)
    mag = np.abs(x * k).sum(-1)
    if dtype == "bf16":
        bound = 2.0 ** -15 * mag + 2.0 ** -18 * np.abs(x).max(-1) * np.abs(k).sum(-1)
    else:
        bound = (D + 8) * 2.0 ** -24 * mag
    off = np.abs(lse.double().cpu().numpy()[:, 0] - want) - (scale * bound.reshape(R, hq) + 2.0 ** -22 * np.abs(want) + 1e-30)
    assert off.max() <= 0, (off.max(), np.unravel_index(off.argmax(), off.shape))
    value = np.broadcast_to(ref.v[::16][:, :, None], x.shape).reshape(R, 1, hq, D)  # a weight of 1 on one token
    assert np.array_equal(out.double().cpu().numpy(), value)


def test_attention_many_heads(torch):
    """More elements in a row than 31 bits count (8 GiB of queries): the last heads' as those of a small call."""
    from paper_2609_22098_amd import kv
    heads, group, D = 65536, 256, 256
    small = kv.empty_cache(1, 2, 16, 1, D)
    x = torch.randn((11, 1, D), device="cuda")
    slot = _dev(torch, np.arange(11))
    kv.append(small, x, x.flip(0).contiguous(), slot)
    block = kv.block_bytes(16, D)
    pages = torch.zeros((1, 2, heads * block), dtype=torch.uint8, device="cuda")
    pages[:, :, -block:] = small.pages
    q = torch.zeros((1, 1, heads * group, D), dtype=torch.bfloat16, device="cuda")
    q[:, :, -group:] = torch.randn((group, D), device="cuda").to(torch.bfloat16)
    args = _dev(torch, [10]), _dev(torch, [0]), _dev(torch, [[0]])
    want, _ = kv.attention(small, q[:, :, -group:].contiguous(), *args)
    out, _ = kv.attention(kv.Cache(pages, 16, heads, D), q, *args)
    # other tiles, so other references of the weights: each side off by half a step of outputs and of weights
    off = (out[:, :, -group:].float() - want.float()).abs().max()
    assert off <= 2 * (2.0 ** -8 + 2.0 ** -8) * x.abs().max() and want.abs().min(dim=-1).values.max() > 0
    assert not out[:, :, : heads // 2].any()


def test_rows_of_a_slice(torch):
    """The last row of every request, as a slice leaves it: rows of one, far apart."""
    from paper_2609_22098_amd import kv
    R, cap, H, D = 3, 4, 2, 64
    cache = kv.empty_cache(1, R, 16, H, D)
    table = _dev(torch, np.arange(R)[:, None])
    x = torch.randn((R, cap, 3 * H, D), device="cuda").to(torch.bfloat16)
    last = x[:, -1:]
    slot = _dev(torch, np.arange(R) * 16)
    kv.append(cache, last[:, :, H: 2 * H], last[:, :, 2 * H:], slot)
    k, v = kv.read(cache, slot)
    zero = _dev(torch, np.zeros(R))
    out, _ = kv.attention(cache, last[:, :, :H], zero, zero, table)
    assert torch.equal(out[:, 0], v[0])
    other = kv.empty_cache(1, R, 16, H, D)
    kv.append(other, last[:, 0, H: 2 * H].contiguous(), last[:, 0, 2 * H:].contiguous(), slot)
    assert torch.equal(other.pages, cache.pages)


def test_binding_refusals(torch):
    """Tensors of another type, shape, spacing or place raise before anything is launched."""
    from paper_2609_22098_amd import kv
    R, cap, H, D = 2, 3, 2, 64
    pool = kv.Pool(6, R, 4, 16)
    cache = kv.empty_cache(2, 6, 16, H, D)
    length, n = _dev(torch, [5, 0]), _dev(torch, [2, 1])
    slot, granted = kv.plan(pool, length, n, cap)
    before = cache.pages.clone()
    k = torch.randn((R * cap, H, D), device="cuda")
    q = torch.randn((R, cap, 2 * H, D), device="cuda")
    path, plen = _dev(torch, np.ones((R, 16))), _dev(torch, [1, 0])
    bad = ValueError, TypeError, kv.TreeSparkError

    for name in ("free_pages", "free_count", "held", "table"):
        with pytest.raises(AttributeError):
            setattr(pool, name, None)
    for call in (
            lambda: kv.Pool(6, R, 4, 16, held=pool.held), lambda: kv.Cache(cache.pages.float(), 16, H, D),
            lambda: kv.Cache(cache.pages, 16, H + 1, D), lambda: kv.Cache(cache.pages, 20, H, D),
            lambda: kv.Cache(cache.pages[..., ::2], 16, 1, D), lambda: kv.Cache(cache.pages[0], 16, H, D),
            lambda: kv.plan(pool, length.long(), n, cap), lambda: kv.plan(pool, length, n[:1], cap),
            lambda: kv.plan(pool, length.cpu(), n, cap), lambda: kv.plan(pool, length, n, 0),
            lambda: kv.plan(pool, length, n, cap, out=(slot[:, :2], granted)),
            lambda: kv.append(cache, k, k, slot.view(-1)[:5]), lambda: kv.append(cache, k, k.bfloat16(), slot),
            lambda: kv.append(cache, k.half(), k.half(), slot), lambda: kv.append(cache, k[:, :1], k, slot),
            lambda: kv.append(cache, k, k, slot.t()), lambda: kv.append(cache, k.cpu(), k.cpu(), slot),
            lambda: kv.append(cache, k, k, slot, layer=2), lambda: kv.append(cache, k.transpose(1, 2), k, slot),
            lambda: kv.append(cache, k.view(-1)[1:-127].view(-1, H, D), k[1:], slot.view(-1)[1:]),
            lambda: kv.append(cache, k[::2].expand(2, 3, H, D), k.view(2, 3, H, D), slot),
            lambda: kv.read(cache, slot.long()), lambda: kv.read(cache, slot, layer=1, layers=2),
            lambda: kv.read(cache, slot, dtype=torch.float16), lambda: kv.read(cache, slot, layer=-1, layers=1),
            lambda: kv.read(cache, slot, out=(torch.empty((1, 6, H, D), device="cuda"), None)),
            lambda: kv.attention(cache, q.half(), length, granted, pool.table),
            lambda: kv.attention(cache, q[..., :32], length, granted, pool.table),
            lambda: kv.attention(cache, q[:, :, :3], length, granted, pool.table),
            lambda: kv.attention(cache, q, length[:1], granted, pool.table),
            lambda: kv.attention(cache, q, length, granted, pool.table[:, ::2]),
            lambda: kv.attention(cache, q, length, granted, pool.table[0]),
            lambda: kv.attention(cache, q[:, ::2], length, granted, pool.table),
            lambda: kv.attention(cache, q, length, granted, pool.table, scale=float("nan")),
            lambda: kv.attention(cache, q, length, granted, pool.table, out=q),
            lambda: kv.attention(cache, q, length, granted, pool.table, out=torch.empty_like(q[:1])),
            lambda: kv.attention(cache, q, length, granted, pool.table, lse=torch.empty((R, cap), device="cuda")),
            lambda: kv.attention(cache, q, length, granted, pool.table, workspace=torch.empty(64, dtype=torch.uint8, device="cuda")),
            lambda: kv.attention(cache, q, length, granted, pool.table, mask=torch.zeros((R, cap, 2), dtype=torch.int32, device="cuda")),
            lambda: kv.accept(cache, length, granted, pool.table, path[:, :4], plen),
            lambda: kv.accept(cache, length, granted, pool.table, path, plen, new_length=length),
            lambda: kv.accept(cache, length, granted, pool.table, path, plen, new_length=granted),
            lambda: kv.accept(cache, length, granted, pool.table, path.cpu(), plen)):
        with pytest.raises(bad):
            call()
    torch.cuda.synchronize()
    assert torch.equal(cache.pages, before) and pool.held.tolist() == [1, 1]


def test_attention_far_pages(torch):
    """Pages whose offset passes 32 bits."""
    from paper_2609_22098_amd import kv
    c = Case(torch, [100, 61], [3, 0], 4, 4, 2, 128, 64, "bf16", True, seed=6)
    want, wl = c.run(torch)
    far = 300000  # 300000 pages of 17408 bytes: 5.2 GB
    pages = torch.zeros((1, far, 64 * 136 * 2), dtype=torch.uint8, device="cuda")
    packed = torch.from_numpy(kv_ref.pack(c.ref)[0].copy()).cuda()
    pages[0, far - len(packed):] = packed
    cache = kv.Cache(pages, 64, 2, 128)
    table = np.where(c.table >= 0, c.table + far - len(packed), -1)
    mask = torch.from_numpy(c.mask.view(np.int32)).cuda()
    out, lse = kv.attention(cache, c.q.cuda(), _dev(torch, c.lens), _dev(torch, c.ns), _dev(torch, table), mask=mask,
                            out=torch.full_like(want, 99.0), lse=torch.full_like(wl, 99.0))
    assert torch.equal(out, want) and torch.equal(lse, wl)
    slot = _dev(torch, np.arange(64) + (far - 1) * 64)
    x = torch.randn((64, 2, 128), device="cuda")
    kv.append(cache, x, x, slot)
    k, v = kv.read(cache, slot, dtype=torch.float32)
    assert torch.equal(k, v) and k.abs().sum() > 0


def test_attention_large_scores(torch):
    """Scores of some hundreds: weights that vanish, maxima that rise late, in an order of either kind."""
    for dtype in ("bf16", "f32"):
        for rows in (1, 40, 70):
            c = Case(torch, [700], [rows - 1], rows, 4, 2, 128, 16, dtype, False, seed=8, kscale=12.0, reach=17000 * (rows != 40))
            c.check(torch)
            # keys that grow along the context, so that every tile raises the maximum
            c.ref.k *= np.exp2(np.minimum(np.arange(len(c.ref.k)) // 100, 6) - 6.0)[:, None, None]
            c.check(torch)
            c.q[:] = c.q.abs()
            c.ref.k[:] = np.abs(c.ref.k)
            c.check(torch)
            c.scale = -c.scale
            c.check(torch)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,reach", [(1, 0), (1, 17000), (40, 0), (40, 17000), (300, 0)])
def test_attention_one_hot(torch, rows, reach, dtype):
    """Scores of 1e13, where fp32 steps by a million: the one token twice above the others has all the weight, early in
    the context or behind keys that grow, and the outputs are its value."""
    for star, grows in ((137, False), (599, True)):
        c = Case(torch, [600], [rows - 1], rows, 4, 1, 128, 64, dtype, False, seed=rows, reach=reach)
        token = np.full(len(c.ref.k), 2.0 ** -20)
        pos = np.arange(600)
        slot = c.table[0, pos // 64] * 64 + pos % 64
        token[slot] = 2.0 ** (pos // 64 - 12) if grows else 1.0
        token[slot[star]] = 4.0
        c.ref.k = kv_ref.rounded(token[:, None, None] * np.ones_like(c.ref.k), c.ref.v)[0]
        c.q[:] = c.q.abs() + 0.5
        c.scale = 1e10
        out, lse = c.run(torch)
        want = np.broadcast_to(c.ref.v[slot[star], 0], out.shape)
        assert np.array_equal(out.double().cpu().numpy(), want)
        score = c.scale * 4.0 * c.q.double().sum(-1).numpy()
        assert (np.abs(lse.double().cpu().numpy() - score) <= 2.0 ** -14 * score).all()


# ---------------------------------------------------------------- accepted rows


@pytest.mark.parametrize("R,heads,D,page,layers", [(1, 1, 64, 16, 1), (6, 2, 128, 16, 3), (9, 8, 128, 64, 2), (5, 3, 256, 32, 2),
                                                   (70, 1, 64, 256, 1)])
def test_accept(torch, R, heads, D, page, layers):
    """Rows move in every layer and head and nothing else changes; broken paths stop where they break."""
    from paper_2609_22098_amd import kv
    rng = np.random.default_rng(R)
    cap, blocks = 40, -(-(130 + 40) // page) + 1
    length, n = rng.integers(0, 130, R), rng.integers(0, cap, R)
    need = -(-(length + n + 1) // page)
    ids = rng.permutation(int(need.sum()) + 1)
    table = np.full((R, blocks), -1, np.int64)
    table[np.arange(blocks) < need[:, None]] = ids[: need.sum()]
    nodes, count = np.zeros((R, 16), np.int64), np.zeros(R, np.int64)
    for q in range(R):
        count[q] = min(rng.integers(0, 17), n[q])
        nodes[q, : count[q]] = 1 + np.sort(rng.permutation(n[q])[: count[q]])
    kept = count.copy()
    if R > 4:
        n[0], nodes[0, :4], count[0], kept[0] = 9, [2, 2, 3, 4], 4, 1      # not larger than the one before
        length[0] = 0
        nodes[1, :2], count[1], kept[1] = [n[1] + 1, n[1] + 2], 2, 0       # past the tree
        count[2], kept[2] = -1, -1                                         # sat out
        n[3], kept[3] = -1, -1
        count[4], kept[4] = min(int(n[4]), 16), min(int(n[4]), 16)
        nodes[4, : count[4]] = np.arange(1, count[4] + 1)
        need0 = -(-(length + np.maximum(n, 0) + 1) // page)
        table[0] = -1
        table[0, : min(need0[0], need[0])] = ids[: min(need0[0], need[0])]
        if need0[0] > need[0]:
            kept[0] = 1 if (2 // page) < need[0] else 0
    pages = torch.randint(0, 256, (layers, len(ids), heads * page * D * 17 // 16), dtype=torch.uint8, device="cuda")
    want = pages.cpu().numpy().copy()
    a, b = page * D // 2, page * D // 32
    for q in range(R):
        for j in range(max(kept[q], 0)):
            s, d = length[q] + nodes[q, j], length[q] + 1 + j
            sp, dp = table[q, s // page], table[q, d // page]
            for h in range(heads):
                base = h * page * D * 17 // 16
                for lo, size in ((0, D // 2), (a, D // 32), (a + b, D // 2), (2 * a + b, D // 32)):
                    f, t = base + lo + s % page * size, base + lo + d % page * size
                    want[:, dp, t:t + size] = want[:, sp, f:f + size]
    cache = kv.Cache(pages, page, heads, D)
    new = kv.accept(cache, _dev(torch, length), _dev(torch, n), _dev(torch, table), nodes.astype(np.int32), count.astype(np.int32))
    assert np.array_equal(new.cpu().numpy(), np.where(kept >= 0, length + 1 + kept, length))
    assert np.array_equal(pages.cpu().numpy(), want)


def test_accept_without_pages(torch):
    """A path stops at a row whose old or new place lies in no page."""
    from paper_2609_22098_amd import kv
    cache = kv.empty_cache(1, 4, 16, 1, 64)
    table = _dev(torch, [[0, 9, 1], [2, 3, -1]])
    nodes, count = np.zeros((2, 16), np.int32), np.array([3, 3], np.int32)
    nodes[0, :3], nodes[1, :3] = [1, 6, 20], [1, 17, 30]
    new = kv.accept(cache, _dev(torch, [10, 12]), _dev(torch, [39, 39]), table, nodes, count)
    assert new.tolist() == [12, 15]  # rows 6 (position 16, page 9) and 30 (position 42, no page) end the paths
    new = kv.accept(cache, _dev(torch, [2**31 - 1, -5]), _dev(torch, [39, -1]), table, nodes, np.array([0, 0], np.int32))
    assert new[1].item() == -5


# ---------------------------------------------------------------- a round


def test_rounds_with_trees(torch):
    """Three rounds as a serving loop has them: trees, their mask, plan, append, attention, accept, on lengths
    that stay on the GPU; the attention of each round equals the oracle over the rows that were kept."""
    from paper_2609_22098_amd import binding as b
    from paper_2609_22098_amd import kv
    rng = np.random.default_rng(1)
    R, cap, hq, hk, D, page, layers = 5, 20, 4, 2, 64, 16, 2
    pool = kv.Pool(60, R, 12, page)
    cache = kv.empty_cache(layers, 60, page, hk, D)
    length = torch.zeros((R,), dtype=torch.int32, device="cuda")
    hist = [[(np.zeros((0, hk, D)), np.zeros((0, hk, D))) for _ in range(R)] for _ in range(layers)]
    for _ in range(3):
        n = rng.integers(-1, cap, R)
        parent = np.full((R, cap), -1, np.int32)
        for q in range(R):
            for i in range(1, n[q] + 1):
                parent[q, i] = rng.integers(0, i)
        path, plen = np.zeros((R, 16), np.int32), np.zeros(R, np.int32)
        for q in range(R):
            if n[q] < 0:
                plen[q] = -1
                continue
            node, depth = 0, 0
            while depth < 16:
                kids = [i for i in range(1, n[q] + 1) if parent[q, i] == node]
                if not kids:
                    break
                node = int(rng.choice(kids))
                path[q, depth] = node
                depth += 1
            plen[q] = depth
        qkv = [torch.randn((R, cap, hq + 2 * hk, D), device="cuda").bfloat16() for _ in range(layers)]
        mask, pos = b.tree_mask(_dev(torch, parent), _dev(torch, n), cap, length)
        slot, granted = kv.plan(pool, length, _dev(torch, n), cap)
        assert np.array_equal(granted.cpu().numpy(), n)
        outs = []
        for layer in range(layers):
            x = qkv[layer]
            kv.append(cache, x[:, :, hq:hq + hk], x[:, :, hq + hk:], slot, layer=layer)
            outs.append(kv.attention(cache, x[:, :, :hq], length, granted, pool.table, mask=mask, layer=layer)[0])
        new = kv.accept(cache, length, granted, pool.table, path, plen)
        bits = mask.cpu().numpy().view(np.uint32)
        for layer in range(layers):
            x = qkv[layer].double().cpu().numpy()
            for q in range(R):
                rows = n[q] + 1
                if not rows:
                    continue
                k0, v0 = hist[layer][q]
                kn, vn = kv_ref.rounded(x[q, :rows, hq:hq + hk], x[q, :rows, hq + hk:])
                k, v = np.concatenate([k0, kn]), np.concatenate([v0, vn])
                see = kv_ref.sees(len(k0), rows, len(k), bits[q])
                want, _, mass, mag = kv_ref.attention(x[q, :rows, :hq], k, v, see, D ** -0.5)
                d = np.expm1(2 * mag * 2.0 ** -15)[..., None]
                got = outs[layer][q, :rows].double().cpu().numpy()
                assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -16 + d) * mass + 1e-30).all()
                keep = [0] + [int(i) for i in path[q, : plen[q]]]
                hist[layer][q] = np.concatenate([k0, kn[keep]]), np.concatenate([v0, vn[keep]])
        length = new
        assert length.tolist() == [len(hist[0][q][0]) for q in range(R)]
    kv.plan(pool, length, _dev(torch, [-1] * R), cap, slots=False)
    assert pool.held.tolist() == [-(-int(x) // page) for x in length.tolist()]
    kv.plan(pool, torch.zeros_like(length), _dev(torch, [-1] * R), cap, slots=False)
    assert int(pool.free_count) == 60 and sorted(pool.free_pages.tolist()) == list(range(60))


def test_round_in_a_graph(torch):
    """A round captured once and replayed on new inputs in the same tensors equals the same calls made eagerly,
    with eager work between the replays; the same call gives the same bits."""
    from paper_2609_22098_amd import kv
    rng = np.random.default_rng(2)
    R, cap, hq, hk, D, page = 4, 33, 8, 2, 128, 16
    st = {k: _dev(torch, v) for k, v in dict(length=[0] * R, n=[0] * R, path=np.zeros((R, 16)), plen=[0] * R).items()}
    st["qkv"] = torch.zeros((R, cap, hq + 2 * hk, D), dtype=torch.bfloat16, device="cuda")
    st["mask"] = torch.zeros((R, cap, 2), dtype=torch.int32, device="cuda")
    pools = [kv.Pool(400, R, 60, page) for _ in range(2)]
    caches = [kv.empty_cache(1, 400, page, hk, D) for _ in range(2)]
    outs = [torch.zeros((R, cap, hq, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]

    def step(i):
        pool, cache, x = pools[i], caches[i], st["qkv"]
        slot, granted = kv.plan(pool, st["length"], st["n"], cap)
        kv.append(cache, x[:, :, hq:hq + hk], x[:, :, hq + hk:], slot)
        kv.attention(cache, x[:, :, :hq], st["length"], granted, pool.table, mask=st["mask"], out=outs[i])
        return kv.accept(cache, st["length"], granted, pool.table, st["path"], st["plen"])

    graph = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        new = step(0)
    length = np.zeros(R, np.int64)
    for r in range(5):
        n = rng.integers(0, cap, R) if r else np.full(R, cap - 1)
        mask = np.zeros((R, cap, 2), np.uint32)
        plen = np.minimum(n, 3)
        for q in range(R):
            mask[q, : n[q] + 1] = kv_ref.tree_bits([-1] + [int(rng.integers(0, i)) for i in range(1, n[q] + 1)], n[q] + 1, 2)
        st["length"].copy_(_dev(torch, length))
        st["n"].copy_(_dev(torch, n))
        st["plen"].copy_(_dev(torch, plen))
        st["path"].copy_(_dev(torch, np.tile(np.arange(1, 17), (R, 1)) + (np.arange(16) == 2) * (plen == 3)[:, None] * (n > 3)[:, None]))
        st["mask"].copy_(torch.from_numpy(mask.view(np.int32)))
        st["qkv"].normal_()
        torch.cuda.synchronize()
        graph.replay()
        eager = step(1)
        torch.cuda.synchronize()
        assert torch.equal(new, eager) and torch.equal(outs[0], outs[1])
        assert torch.equal(caches[0].pages, caches[1].pages) and torch.equal(pools[0].table, pools[1].table)
        length = length + 1 + plen + (37 * r if r < 2 else 0)  # some contexts jump ahead, over rows never written
        assert outs[0].isfinite().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_calls_at_once_and_a_shared_workspace(torch, dtype):
    """Calls in flight on two streams, each with a workspace; two captured graphs of other sizes that share one and are
    replayed in turn: the bits of the same calls alone."""
    from paper_2609_22098_amd import kv
    calls = []
    for seed, (lens, n, cap, hq, heads, page, reach) in enumerate([
            ([7000, 2100], [16, 3], 17, 8, 2, 64, 0), ([3000] * 20, [64] * 20, 65, 8, 2, 16, 4000)]):
        c = Case(torch, lens, n, cap, hq, heads, 128, page, dtype, True, seed=seed, reach=reach)
        want, _ = c.run(torch)
        cache = kv.Cache(torch.from_numpy(kv_ref.pack(c.ref, 1).copy()).cuda(), page, heads, 128)
        args = [_dev(torch, a) for a in (c.lens, c.ns, c.table)]
        kw = dict(mask=torch.from_numpy(c.mask.view(np.int32)).cuda(), scale=c.scale)
        size = kv.attention_workspace_size(cache, len(lens), cap, hq, c.t)
        calls.append((cache, c.q.cuda(), args, kw, want, size))
    streams = [torch.cuda.Stream() for _ in calls]
    own = [torch.empty(size, dtype=torch.uint8, device="cuda") for *_, size in calls]
    outs = [[torch.full_like(want, 99.0) for _ in range(6)] for *_, want, _ in calls]
    torch.cuda.synchronize()
    for r in range(6):
        for i, (cache, q, args, kw, _, _) in enumerate(calls):
            kv.attention(cache, q, *args, out=outs[i][r], workspace=own[i], stream=streams[i], **kw)
    torch.cuda.synchronize()
    for i, (*_, want, _) in enumerate(calls):
        assert all(torch.equal(o, want) for o in outs[i])

    shared = torch.empty(max(size for *_, size in calls), dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for cache, q, args, kw, want, _ in calls:
        out, graph = torch.full_like(want, 99.0), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=streams[0]):
            kv.attention(cache, q, *args, out=out, workspace=shared, **kw)
        graphs.append(graph)
        outs.append(out)
    for r in range(4):
        for i in (0, 1, 0) if r % 2 else (1, 0):
            outs[i].fill_(99.0)
            graphs[i].replay()
        torch.cuda.synchronize()
        for i, (*_, want, _) in enumerate(calls):
            assert torch.equal(outs[i], want)
