"""The cache attention at the ends of what its header allows: scores whose products the matrix unit cuts off most,
numbers near the ends of their types.  Oracles are plain numpy in 64 bits."""
import numpy as np
import pytest

import kv_ref
from test_gpu_kv import Case

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


def _one_token(torch, q, k, scale, dtype):
    """Query heads q [R][hq][D] on one token each, keys k [R][heads][D] (values of the format): the log-sum-exp, which is
    the score, and the output over values of ones."""
    from paper_2609_22098_amd import kv
    R, hq, D = q.shape
    heads = k.shape[1]
    ref = kv_ref.Cache(R, 16, heads, D)
    ref.k[::16], ref.v[:] = k, 1.0
    cache = kv.Cache(torch.from_numpy(kv_ref.pack(ref, 1).copy()).cuda(), 16, heads, D)
    q = torch.from_numpy(q[:, None]).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()
    lse = torch.full((R, 1, hq), 99.0, device="cuda")
    zero = _dev(torch, np.zeros(R))
    out, _ = kv.attention(cache, q, zero, zero, _dev(torch, np.arange(R)[:, None]), scale=scale, lse=lse)
    return lse.double().cpu().numpy()[:, 0], out.double().cpu().numpy()[:, 0]


# ---------------------------------------------------------------- products that are cut off


# (query, key) of the largest of eight neighbouring elements, and of the seven others: a query that rounds up to the next
# power of two where it is held in 4 bits, beside the least that those bits show; a product 2^13 above its neighbours;
# queries that leave as much as one can to their second part, beside products just too small for that; and two that
# round up beside such.
DOMINATED = [((3.90625, 6.0), (2.0 ** -9, 0.5)), ((3.5, 6.0), (2.0 ** -9, 1.0)), ((2.125, 4.0), (1.875 * 2.0 ** -15, 1.0)),
             ((3.125, 4.0), (1.875 * 2.0 ** -15, 1.0)), ((1.9375, 6.0), (1.875 * 2.0 ** -10, 0.5)),
             ((3.96875, 4.0), (1.75 * 2.0 ** -14, 1.5))]


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("case", range(len(DOMINATED)))
def test_scores_with_one_large_product_in_eight(torch, case, D):
    """One channel of queries and keys far above its neighbours, in one group of eight or in all.  Off by at most what
    the header states: of eight products the matrix unit cuts off what lies below 2^-13 of the largest's power of
    two.  The first part of a query loses nothing of that; the second, at most 2^-4 of an element, less than 7 * 2^-17 of
    the largest |Q| |K| of the eight; 64 sums in 32 bits add 64 * 2^-24 of all."""
    (q0, k0), (q1, k1) = DOMINATED[case]
    rng = np.random.default_rng(case)
    R, heads, group = 32, 2, 2
    at = rng.integers(0, 8, (R, heads, D // 8, 1))  # the large one's place among its eight
    large = np.arange(8) == at
    some = rng.random((R, heads, D // 8, 1)) < np.where(np.arange(R) % 2, 1.0, 0.1)[:, None, None, None]
    some[:, :, 0] = True
    k = np.where(large & some, k0, k1).reshape(R, heads, D)
    q = np.where(large & some, q0, q1).reshape(R, heads, 1, D) * np.array([1.0, -0.125])[:, None]
    sign = np.where(rng.random((R, heads, D)) < np.where(np.arange(R) % 4 < 2, 0.0, 0.5)[:, None, None], -1.0, 1.0)
    k, q = k * sign, q * sign[:, :, None]  # products of one sign: what is cut off adds up
    q = q * 2.0 ** rng.integers(-20, 20, (R, 1, 1, 1))
    scale = 0.25
    got, _ = _one_token(torch, q.reshape(R, heads * group, D), k, scale, "bf16")
    want = scale * (q * k[:, :, None]).sum(-1).reshape(R, -1)
    mag = np.abs(q * k[:, :, None]).sum(-1).reshape(R, -1)
    held = (np.abs(q).max(-1) * np.abs(k[:, :, None]).sum(-1)).reshape(R, -1)
    bound = scale * (2.0 ** -14 * mag + 2.0 ** -18 * held) + 2.0 ** -22 * np.abs(want)
    over = np.abs(got - want) / bound
    assert over.max() <= 1, (over.max(), np.unravel_index(over.argmax(), over.shape))


# ---------------------------------------------------------------- the ends of the types


# Exponents of queries, keys and the scale: a scale times a query, and a query scaled to one times a key, that pass fp32
# where the score does not; queries and keys next to the largest and the least of their types.
FAR = [(30, -123, 100), (-100, 122, -18), (127, -123, 0), (-118, 122, 0), (-126, 100, 30), (60, -20, -36), (-60, -20, 84),
       (100, -110, 20), (-133, 122, 15), (-126, 122, 4)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 256])
@pytest.mark.parametrize("case", range(len(FAR)))
def test_scores_of_far_exponents(torch, case, D, dtype):
    """Scores of ordinary size from queries, keys and scales that are far from it; <Q, K> itself is an fp32 number.  The
    bounds are the header's, and in fp32 D + 8 roundings of the sum of magnitudes."""
    eq, ek, es = FAR[case]
    rng = np.random.default_rng(case)
    R, heads, group = 16, 2, 3
    q = rng.integers(-127, 128, (R, heads, group, D)) / 64.0
    q[..., 3] = 127 / 64  # the largest, in bf16 too; whole steps of the least subnormal at 2^-133 are few
    q = np.rint(q) if eq < -126 else q
    k = kv_ref.rounded(rng.standard_normal((R, heads, D)) * 2.0 ** (ek - 1), np.ones((R, heads, D)))[0]
    same = (np.arange(R) % 2 == 0)[:, None, None, None]  # half of the rows: products of one sign
    q, scale = np.where(same, np.abs(q) * np.sign(k)[:, :, None], q) * 2.0 ** eq, 2.0 ** es * -0.75
    got, out = _one_token(torch, q.reshape(R, heads * group, D), k, scale, dtype)
    want = scale * (q * k[:, :, None]).sum(-1).reshape(R, -1)
    mag = np.abs(q * k[:, :, None]).sum(-1).reshape(R, -1)
    held = (np.abs(q).max(-1) * np.abs(k[:, :, None]).sum(-1)).reshape(R, -1)
    bound = 2.0 ** -14 * mag + 2.0 ** -18 * held if dtype == "bf16" else (D + 8) * 2.0 ** -24 * mag
    over = np.abs(got - want) / (abs(scale) * bound + 2.0 ** -22 * np.abs(want))
    assert over.max() <= 1, (over.max(), np.unravel_index(over.argmax(), over.shape))
    assert (out == 1).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 30, 70])
def test_queries_that_are_not_finite(torch, rows, dtype):
    """A query with an infinity or a not-a-number gives not-a-number, and no other row is touched by it."""
    from paper_2609_22098_amd import kv
    rng = np.random.default_rng(rows)
    heads, hq, D, context = 2, 6, 128, 90
    ref = kv_ref.Cache(-(-(context + rows) // 16), 16, heads, D)
    ref.k, ref.v = kv_ref.rounded(rng.standard_normal(ref.k.shape), rng.standard_normal(ref.v.shape))
    cache = kv.Cache(torch.from_numpy(kv_ref.pack(ref, 1).copy()).cuda(), 16, heads, D)
    table = _dev(torch, np.arange(len(ref.k) // 16)[None])
    q = torch.from_numpy(rng.standard_normal((1, rows, hq, D))).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    args = _dev(torch, [context]), _dev(torch, [rows - 1]), table

    def run(x):
        lse = torch.full((1, rows, hq), 99.0, device="cuda")
        out, _ = kv.attention(cache, x.cuda(), *args, lse=lse)
        return out, lse

    want, wl = run(q)
    bad = torch.zeros((1, rows, hq), dtype=torch.bool)
    for i, (at, x) in enumerate(((5, float("inf")), (127, -float("inf")), (64, float("nan")))):
        q[0, rows // 2, 2 * i, at] = x
        bad[0, rows // 2, 2 * i] = True
    out, lse = run(q)
    bad = bad.cuda()
    assert torch.isnan(out[bad]).all() and torch.isnan(lse[bad]).all()
    assert torch.equal(out[~bad], want[~bad]) and torch.equal(lse[~bad], wl[~bad])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-37, -1e-37, 1e-45])
@pytest.mark.parametrize("rows,reach", [(1, 0), (1, 17000), (40, 0), (70, 0), (70, 17000)])
def test_scales_next_to_zero(torch, rows, reach, scale, dtype):
    """Keys near 1e35 under a scale of zero weigh alike, under one of 1e-37 by their scores of about one; what the mask
    hides has no weight under either."""
    c = Case(torch, [100, 0], [rows - 1, max(rows - 3, 0)], rows, 4, 2, 128, 16, dtype, True, seed=rows, reach=reach, kscale=1e35)
    c.scale = scale
    c.check(torch)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_largest_fp32_queries(torch, D):
    """fp32 queries up to the type's largest number, which bf16, a part of them, would round to infinity."""
    rng = np.random.default_rng(D)
    R, heads, group = 8, 2, 3
    top = float(np.finfo(np.float32).max)
    q = rng.choice([top, -top, 3.4e38, 3.397e38, -3.3961775e38, 1.0, -3e38], (R, heads, group, D))
    q = q.astype(np.float32).astype(np.float64)
    k = kv_ref.rounded(rng.standard_normal((R, heads, D)) * 2.0 ** -110, np.ones((R, heads, D)))[0]
    scale = 2.0 ** -15
    got, out = _one_token(torch, q.reshape(R, heads * group, D), k, scale, "f32")
    want = scale * (q * k[:, :, None]).sum(-1).reshape(R, -1)
    mag = scale * np.abs(q * k[:, :, None]).sum(-1).reshape(R, -1)
    over = np.abs(got - want) / ((D + 8) * 2.0 ** -24 * mag + 2.0 ** -22 * np.abs(want))  # fp32 sums of D products
    assert over.max() <= 1, (over.max(), np.unravel_index(over.argmax(), over.shape))
    assert (out == 1).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,rows,reach", [(1, 1, 0), (1, 1, 17000), (1, 40, 17000), (90, 70, 0), (90, 70, 17000), (40, 300, 17000)])
@pytest.mark.parametrize("far", [32, 64, 200, 500])
def test_scores_of_minus_infinity(torch, far, R, rows, reach, dtype):
    """The first tokens' scores pass fp32 and are -inf, which is a weight of zero; the others', however low, have all of
    it, in one step of a workgroup or in many."""
    c = Case(torch, [501] * R, [rows - 1] * R, rows, 4, 1, 64, 16, dtype, False, seed=far, reach=reach)
    pos = np.arange(501 + rows)
    slot = c.table[:, pos // 16] * 16 + pos % 16
    c.q[:] = c.q.abs() + 0.5
    key = np.where(pos < far, -(2.0 ** 33), -(2.0 ** -95) * (1 + pos % 3))
    c.ref.k[slot] = key[:, None, None]
    c.scale = 2.0 ** 100
    out, lse = c.run(torch)
    for q in (0, R - 1):
        k, v = c.rows_of(q, 501 + rows)
        see = kv_ref.sees(501, rows, 501 + rows)[:, far:]
        want, wl, mass, mag = kv_ref.attention(c.q[q].double().numpy(), k[far:], v[far:], see, c.scale)
        assert np.isfinite(wl).all() and wl.max() < -1000
        got, gl = out[q].double().cpu().numpy(), lse[q].double().cpu().numpy()
        # a key's elements are alike, so max |Q| sum |K| is sum |Q| |K| times the largest |Q| (of 1.4 million normal
        # numbers: below 7.5 + 0.5) over their mean (above 0.5), under 16: a score is off by what the header states of
        # these, in fp32 by 72 roundings
        d = mag * (2.0 ** -14 + 2.0 ** -18 * 16 if dtype == "bf16" else 72 * 2.0 ** -24)
        small = (501 + rows + 16) * 2.0 ** -24 + 2.0 ** -22
        assert (np.abs(gl - wl) <= d + small + 2.0 ** -22 * np.abs(wl)).all()
        half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
        weight = (half if dtype == "bf16" else 0) + small
        assert (np.abs(got - want) <= half * np.abs(want) + (np.expm1(2 * d)[..., None] + weight) * mass + 1e-30).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,rows,reach", [(1, 1, 17000), (1, 40, 0), (90, 70, 0), (40, 300, 17000)])
def test_scores_of_plus_infinity(torch, R, rows, reach, dtype):
    """One token whose scores pass fp32 makes not-a-number of the rows that see it and of no other; where every score
    of a row is -inf the row gives what one that sees nothing gives."""
    c = Case(torch, [400] * R, [rows - 1] * R, rows, 4, 1, 64, 16, dtype, False, seed=rows, reach=reach)
    c.q[:] = c.q.abs() + 0.5
    c.scale = 2.0 ** 100
    pos = np.arange(400 + rows)
    slot = c.table[:, pos // 16] * 16 + pos % 16
    c.ref.k[slot] = -(2.0 ** -95)
    c.ref.k[slot[0, 400 + rows // 2]] = 2.0 ** 33
    c.ref.k[slot[R - 1, : 400 + rows // 2]] = -(2.0 ** 33) if R > 1 else -(2.0 ** -95)
    out, lse = c.run(torch)
    sees = torch.arange(rows, device="cuda") >= rows // 2
    assert torch.isnan(out[0, sees]).all() and torch.isnan(lse[0, sees]).all()
    assert out[0, ~sees].isfinite().all() and lse[0, ~sees].isfinite().all() and out[1 : R - 1].isfinite().all()
    if R > 1:
        assert (out[R - 1, ~sees] == 0).all() and torch.isneginf(lse[R - 1, ~sees]).all()
        assert out[R - 1, sees].isfinite().all() and lse[R - 1, sees].isfinite().all()
