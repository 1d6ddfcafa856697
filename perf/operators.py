"""The target's 4-bit key-value cache around a draft tree: performance cases of its operators.

A round of speculative decoding gives every row of the round's trees a place in the target's paged cache
(`plan`), writes the rows' keys and values there in 4 bits (`append`), attends over context and tree under
the tree mask (`attend`), and keeps the accepted path's rows (`accept`).  Each case is one of these steps,
with what a serving program keeps (cache, block tables, masks, output buffers) made in prepare().

The cache is [layers][pages][heads][block] bytes.  A block holds one kv head of a page of P tokens, D values
each: key codes [P][D/2], key scales [P][D/32], value codes [P][D/2], value scales [P][D/32].  A code is
E2M1 (element d of a token in byte d / 2, the low half for even d), a scale byte s stands for 2^(s - 127)
and covers 32 values; 255 makes keys not-a-number and values zero.
"""
import math

import numpy as np
import torch

own = False

PATH = 16  # most accepted nodes of a round


def listed():
    return [
        # one interactive user: the tree's rows after a context of some thousand tokens; latency counts
        dict(name="plan-single", kind="plan", R=1, cap=65, lo=3001, hi=3001, nlo=64, nhi=64, page=64, blocks=128),
        # high load: 256 requests, a chunk of a prompt or a round's tree each, the largest slot map
        dict(name="plan-wave", kind="plan", R=256, cap=2049, lo=100, hi=30000, nlo=0, nhi=2048, page=16, blocks=2048),
        # one layer's new rows of 32 requests that decode without a tree
        dict(name="append-tokens", kind="append", dtype="bf16", R=32, cap=1, lo=64, hi=2000, nlo=0, nhi=0, heads=8,
             D=128, page=64),
        # one layer's rows of a long prompt, as its chunk is read in
        dict(name="append-prompt", kind="append", dtype="bf16", R=4, cap=4096, lo=0, hi=1000, nlo=4095, nhi=4095,
             heads=8, D=128, page=64),
        # the accepted rows of one user's tree, in every layer
        dict(name="accept-single", kind="accept", R=1, cap=65, lo=700, hi=700, nlo=64, nhi=64, layers=16, heads=8,
             D=128, page=64),
        # the accepted rows of a serving batch, in every layer
        dict(name="accept-serving", kind="accept", R=64, cap=65, lo=20, hi=300, nlo=16, nhi=64, layers=32, heads=8,
             D=128, page=64),
        # a small model kept in 32 bits, a head of keys for each of queries, pages of 16: the smallest attention
        dict(name="attend-f32", kind="attend", dtype="f32", R=3, cap=33, lo=50, hi=700, nlo=5, nhi=32, hq=12, heads=12,
             D=64, page=16, tree=True),
        # one interactive user: a full tree of 64 nodes over a few thousand tokens
        dict(name="attend-single", kind="attend", dtype="bf16", R=1, cap=65, lo=5003, hi=5003, nlo=64, nhi=64, hq=32,
             heads=8, D=128, page=64, tree=True),
        # one user, one token, a context of a whole book: the work is split over the context
        dict(name="attend-long", kind="attend", dtype="bf16", R=1, cap=1, lo=131001, hi=131001, nlo=0, nhi=0, hq=32,
             heads=8, D=128, page=64, tree=False),
        # a batch that decodes without trees (the price ladder's chain at its shortest), ragged contexts
        dict(name="attend-tokens", kind="attend", dtype="bf16", R=128, cap=1, lo=300, hi=16000, nlo=0, nhi=0, hq=32,
             heads=8, D=128, page=16, tree=False),
        # the serving batch's verification: 64 requests, trees of 8 to 64 nodes, ragged contexts
        dict(name="attend-serving", kind="attend", dtype="bf16", R=64, cap=65, lo=500, hi=8000, nlo=8, nhi=64, hq=32,
             heads=8, D=128, page=64, tree=True),
        # two prompts' chunks over what was read before them, causal
        dict(name="attend-prompt", kind="attend", dtype="bf16", R=2, cap=4096, lo=2000, hi=4100, nlo=4000, nhi=4095,
             hq=32, heads=8, D=128, page=64, tree=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "append", "accept", "attend", "attend", "attend"])
    page = rng.choice([16, 32, 64, 128])
    D = rng.choice([64, 128, 128, 128])
    if kind == "plan":
        R, cap = _log_int(rng, 1, 256), _log_int(rng, 1, 2049)
        hi = _log_int(rng, 100, 30000)
        return dict(kind=kind, R=R, cap=cap, lo=max(0, hi // rng.choice([1, 10, 200])), hi=hi,
                    nlo=rng.choice([0, cap - 1]), nhi=cap - 1, page=page,
                    blocks=-(-(hi + cap + 40) // page) + rng.randrange(9))
    if kind == "append":
        R, cap = _log_int(rng, 1, 64), _log_int(rng, 1, 1024)
        cap = max(1, min(cap, 16384 // R))
        return dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]), R=R, cap=cap, lo=0, hi=_log_int(rng, 1, 2000),
                    nlo=rng.choice([0, cap - 1]), nhi=cap - 1, heads=rng.choice([1, 2, 4, 5, 8]), D=D, page=page)
    if kind == "accept":
        R, cap = _log_int(rng, 1, 64), _log_int(rng, 2, 129)
        return dict(kind=kind, R=R, cap=cap, lo=1, hi=_log_int(rng, 10, 300), nlo=rng.choice([0, cap - 1]), nhi=cap - 1,
                    layers=_log_int(rng, 1, 32), heads=rng.choice([1, 2, 4, 8]), D=D, page=page)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    heads = rng.choice([1, 2, 4, 8])
    hq = heads * rng.choice([1, 2, 3, 4, 4, 7, 8])
    shape = rng.choice(["token", "tree", "prompt"])
    if shape == "token":  # single tokens: many short contexts or few long ones
        R = _log_int(rng, 1, 128)
        hi = _log_int(rng, 64, min(131072, 1200000 // R))
        cap = 1
    elif shape == "tree":
        R, cap = _log_int(rng, 1, 64), _log_int(rng, 2, 129)
        hi = max(40, min(_log_int(rng, 64, 16000), 200_000_000 // (R * cap * hq)))
    else:  # a prompt's chunk
        R, cap = rng.choice([1, 1, 2, 3]), _log_int(rng, 130, 4096)
        hi = _log_int(rng, 16, 4100)
        while R * cap * hq * (hi + cap) > 2_000_000_000:
            cap, hi = cap * 3 // 4, hi * 3 // 4
    if dtype == "f32":
        hi = max(16, hi // 2)
    return dict(kind="attend", dtype=dtype, R=R, cap=cap, lo=max(0, hi // rng.choice([1, 3, 20])), hi=hi,
                nlo=rng.choice([0, cap // 2, cap - 1]) if shape == "tree" else cap - 1, nhi=cap - 1, hq=hq, heads=heads,
                D=D, page=page, tree=shape == "tree")


# ---------------------------------------------------------------- inputs


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _lengths(c):
    """Context lengths, spread evenly over their logarithm, and nodes per request, spread evenly: the case's
    alone, so that its work is known; prepare() deals them out by its seed."""
    at = np.linspace(0.0, 1.0, c["R"]) if c["R"] > 1 else np.ones(1)
    length = np.rint((c["lo"] + 1.0) ** (1 - at) * (c["hi"] + 1.0) ** at - 1).astype(np.int64)
    return length, np.rint(c["nlo"] + at * (c["nhi"] - c["nlo"])).astype(np.int64)


def _paths(R, n, rng):
    """Accepted paths: increasing nodes, of uneven lengths, some empty."""
    nodes, count = np.zeros((R, PATH), np.int64), np.zeros(R, np.int64)
    for q in range(R):
        count[q] = min(int(n[q]), int(rng.integers(0, PATH + 1)) if R > 1 else 9)
        nodes[q, :count[q]] = 1 + np.sort(rng.permutation(int(n[q]))[:count[q]])
    return nodes, count


def _tree_masks(R, cap, n, rng):
    """Masks of random trees: bit j of row i is set where node j is i or one of its ancestors."""
    sees = np.zeros((R, cap, cap), bool)
    for i in range(cap):
        if i:
            parent = (rng.random(R) * i).astype(np.int64)
            parent = np.where(rng.random(R) < 0.3, i - 1, parent)
            sees[:, i] = sees[np.arange(R), parent]
        sees[:, i, i] = True
    sees &= (np.arange(cap) <= n[:, None])[:, :, None]
    words = (cap + 31) // 32
    bits = np.zeros((R, cap, words * 32), np.uint64)
    bits[:, :, :cap] = sees
    packed = (bits.reshape(R, cap, words, 32) << np.arange(32, dtype=np.uint64)).sum(-1)
    return torch.from_numpy(packed.astype(np.uint32).view(np.int32)).cuda()


def _values(shape, gen, outliers):
    """Keys have a few channels of far larger values, as a target's keys do; values have none."""
    x = torch.randn(shape, generator=gen, device="cuda")
    if outliers:
        x *= 1 + 7 * (torch.rand(shape[-2:], generator=gen, device="cuda") < 0.03)
    return x


def prepare(case, seed):
    c = case
    rng = np.random.default_rng(seed)
    gen = torch.Generator("cuda").manual_seed(seed)
    R, cap, page = c["R"], c["cap"], c["page"]
    length, n = _lengths(c)
    length, n = rng.permutation(length), rng.permutation(n)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).cuda()  # noqa: E731
    s = {"c": c, "len": dev(length), "n": dev(n), "most": int(length.max() + n.max() + 1)}
    if c["kind"] == "plan":
        # a pool with the context's pages dealt out, and as many free as the largest round takes
        held = -(-length // page)
        spare = R * (c["nhi"] // page + 2)
        pages = rng.permutation(int(held.sum()) + spare)
        table = np.full((R, c["blocks"]), -1, np.int64)
        table[np.arange(c["blocks"]) < held[:, None]] = pages[: held.sum()]
        free = np.full(len(pages), -1, np.int64)
        free[:spare] = pages[held.sum():]
        _, count = _paths(R, n, rng)
        s |= {"pages": len(pages), "held": dev(held), "table": dev(table), "free": dev(free),
              "count": dev(np.array([spare])), "len2": dev(length + 1 + count), "n2": dev(np.full(R, -1))}
        return s
    heads, D = c["heads"], c["D"]
    blocks = -(-s["most"] // page)
    need = -(-(length + n + 1) // page)
    ids = rng.permutation(int(need.sum()))
    table = np.full((R, blocks), -1, np.int64)
    table[np.arange(blocks) < need[:, None]] = ids
    layers, block = c.get("layers", 1), page * D * 17 // 16
    s |= {"table": dev(table), "layers": layers, "block": block}
    pos = length[:, None] + np.arange(max(cap, PATH + 1))
    at = np.where(pos < need[:, None] * page, np.take_along_axis(table, np.minimum(pos // page, blocks - 1), 1) * page + pos % page, -1)
    slot = np.where(np.arange(cap) <= n[:, None], at[:, :cap], -1)
    cache = torch.zeros((layers, len(ids), heads * block), dtype=torch.uint8, device="cuda")
    if c["kind"] != "append":  # the pages hold rows of earlier rounds
        for layer in range(layers):
            k, sk = _quantise(_values((len(ids) * page, heads, D), gen, True))
            v, sv = _quantise(_values((len(ids) * page, heads, D), gen, False))
            _store(cache[layer], page, heads, D, torch.arange(len(ids) * page, device="cuda"), k, sk, v, sv)
    s["cache"] = cache
    if c["kind"] == "append":
        s["slot"] = dev(slot.reshape(-1))
        s["kv"] = torch.cat([_values((R * cap, heads, D), gen, True), _values((R * cap, heads, D), gen, False)],
                            1).to(_dtype(c))  # one projection gives both
        s["k_out"], s["v_out"] = (torch.zeros((1, R * cap, heads, D), dtype=_dtype(c), device="cuda") for _ in "kv")
    elif c["kind"] == "accept":
        nodes, count = _paths(R, n, rng)
        s |= {"nodes": dev(nodes), "count": dev(count)}
        kept = np.where(np.arange(PATH + 1) <= count[:, None], at[:, : PATH + 1], -1)
        s["slot"] = dev(kept.reshape(-1))
        s["k_out"], s["v_out"] = (torch.zeros((layers, R * (PATH + 1), heads, D), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    else:
        hq = c["hq"]
        s["q"] = torch.randn((R, cap, hq, D), generator=gen, device="cuda").to(_dtype(c))
        s["mask"] = _tree_masks(R, cap, n, rng) if c["tree"] else None
        s["out"] = torch.zeros((R, cap, hq, D), dtype=_dtype(c), device="cuda")
        s["lse"] = torch.zeros((R, cap, hq), dtype=torch.float32, device="cuda")
    return s


# ---------------------------------------------------------------- the plain forms


def _quantise(x):
    """Codes (a byte each) and scale bytes of x [..., D]: per 32 values the least power of two with which the
    largest is at most 7, the nearest E2M1 value, ties to the even code, at most 6."""
    g = x.float().unflatten(-1, (-1, 32))
    top = g.abs().amax(-1)
    frac, exp = torch.frexp(top)  # top = frac * 2^exp, frac in [0.5, 1)
    byte = (exp - 3 + (frac > 0.875) + 127).clamp(2, 252).to(torch.int32)
    y = torch.ldexp(g, (127 - byte).unsqueeze(-1))
    a = y.abs()
    step = 0.5 + 0.5 * (a >= 2) + 1.0 * (a >= 4)
    a = torch.clamp(torch.round(a / step) * step, max=6.0)
    code = 2 * a - (a > 2) * (a - 2) - (a > 4) * (a - 4) / 2
    code = code.to(torch.uint8) + 8 * (y < 0).to(torch.uint8)
    return code.flatten(-2), byte.to(torch.uint8)


def _parts(cache, page, heads, D):
    """Views of cache [..., pages, heads * block]: key codes, key scales, value codes, value scales, each
    [..., pages, heads, page, bytes of a token]."""
    block = cache.unflatten(-1, (heads, page * D * 17 // 16))
    a, b = page * D // 2, page * D // 32
    cut = ((0, a), (a, a + b), (a + b, 2 * a + b), (2 * a + b, 2 * a + 2 * b))
    return [block[..., lo:hi].unflatten(-1, (page, -1)) for lo, hi in cut]


def _store(cache, page, heads, D, slot, k, sk, v, sv):
    """Codes k, v [rows][heads][D] and scales into cache [pages][heads * block] at slots."""
    pairs = [x[..., 0::2] + 16 * x[..., 1::2] for x in (k, v)]
    kc, ks, vc, vs = _parts(cache, page, heads, D)
    at = (slot // page, slice(None), slot % page)
    kc[at], ks[at], vc[at], vs[at] = pairs[0], sk, pairs[1], sv


def _load(codes, scales, key):
    """32-bit values of codes [..., D/2] under scales [..., D/32]; a scale of 255 is not-a-number or zero."""
    both = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    step = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    scale = torch.ldexp(torch.ones((), device=codes.device), scales.to(torch.int32) - 127)
    scale = torch.where(scales == 255, math.nan if key else 0.0, scale)
    return (step[both.int()].unflatten(-1, (-1, 32)) * scale.unsqueeze(-1)).flatten(-2)


def _read_back(s, slot, dtype):
    """[layers][rows][heads][D] keys and values at slots; rows without a slot are zero."""
    c = s["c"]
    there = (slot >= 0).view(1, -1, 1, 1)
    at = (slice(None), slot.clamp(min=0) // c["page"], slice(None), slot.clamp(min=0) % c["page"])
    kc, ks, vc, vs = (x[at].transpose(0, 1) for x in _parts(s["cache"], c["page"], c["heads"], c["D"]))
    return [torch.where(there, _load(a, b, key), 0.0).to(dtype) for a, b, key in ((kc, ks, True), (vc, vs, False))]


def _plain_plan(c, pages, length, n, held, table, free, count, with_slots):
    """One planning step on (held, table, free, count), in place; the slot map and the granted nodes."""
    page, cap, blocks = c["page"], c["cap"], c["blocks"]
    length, nodes = length.long().clamp(min=0), n.long().clamp(max=cap - 1)
    want = length + (nodes + 1).clamp(min=0)
    need = (want + page - 1) // page
    fits = need <= blocks
    h = held.long()
    add = torch.where(fits, need - h, 0).clamp(min=0)
    # pages given back: the stack gets them so that the last block of the last request lies lowest
    col = torch.arange(blocks, device=table.device)
    back = fits[:, None] & (col >= need[:, None]) & (col < h[:, None])
    order = torch.cumsum(back.flatten().long(), 0).view_as(back)
    total = order[-1, -1]
    top = count.long() + total
    stack = torch.cat([free, free.new_zeros(1)])  # one place more, for what is not given back
    place = torch.where(back, top - order, len(free))
    stack[place.flatten()] = torch.where(back, table, 0).flatten()
    # pages taken: requests in their order, each whole or not at all
    upto = torch.cumsum(add, 0)
    ok = fits & ((add == 0) | (upto <= top))
    take = ok[:, None] & (col >= h[:, None]) & (col < need[:, None])
    nth = (upto - add - h)[:, None] + col
    got = stack[(top - 1 - nth).clamp(0, len(free) - 1)]
    table.copy_(torch.where(take, got, torch.where(back, -1, table)))
    count.copy_(top - torch.where(ok, add, 0).sum())
    held.copy_(torch.where(ok, need, h))
    free.copy_(stack[:-1])
    granted = torch.where(ok & (nodes >= 0), nodes, -1)
    if not with_slots:
        return None, granted.int()
    i = torch.arange(cap, device=table.device)
    pos = length[:, None] + i
    slot = torch.gather(table.long(), 1, (pos // page).clamp(max=blocks - 1)) * page + pos % page
    return torch.where(i <= granted[:, None], slot, -1).int(), granted.int()


def _plain_attend(s):
    c = s["c"]
    R, cap, hq, heads, D, page = c["R"], c["cap"], c["hq"], c["heads"], c["D"], c["page"]
    pages = s["cache"][0][s["table"].long().clamp(min=0)]  # [R][blocks][heads * block]
    kc, ks, vc, vs = (x.transpose(1, 2).flatten(2, 3) for x in _parts(pages, page, heads, D))
    t = torch.arange(kc.shape[2], device="cuda")
    length, n = s["len"].long(), s["n"].long()
    there = t < (length + n + 1)[:, None]
    k = torch.where(there[:, None, :, None], _load(kc, ks, True), 0.0)
    v = torch.where(there[:, None, :, None], _load(vc, vs, False), 0.0)
    i = torch.arange(cap, device="cuda")
    j = t - length[:, None]
    if s["mask"] is None:
        new = j[:, None, :] <= i[:, None]
    else:
        jc = j.clamp(0, cap - 1)[:, None, :].expand(R, cap, len(t))
        new = ((torch.gather(s["mask"].long(), 2, jc // 32) >> (jc % 32)) & 1).bool() & (j >= 0)[:, None, :]
    sees = ((j < 0)[:, None, :] | new) & there[:, None, :]  # [R][cap][tokens]
    group = hq // heads
    q = s["q"].float().view(R, cap, heads, group, D).permute(0, 2, 1, 3, 4).reshape(R, heads, cap * group, D)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()) * D ** -0.5
    x = x.view(R, heads, cap, group, -1).masked_fill(~sees[:, None, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(R, heads, cap * group, -1), v).view(R, heads, cap, group, D)
    o = torch.where(total > 0, o / total, torch.where(total == 0, 0.0, math.nan))
    lse = (top + torch.log(total)).squeeze(-1)
    row = (i <= n[:, None])
    o = torch.where(row[:, None, :, None, None], o, 0.0).permute(0, 2, 1, 3, 4).reshape(R, cap, hq, D)
    lse = torch.where(row[:, None, :, None], lse, 0.0).permute(0, 2, 1, 3).reshape(R, cap, hq)
    return {"out": o.to(s["q"].dtype), "lse": lse}


def _plain(s):
    c = s["c"]
    if c["kind"] == "plan":
        pool = s["held"], s["table"], s["free"], s["count"]
        slot, granted = _plain_plan(c, s["pages"], s["len"], s["n"], *pool, True)
        _plain_plan(c, s["pages"], s["len2"], s["n2"], *pool, False)
        return {"slot": slot, "granted": granted, "held": s["held"], "table": s["table"], "free": s["free"],
                "count": s["count"]}
    if c["kind"] == "append":
        row = torch.nonzero(s["slot"] >= 0).flatten()
        kv = s["kv"][row]
        _store(s["cache"][0], c["page"], c["heads"], c["D"], s["slot"][row].long(),
               *_quantise(kv[:, : c["heads"]]), *_quantise(kv[:, c["heads"]:]))
        return _read_back(s, s["slot"].long(), _dtype(c))
    if c["kind"] == "accept":
        # rows past the path move from the root's place to the root's place
        j = torch.arange(PATH, device="cuda")
        on = j < s["count"][:, None]
        src = s["len"][:, None].long() + torch.where(on, s["nodes"], 0)
        dst = s["len"][:, None].long() + torch.where(on, j + 1, 0)
        to, frm = ((torch.gather(s["table"].long(), 1, x // c["page"]).flatten(), slice(None), (x % c["page"]).flatten()) for x in (dst, src))
        for part in _parts(s["cache"], c["page"], c["heads"], c["D"]):
            part[(slice(None), *to)] = part[(slice(None), *frm)]
        return [s["len"] + 1 + s["count"], *_read_back(s, s["slot"].long(), torch.bfloat16)]
    return _plain_attend(s)


# ---------------------------------------------------------------- the framework's operators


def _own(s):
    from paper_2609_22098_amd import kv

    c = s["c"]
    if c["kind"] == "plan":
        if "pool" not in s:
            s["pool"] = kv.Pool(s["pages"], c["R"], c["blocks"], c["page"], free_pages=s["free"], free_count=s["count"],
                                held=s["held"], table=s["table"])
        pool = s["pool"]
        slot, granted = kv.plan(pool, s["len"], s["n"], c["cap"])
        kv.plan(pool, s["len2"], s["n2"], c["cap"], slots=False)
        return {"slot": slot, "granted": granted, "held": pool.held, "table": pool.table, "free": pool.free_pages,
                "count": pool.free_count}
    if "handle" not in s:
        s["handle"] = kv.Cache(s["cache"], c["page"], c["heads"], c["D"])
    cache = s["handle"]
    if c["kind"] == "append":
        kv.append(cache, s["kv"][:, : c["heads"]], s["kv"][:, c["heads"]:], s["slot"], layer=0)
        return list(kv.read(cache, s["slot"], out=(s["k_out"], s["v_out"])))
    if c["kind"] == "accept":
        new = kv.accept(cache, s["len"], s["n"], s["table"], s["nodes"], s["count"])
        return [new, *kv.read(cache, s["slot"], out=(s["k_out"], s["v_out"]))]
    out, lse = kv.attention(cache, s["q"], s["len"], s["n"], s["table"], mask=s["mask"], layer=0, out=s["out"],
                            lse=s["lse"])
    return {"out": out, "lse": lse}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    """Bytes and operations of one pass: inputs and outputs once each; for `plan` both of its calls, for
    `append` and `accept` the read back."""
    c = case
    length, n = _lengths(c)
    rows = int((n + 1).sum())
    if c["kind"] == "plan":
        held = -(-length // c["page"])
        changed = int((-(-(length + n + 1) // c["page"]) - held).sum())
        return {"bytes": 4 * c["R"] * c["cap"] + 2 * 16 * c["R"] + 2 * 8 * changed, "flops": 0}
    token = c["heads"] * c["D"] * 17 // 16  # bytes of a token's key and value
    size = 2 if c.get("dtype") != "f32" else 4
    if c["kind"] == "append":
        return {"bytes": rows * (2 * c["heads"] * c["D"] * 2 * size + 2 * token + 8), "flops": 0}
    if c["kind"] == "accept":
        kept = np.minimum(n, 8).sum()  # paths of 0 to 16 nodes, 8 on average
        return {"bytes": int(c["layers"] * (kept * 2 * token + (kept + c["R"]) * (token + 2 * c["heads"] * c["D"] * 2))), "flops": 0}
    pairs = int(((n + 1) * length).sum())
    if c["tree"]:
        pairs += int(((n + 1) * np.minimum(n + 1, 5)).sum())  # a random tree's rows see a few ancestors each
    else:
        pairs += int(((n + 1) * (n + 2) // 2).sum())
    mask = rows * -(-c["cap"] // 32) * 4 if c["tree"] else 0
    return {"bytes": int((length + n + 1).sum()) * token + rows * c["hq"] * (2 * c["D"] * size + 4) + mask,
            "flops": 4 * c["D"] * c["hq"] * pairs}


# ---------------------------------------------------------------- 64 bits


def _exact_value(code, byte, key):
    """What a code (0..15) stands for under its scale byte, from the format's bits."""
    code, byte = code.astype(np.int64), byte.astype(np.int64)
    exp, man = code >> 1 & 3, code & 1
    mag = np.where(exp == 0, man * 0.5, (1 + man * 0.5) * 2.0 ** (exp - 1))
    return np.where(byte == 255, np.nan if key else 0.0, np.where(code & 8, -mag, mag) * 2.0 ** (byte - 127.0))


def _exact_rounded(x):
    """x [..., 32] in 64 bits as its group in the cache would give it back."""
    top = np.abs(x).max(-1, keepdims=True)
    with np.errstate(divide="ignore"):
        byte = np.clip(np.where(top > 0, np.ceil(np.log2(top / 7)), -999) + 127, 2, 252)
    grid = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    a = np.abs(x) / 2.0 ** (byte - 127)
    border = (grid[1:] + grid[:-1]) / 2
    code = np.zeros(a.shape, np.int64)
    for i, b in enumerate(border):
        code += (a > b) | ((a == b) & (i % 2 == 1))  # a tie goes to the even code
    return np.sign(x) * grid[code] * 2.0 ** (byte - 127)


def _exact_rows(cache, c, part, table, pos):
    """[layers][heads][positions][D] in 64 bits: the keys (part 0) or values (part 1) of a request's positions."""
    page, D, heads, count = c["page"], c["D"], c["heads"], len(pos)
    block = cache.reshape(cache.shape[0], cache.shape[1], heads, -1)
    codes, scales = page * D // 2, page * D // 32
    base = part * (codes + scales)
    pg = block[:, table[pos // page]].transpose(0, 2, 1, 3)  # [layers][heads][count][block]
    at = (pos % page)[:, None]
    byte = np.take_along_axis(pg, np.broadcast_to(base + at * (D // 2) + np.arange(D // 2), pg.shape[:2] + (count, D // 2)), 3)
    scale = np.take_along_axis(pg, np.broadcast_to(base + codes + at * (D // 32) + np.arange(D // 32), pg.shape[:2] + (count, D // 32)), 3)
    code = np.stack([byte & 15, byte >> 4], -1).reshape(byte.shape[:3] + (D,))
    return _exact_value(code, np.repeat(scale, 32, -1), part == 0)


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["kind"] == "plan":
        return None  # whole numbers
    R, cap, heads, D = c["R"], c["cap"], c["heads"], c["D"]
    if c["kind"] == "append":
        x = s["kv"].double().cpu().numpy().reshape(R * cap, 2, heads, D // 32, 32)
        y = _exact_rounded(x).reshape(R * cap, 2, heads, D)
        y[s["slot"].cpu().numpy() < 0] = 0.0
        return [np.ascontiguousarray(y[None, :, 0]), np.ascontiguousarray(y[None, :, 1])]
    length, n, table = (s[k].cpu().numpy().astype(np.int64) for k in ("len", "n", "table"))
    if c["kind"] == "accept":
        cache, nodes, count = s["cache"].cpu().numpy(), s["nodes"].cpu().numpy(), s["count"].cpu().numpy()
        outs = np.zeros((2, s["layers"], R, PATH + 1, heads, D))
        for q in range(R):
            pos = length[q] + np.concatenate([[0], nodes[q, : count[q]]])
            for part in (0, 1):
                outs[part, :, q, : len(pos)] = _exact_rows(cache, c, part, table[q], pos).transpose(0, 2, 1, 3)
        outs = outs.reshape(2, s["layers"], R * (PATH + 1), heads, D)
        return [None, outs[0], outs[1]]
    hq, group = c["hq"], c["hq"] // heads
    step = torch.from_numpy(_exact_value(np.arange(16), np.full(16, 127), True)).cuda()
    out = torch.zeros((R, cap, hq, D), dtype=torch.float64, device="cuda")
    lse = torch.zeros((R, cap, hq), dtype=torch.float64, device="cuda")
    page, codes, scales = c["page"], c["page"] * D // 2, c["page"] * D // 32
    for q in range(R):
        total, rows = int(length[q] + n[q] + 1), int(n[q]) + 1
        pos = torch.arange(total, device="cuda")
        pages = s["cache"][0][s["table"][q].long()[: -(-total // page)]].view(-1, heads, s["block"])
        if s["mask"] is None:
            sees = pos[None] <= length[q] + torch.arange(rows, device="cuda")[:, None]
        else:
            word = s["mask"][q, :rows].long()
            bit = (word[:, :, None] >> torch.arange(32, device="cuda") & 1).reshape(rows, -1)[:, :rows].bool()
            sees = torch.cat([torch.ones((rows, int(length[q])), dtype=torch.bool, device="cuda"), bit], 1)
        for h in range(heads):
            kv = []
            for base in (0, codes + scales):
                byte = pages[:, h, base : base + codes].reshape(-1, D // 2)[:total].long()
                sc = pages[:, h, base + codes : base + codes + scales].reshape(-1, D // 32)[:total].double()
                val = torch.stack([step[byte & 15], step[byte >> 4]], -1).view(total, D // 32, 32)
                kv.append((val * torch.exp2(sc - 127)[:, :, None]).view(total, D))
            for g in range(group):
                a = h * group + g
                x = s["q"][q, :rows, a].double() @ kv[0].T.contiguous() / math.sqrt(D)
                x = x.masked_fill(~sees, -math.inf)
                lse[q, :rows, a] = torch.logsumexp(x, -1)
                out[q, :rows, a] = torch.softmax(x, -1) @ kv[1]
    return {"out": out, "lse": lse}
