"""GPU parity of the serving operators (plan of a step, append to a paged cache, attention of drafted tokens over the pages,
rules on the logits) against plain implementations written from their definitions, in Python integers and 64-bit floats."""
import ctypes
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def zq():
    from paper_2509_00031_b200 import binding
    binding.lib()
    return binding


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def rand_parents(rng, new):
    """Per request: draft 0 follows the context, draft i one of the drafts before it or the context."""
    out = []
    for n in new:
        out += [-1 if i == 0 else int(rng.integers(max(-1, i - 6), i)) for i in range(n)]
    return out


def ancestors(parents, i):
    seen = []
    while i >= 0:
        seen.append(i)
        i = parents[i]
    return seen


def words_of(bits, words):
    """Set of bit numbers -> signed 32-bit words."""
    out = [0] * words
    for b in bits:
        out[b // 32] |= 1 << (b % 32)
    return [w - 2 ** 32 if w >= 2 ** 31 else w for w in out]


# ---- plan -----------------------------------------------------------------------------------------------------------
def plan_oracle(cached, new, page, free, n_free, table, max_rows, parents, words):
    table = [list(r) for r in table]
    top, start, request, pos, slot, mask = n_free, [0], [], [], [], []
    for b, (c, n) in enumerate(zip(cached, new)):
        for k in range(-(-c // page), -(-(c + n) // page)):
            top -= 1
            table[b][k] = free[top]
        mine = parents[start[-1]:start[-1] + n] if parents else list(range(-1, n - 1))
        for i in range(n):
            line = ancestors(mine, i)
            request.append(b)
            pos.append(c + len(line) - 1)
            slot.append(table[b][(c + i) // page] * page + (c + i) % page)
            mask.append(words_of(line, words) if words else [])
        start.append(start[-1] + n)
    pad = max_rows - start[-1]
    return dict(kv_len=[c + n for c, n in zip(cached, new)], row_start=start, row_request=request + [-1] * pad, row_pos=pos + [-1] * pad,
                slot=slot + [-1] * pad, tree_mask=mask + [[0] * words] * pad, n_free=[top], table=table)


def plan_inputs(rng, cached, new, page, spare=4):
    held = [-(-c // page) for c in cached]
    need = sum(-(-(c + n) // page) - h for c, n, h in zip(cached, new, held))
    max_pages = max(max(-(-(c + n) // page) for c, n in zip(cached, new)), 1) + 1
    order = rng.permutation(sum(held) + need + spare).tolist()
    table = []
    for h in held:
        table.append(order[:h] + [-7] * (max_pages - h))
        order = order[h:]
    return table, order, max_pages, sum(held) + need + spare


@pytest.mark.parametrize("batch,page,hi_cached,hi_new,words,tree", [
    (1, 16, 0, 1, 0, False), (1, 1, 5, 3, 1, True), (3, 16, 40, 5, 0, False), (7, 8, 100, 33, 2, True), (7, 8, 100, 33, 2, False),
    (64, 128, 2000, 9, 1, True), (1025, 16, 300, 3, 1, True), (2500, 32, 70, 2, 0, True), (5, 48, 97, 1023, 32, True), (9, 64, 0, 700, 0, False)])
def test_plan_matches_the_definition(zq, batch, page, hi_cached, hi_new, words, tree):
    rng = np.random.default_rng(batch + page)
    cached = rng.integers(0, hi_cached + 1, batch).tolist()
    new = rng.integers(0, hi_new + 1, batch).tolist()
    new[-1] = hi_new                                   # (requests without a token are among the others)
    table, free, max_pages, n_pages = plan_inputs(rng, cached, new, page)
    rows = sum(new)
    max_rows = rows + 3
    parents = rand_parents(rng, new) if tree else None
    want = plan_oracle(cached, new, page, free, len(free), table, max_rows, parents, words)
    t = ints(table)
    run = lambda out=None: zq.zoqat_op_cache_plan(ints(cached), ints(new), page, n_pages, ints(free), ints([len(free)]), t, max_rows,  # noqa: E731
                                                  parents=ints(parents + [-1] * 3) if tree else None, mask_words=words, out=out)
    got = run()
    for again in range(2):
        assert got["status"].item() == 0
        for n in ("kv_len", "row_start", "row_request", "row_pos", "slot", "n_free"):
            assert got[n].tolist() == want[n], n
        if words:
            assert got["tree_mask"].tolist() == want["tree_mask"]
        assert t.tolist() == want["table"]
        got = run(out=got)                             # the same call on its own results: nothing changes


def test_plan_reports_what_it_cannot_serve_and_leaves_the_tables(zq):
    table = [[4, -7, -7], [-7, -7, -7]]

    def call(cached, new, free=(0, 1, 2, 3), n_free=None, n_pages=5, max_rows=40, parents=None, words=0):
        t = ints(table)
        got = zq.zoqat_op_cache_plan(ints(cached), ints(new), 16, n_pages, ints(list(free)), ints([len(free) if n_free is None else n_free]), t, max_rows,
                                     parents=None if parents is None else ints(parents), mask_words=words)
        return got, t.tolist()

    for kw, status in ((dict(cached=[3, -1], new=[1, 1]), 1), (dict(cached=[3, 0], new=[1, -2]), 1), (dict(cached=[3, 0], new=[46, 0]), 1),
                       (dict(cached=[3, 0], new=[20, 21]), 1), (dict(cached=[3, 0], new=[33, 0], words=1), 1),
                       (dict(cached=[3, 0], new=[1, 1], n_free=5), 1), (dict(cached=[3, 0], new=[1, 1], n_free=-1), 1),
                       (dict(cached=[2 ** 31 - 1, 0], new=[2 ** 31 - 1, 2 ** 31 - 1]), 1),
                       (dict(cached=[3, 0], new=[14, 17], free=(0, 1)), 2), (dict(cached=[3, 0], new=[0, 1], free=(), n_free=0), 2)):
        got, t = call(**kw)
        assert got["status"].item() == status, kw
        assert t == table and got["row_start"].tolist() == [0, 0, 0] and got["kv_len"].tolist() == [0, 0]
        assert set(got["slot"].tolist()) == {-1} and set(got["row_request"].tolist()) == {-1}
    # a page outside the pool costs the rows on it their slots and nothing else
    got, t = call(cached=[3, 0], new=[1, 2], free=(0, 1, 2, 77))
    assert got["status"].item() == 4 and got["slot"].tolist()[:3] == [4 * 16 + 3, -1, -1] and got["row_start"].tolist() == [0, 1, 3]
    # a parent that is not before its child ends the walk there
    got, _ = call(cached=[3, 0], new=[3, 0], parents=[-1, 1, 0] + [-1] * 37, words=1)
    assert got["status"].item() == 8 and [r[0] for r in got["tree_mask"].tolist()[:3]] == [1, 2, 5]
    got, _ = call(cached=[3, 0], new=[2, 0], parents=[-1, -2] + [-1] * 38, words=1)
    assert got["status"].item() == 8


# ---- append ---------------------------------------------------------------------------------------------------------
def make_cache(n_pages, page, kv, dh, dtype, layout, fill=float("nan")):
    if layout == "token":
        return [torch.full((n_pages, page, kv, dh), fill, dtype=TYPES[dtype], device="cuda") for _ in range(2)]
    if layout == "head":
        return [torch.full((n_pages, kv, page, dh), fill, dtype=TYPES[dtype], device="cuda").transpose(1, 2) for _ in range(2)]
    both = torch.full((n_pages, page, 2, kv, dh), fill, dtype=TYPES[dtype], device="cuda")      # k and v of a page side by side
    return [both[:, :, 0], both[:, :, 1]]


@pytest.mark.parametrize("dtype,rows,heads,kv,dh,page,layout,rope", [
    ("f32", 1, 1, 1, 64, 16, "token", True), ("bf16", 5, 4, 2, 128, 16, "head", True), ("f16", 33, 7, 1, 64, 1, "token", False),
    ("bf16", 8, 32, 32, 128, 64, "joint", True), ("f16", 300, 12, 4, 128, 128, "head", True), ("f32", 17, 6, 3, 128, 24, "joint", True)])
def test_append_matches_the_definition(zq, dtype, rows, heads, kv, dh, page, layout, rope):
    rng = np.random.default_rng(rows + heads)
    n_pages = -(-rows // page) + 2
    k, v = make_cache(n_pages, page, kv, dh, dtype, layout)
    wide = (heads + 2 * kv) * dh
    slab = torch.from_numpy(rng.standard_normal((rows, wide + 8)).astype(np.float32)).cuda()
    qkv = slab[:, :wide]                                                # rows that stand apart
    slot = rng.permutation(n_pages * page)[:rows]
    pos = rng.integers(0, 50, rows)
    if rows > 4:
        slot[2] = -1
    cos, sin = [torch.from_numpy(f(np.arange(50)[:, None] * 10000.0 ** (-np.arange(dh // 2) / (dh // 2))).astype(np.float32)).cuda() for f in (np.cos, np.sin)]
    q_out = torch.full((rows, heads + 1, dh), 7.0, dtype=TYPES[dtype], device="cuda")[:, :heads]
    q, err = zq.zoqat_op_cache_append(qkv, ints(pos.tolist()), ints(slot.tolist()), k, v, heads, cos=cos if rope else None, sin=sin if rope else None, q_out=q_out)
    assert err.item() == 0
    x = qkv.double().reshape(rows, heads + 2 * kv, dh).clone()
    turned = x[:, :heads + kv].clone()
    size = x.abs()
    if rope:
        c, s = cos.double()[pos][:, None], sin.double()[pos][:, None]
        a, b = x[:, :heads + kv, :dh // 2], x[:, :heads + kv, dh // 2:]
        turned = torch.cat([a * c - b * s, b * c + a * s], -1)
        size = x.clone()
        size[:, :heads + kv] = torch.cat([(a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()], -1)
        size = size.abs()
    # one rounding to the type, two binary32 operations before it (three roundings of at most half a step of the parts)
    half = torch.finfo(TYPES[dtype]).eps / 2
    tiny = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}[dtype]
    near = lambda got, want, sz: bool(((got.double() - want).abs() <= half * want.abs() + 3 * 2.0 ** -24 * sz * (1 + half) + tiny).all())  # noqa: E731
    live = slot >= 0
    assert near(q[live], turned[live][:, :heads], size[live][:, :heads])
    assert bool((q[~live] == 7.0).all())
    pg, off = slot[live] // page, slot[live] % page
    assert near(k[pg, off], turned[live][:, heads:], size[live][:, heads:heads + kv])
    assert near(v[pg, off], x[live][:, heads + kv:], torch.zeros_like(x[live][:, heads + kv:]))
    # every other slot is as it was
    other = torch.ones((n_pages, page), dtype=torch.bool)
    other[pg, off] = False
    assert bool(torch.isnan(k[other.cuda()]).all()) and bool(torch.isnan(v[other.cuda()]).all())


def test_append_skips_and_reports_slots_and_positions_outside(zq):
    k, v = make_cache(2, 16, 1, 64, "f32", "token", fill=3.0)
    qkv = torch.ones((4, 3 * 64), device="cuda")
    cos = torch.ones((8, 32), device="cuda")
    q = torch.full((4, 1, 64), 7.0, device="cuda")
    for pos, slot in (([0, 1, 2, 3], [0, 32, -1, 2 ** 30]), ([0, 8, -1, 99], [0, 5, 6, 7])):
        k.fill_(3.0); v.fill_(3.0); q.fill_(7.0)
        _, err = zq.zoqat_op_cache_append(qkv, ints(pos), ints(slot), k, v, 1, cos=cos, sin=cos, q_out=q)
        assert err.item() == 40
        assert bool((q[1:] == 7.0).all()) and bool((q[0] != 7.0).all())
        if pos[1] == 1:
            assert bool((k.view(32, 64)[1:] == 3.0).all()) and bool((v.view(32, 64)[1:] == 3.0).all())
        else:
            assert bool((k.view(32, 64)[1:] == 3.0).all())              # (v needs no position)


@pytest.mark.parametrize("dtype,heads,kv,dh,layout", [("f32", 1, 1, 64, "token"), ("bf16", 40, 8, 128, "head"), ("f16", 4, 2, 64, "joint")])
def test_append_skips_rows_with_a_bad_position_whole(zq, dtype, heads, kv, dh, layout):
    # the slot of such a row keeps its old key and its old value; the rows around it are written
    k, v = make_cache(3, 16, kv, dh, dtype, layout, fill=3.0)
    qkv = torch.ones((6, (heads + 2 * kv) * dh), device="cuda")
    cos, sin = torch.ones((8, dh // 2), device="cuda"), torch.zeros((8, dh // 2), device="cuda")
    q = torch.full((6, heads, dh), 7.0, dtype=TYPES[dtype], device="cuda")
    _, err = zq.zoqat_op_cache_append(qkv, ints([7, 8, -1, 0, 2 ** 31 - 1, -2 ** 31]), ints([40, 1, 2, 17, 4, 5]), k, v, heads, cos=cos, sin=sin, q_out=q)
    assert err.item() == 40
    assert bool((q[[0, 3]] == 1.0).all()) and bool((q[[1, 2, 4, 5]] == 7.0).all())
    for c in (k, v):
        want = torch.full((48, kv, dh), 3.0, dtype=TYPES[dtype], device="cuda")
        want[[40, 17]] = 1.0
        assert torch.equal(c.reshape(48, kv, dh), want)


# ---- attention --------------------------------------------------------------------------------------------------------
def attention_problem(seed, dtype, heads, kv, dh, page, layout, cached, new, mask="tree", pad=2, gap=0, q_scale=1.0):
    """Everything that no row may see is NaN: unused pages, the slots behind each request's end."""
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    batch, rows = len(cached), sum(new)
    L = [c + n for c, n in zip(cached, new)]
    pages = [-(-x // page) for x in L]
    max_pages, n_pages = max(pages) + 1, sum(pages) + 2
    order = rng.permutation(n_pages).tolist()
    k, v = make_cache(n_pages, page, kv, dh, dtype, layout)
    table, keys, vals = [], [], []
    for x, n in zip(L, pages):
        mine, order = order[:n], order[n:]
        table.append(mine + [-3] * (max_pages - n))
        t = torch.arange(x, device="cuda")
        pg, off = torch.tensor(mine + [0], device="cuda")[t // page], t % page
        keys.append(torch.randn((x, kv, dh), generator=gen, device="cuda").to(TYPES[dtype]))
        vals.append(torch.randn((x, kv, dh), generator=gen, device="cuda").to(TYPES[dtype]))
        k[pg, off], v[pg, off] = keys[-1], vals[-1]
    q = torch.full((rows + pad, heads + gap, dh), float("nan"), dtype=TYPES[dtype], device="cuda")[:, :heads]
    q[:rows] = (q_scale * torch.randn((rows, heads, dh), generator=gen, device="cuda")).to(TYPES[dtype])
    words = -(-max(new) // 32) if max(new) else 1
    seen = []
    for n in new:
        if mask == "tree":
            par = rand_parents(rng, [n])
            seen.append([set(ancestors(par, i)) for i in range(n)])
        elif mask == "random":                                          # rows that see no draft, not even themselves, among them
            seen.append([set(np.nonzero(rng.random(n) < 0.3)[0].tolist()) if i % 3 else set() for i in range(n)])
        else:
            seen.append([set(range(i + 1)) for i in range(n)])
    bits = [words_of(s, words) for r in seen for s in r] + [[-1] * words] * pad
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    return dict(dtype=dtype, q=q, k=k, v=v, table=ints(table), kv_len=ints(L), row_start=ints(start), mask=ints(bits) if mask else None, rows=rows,
                start=start, new=new, L=L, keys=keys, vals=vals, seen=seen, heads=heads, kv=kv, dh=dh, scale=1.0 / math.sqrt(dh))


def attention_oracle(pr):
    """(out, bound) in 64 bits.  bound: how far a correct evaluation may be off, element by element - see the test."""
    out = torch.zeros((pr["rows"], pr["heads"], pr["dh"]), dtype=torch.float64, device="cuda")
    bound = torch.zeros_like(out)
    g, eps = pr["heads"] // pr["kv"], 2.0 ** -24
    half = torch.finfo(TYPES[pr["dtype"]]).eps / 2
    for b, (n, L) in enumerate(zip(pr["new"], pr["L"])):
        if n == 0:
            continue
        vis = torch.zeros((n, L), dtype=torch.bool)
        vis[:, :L - n] = True
        for i, s in enumerate(pr["seen"][b]):
            for j in s:
                vis[i, L - n + j] = True
        vis = vis.cuda()[:, None]
        r = slice(pr["start"][b], pr["start"][b + 1])
        for h in range(pr["kv"]):
            hs = slice(h * g, (h + 1) * g)
            q, k, v = pr["q"][r, hs].double(), pr["keys"][b][:, h].double(), pr["vals"][b][:, h].double()
            s = torch.einsum("ngd,td->ngt", q, k) * pr["scale"]
            mag = (torch.einsum("ngd,td->ngt", q.abs(), k.abs()) * pr["scale"]).amax(-1, keepdim=True)
            s = s.masked_fill(~vis, -math.inf)
            top = s.amax(-1, keepdim=True)
            p = torch.exp(s - torch.where(torch.isinf(top), 0.0, top)).masked_fill(~vis, 0.0)
            total = p.sum(-1, keepdim=True)
            w = torch.where(total > 0, p / total, 0.0)
            o = torch.einsum("ngt,td->ngd", w, torch.where(torch.isfinite(v), v, 0.0))
            a = torch.einsum("ngt,td->ngd", w, torch.where(torch.isfinite(v), v.abs(), 0.0))
            # scores: d products and sums in binary32, scaled, turned into base 2 (each a rounding of the score's size); the
            # exponential 2^-22; sums over the keys in binary32; each moves the weights relatively by the sum of these
            rel = 2 * ((pr["dh"] + 8) * eps * mag + 4 * 2.0 ** -22) + (L / 4 + 64) * eps
            e = rel * 2 * a
            if pr["dtype"] != "f32":
                e = e + half * a * (1 + 2 * half)                       # the weights, rounded for the second product
            if pr["dtype"] == "f16":
                # weights under the subnormal step of binary16, after the scaling by 2^7
                e = e + 2.0 ** -25 / 2.0 ** 7 * torch.where(torch.isfinite(v), v.abs(), 0.0).sum(0)[None, None] + 2.0 ** -25
            out[r, hs], bound[r, hs] = o, e + half * (o.abs() + e)
    return out, bound


def run_attention(zq, pr, **kw):
    rows, pad = pr["rows"], pr["q"].shape[0] - pr["rows"]
    out = torch.full_like(pr["q"], 5.0) if "out" not in kw else kw.pop("out")
    got, err = zq.zoqat_op_tree_attention(pr["q"], pr["k"], pr["v"], pr["table"], pr["kv_len"], pr["row_start"], tree_mask=pr["mask"], out=out, **kw)
    assert err.item() == 0
    if pad:
        assert bool((got[rows:] == 5.0).all())                          # rows behind the last request
    return got


ATTENTION = [
    # dtype, heads, kv, dh, page, layout, cached, new, mask
    ("f32", 2, 2, 128, 16, "token", [37], [1], "tree"),
    ("bf16", 2, 2, 128, 16, "token", [37], [1], "tree"),
    ("f16", 2, 2, 64, 16, "token", [0], [1], "tree"),                       # nothing but the draft itself
    ("f32", 4, 1, 64, 24, "joint", [0, 5, 63, 64, 65, 200], [1, 3, 0, 7, 2, 9], "tree"),
    ("bf16", 4, 1, 64, 8, "joint", [0, 5, 127, 128, 129, 300], [1, 3, 0, 7, 2, 9], "tree"),
    ("f16", 8, 2, 128, 64, "head", [0, 1, 255, 256, 511], [4, 4, 4, 4, 4], "random"),
    ("f32", 8, 2, 128, 1, "head", [0, 1, 61, 62, 130], [4, 3, 4, 5, 4], "random"),
    ("bf16", 8, 8, 128, 32, "token", [100, 0, 7], [33, 64, 40], "tree"),    # masks of two words, drafts across tile borders
    ("bf16", 6, 2, 64, 128, "head", [500, 20], [50, 100], None),            # no mask; more than 128 queries per key head
    ("f16", 14, 2, 128, 256, "joint", [300, 129, 0], [20, 37, 19], "tree"), # 7 query heads per key head
    ("f16", 16, 1, 128, 16, "token", [90], [17], "random"),                 # one key head
    ("f32", 14, 2, 64, 16, "token", [90, 3], [5, 2], "random"),
    ("bf16", 3, 3, 128, 16, "token", [5000], [2], "tree"),                  # one context split over many CTAs
    ("f32", 1, 1, 128, 64, "head", [9000], [3], "tree"),
    ("f16", 4, 4, 64, 64, "token", [3] * 300, [1] * 300, None),             # many short requests
    ("bf16", 20, 1, 128, 16, "token", [130, 1], [9, 2], "tree"),            # 20 query heads per key head
    ("f16", 20, 1, 128, 16, "token", [130, 1, 40, 700], [1, 1, 1, 1], "tree"),
    ("bf16", 8, 2, 128, 16, "token", [700, 33], [8, 9], "tree"),
    ("f16", 8, 2, 64, 128, "head", [1290, 0], [8, 9], "random"),
    ("bf16", 14, 2, 64, 32, "joint", [300, 129, 0, 4], [1, 2, 5, 1], "tree"),   # tiles that cut a draft's heads apart
    ("f16", 7, 1, 128, 16, "token", [300, 129, 0, 4], [3, 2, 5, 30], "random"),
    ("bf16", 2, 2, 128, 16, "token", [4000] * 9, [1] * 9, None),
    # long runs of tiles for every tile width of the tensor-core kernels (16, 32, 64 and 256 queries)
    ("bf16", 16, 4, 128, 64, "token", [5000, 20011, 9000, 16], [1, 1, 1, 1], "tree"),
    ("bf16", 16, 4, 128, 64, "token", [5000, 20011, 9000, 16], [4, 4, 4, 4], "tree"),
    ("f16", 16, 4, 64, 16, "head", [5000, 20011, 9000, 16], [4, 4, 4, 4], "tree"),
    ("f16", 16, 4, 128, 64, "token", [5000, 20011, 9000, 16], [8, 8, 8, 8], "tree"),
    ("bf16", 16, 4, 64, 16, "head", [5000, 20011, 9000, 16], [8, 9, 8, 8], "tree"),
    ("bf16", 16, 4, 128, 16, "token", [5000, 20011, 9000, 16], [40, 33, 64, 20], "tree"),
    ("f16", 16, 4, 64, 256, "joint", [5000, 20011, 9000, 16], [40, 33, 64, 20], "tree"),
    ("f32", 16, 4, 128, 64, "token", [5000, 8011, 900, 16], [1, 2, 3, 1], "tree"),
]


@pytest.mark.parametrize("case", ATTENTION, ids=lambda c: "-".join(str(x) for x in c[:6]) + f"-b{len(c[6])}-{c[8]}")
def test_attention_matches_the_definition(zq, case):
    dtype, heads, kv, dh, page, layout, cached, new, mask = case
    pr = attention_problem(7, dtype, heads, kv, dh, page, layout, cached, new, mask)
    got = run_attention(zq, pr)
    want, bound = attention_oracle(pr)
    off = (got[:pr["rows"]].double() - want).abs()
    assert bool((off <= bound).all()), (float(off.max()), float((off / bound.clamp(min=1e-30)).max()))
    if mask == "random" and cached[0] == 0:
        assert bool((got[0] == 0).all())                                # a row that sees nothing
    again = run_attention(zq, pr)
    assert torch.equal(again[:pr["rows"]], got[:pr["rows"]])            # the same bits


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_attention_with_steep_scores_and_strided_rows(zq, dtype):
    # scores of some hundreds: the running reference moves often, most weights vanish
    pr = attention_problem(11, dtype, 4, 2, 128, 16, "token", [700, 45], [6, 9], "tree", gap=1, q_scale=30.0)
    scratch = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")
    got = run_attention(zq, pr, scratch=scratch)                        # (scratch full of NaN)
    want, bound = attention_oracle(pr)
    off = (got[:pr["rows"]].double() - want).abs()
    assert bool((off <= bound).all()), (float(off.max()), float((off / bound.clamp(min=1e-30)).max()))


@pytest.mark.parametrize("dtype,page", [("f32", 16), ("bf16", 16), ("f16", 128)])
def test_unseen_drafts_may_hold_anything_and_seen_ones_count(zq, dtype, page):
    # drafts 0 <- 1, 0 <- 2; draft 2's value holds infinities and NaN, its key NaN: rows 0 and 1 do not see it, row 2 does
    for C in (0, 126, 300):
        pr = attention_problem(5, dtype, 4, 2, 64, page, "token", [C], [3], "tree")
        pr["mask"][:3] = ints([[1], [3], [5]])
        pr["seen"] = [[{0}, {0, 1}, {0, 2}]]
        want, bound = attention_oracle(pr)
        at = C + 2
        pg = pr["table"][0, at // page].item()
        pr["v"][pg, at % page, :, 5] = float("inf")
        pr["v"][pg, at % page, :, 6] = -float("inf")
        pr["v"][pg, at % page, :, 7] = float("nan")
        got = run_attention(zq, pr)
        off = (got[:2].double() - want[:2]).abs()
        assert bool((off <= bound[:2]).all())
        assert bool((got[2, :, 5] == float("inf")).all()) and bool((got[2, :, 6] == -float("inf")).all()) and bool(torch.isnan(got[2, :, 7]).all())
        clean = [e for e in range(64) if e not in (5, 6, 7)]
        assert bool(((got[2][:, clean].double() - want[2][:, clean]).abs() <= bound[2][:, clean]).all())
        pr["k"][pg, at % page] = float("nan")
        got = run_attention(zq, pr)
        assert bool(((got[:2].double() - want[:2]).abs() <= bound[:2]).all()) and bool(torch.isnan(got[2]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_reports_bad_pages_and_requests(zq, dtype):
    pr = attention_problem(3, dtype, 2, 2, 64, 16, "token", [40, 40, 40], [2, 2, 2], "tree")
    good = run_attention(zq, pr).clone()
    table = pr["table"].clone()
    for bad in (-1, pr["k"].shape[0], 2 ** 31 - 1):
        pr["table"][1, 1] = bad
        out, err = zq.zoqat_op_tree_attention(pr["q"], pr["k"], pr["v"], pr["table"], pr["kv_len"], pr["row_start"], tree_mask=pr["mask"])
        assert err.item() == 42 and bool(torch.isfinite(out[:6]).all())
        assert torch.equal(out[:2], good[:2]) and torch.equal(out[4:6], good[4:6])
    pr["table"].copy_(table)
    for kv_len, start in (([42, 1, 42], [0, 2, 4, 6]), ([42, -5, 42], [0, 2, 4, 6]), ([42, 10 ** 6, 42], [0, 2, 4, 6]), ([42, 42, 42], [0, 2, 900, 902])):
        out = torch.full_like(pr["q"], 5.0)
        _, err = zq.zoqat_op_tree_attention(pr["q"], pr["k"], pr["v"], pr["table"], ints(kv_len), ints(start), tree_mask=pr["mask"], out=out)
        assert err.item() == 41
        assert torch.equal(out[:2], good[:2]) and bool((out[2:4] == 5.0).all())


def test_attention_captured_and_replayed_as_lengths_change(zq):
    # one graph; the lengths, tables and rows in its buffers change between replays (fewer tokens, other requests, none at all)
    big = attention_problem(9, "bf16", 8, 2, 128, 16, "token", [900, 40, 3], [5, 5, 5], "tree")
    out, err = torch.zeros_like(big["q"]), torch.zeros(1, dtype=torch.int32, device="cuda")
    scratch = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    call = lambda: zq.zoqat_op_tree_attention(big["q"], big["k"], big["v"], big["table"], big["kv_len"], big["row_start"], tree_mask=big["mask"],  # noqa: E731
                                              out=out, scratch=scratch, err=err)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for L, new, start in (([905, 45, 8], [5, 5, 5], [0, 5, 10, 15]), ([300, 0, 8], [2, 0, 5], [0, 2, 2, 7]), ([0, 0, 0], [0, 0, 0], [0, 0, 0, 0])):
        big["kv_len"].copy_(ints(L))
        big["row_start"].copy_(ints(start))
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert err.item() == 0
        pr = dict(big, rows=sum(new), start=start, new=new, L=L, keys=[k[:x] for k, x in zip(big["keys"], L)], vals=[v[:x] for v, x in zip(big["vals"], L)])
        words = big["mask"].tolist()
        pr["seen"] = [[{j for j in range(n) if (words[s + i][0] >> j) & 1} for i in range(n)] for n, s in zip(new, start)]
        want, bound = attention_oracle(pr)
        rows = sum(new)
        assert bool(((out[:rows].double() - want).abs() <= bound).all()) and bool((out[rows:] == 5.0).all())


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("f16", 64)])
def test_unseen_drafts_of_wide_trees_may_hold_anything(zq, dtype, dh):
    # 72 drafts of 4 heads are two tiles of queries, the first one full; drafts lie in one, two and two tiles of keys
    for C in (0, 100, 700):
        pr = attention_problem(C + 3, dtype, 8, 2, dh, 16, "token", [C], [72], "tree")
        want, bound = attention_oracle(pr)
        marks = {20: float("inf"), 41: -float("inf"), 71: float("nan")}
        for j, x in marks.items():
            pr["v"][pr["table"][0, (C + j) // 16].item(), (C + j) % 16, :, j % 64] = x
        got = run_attention(zq, pr)
        for i in range(72):
            hit = {j % 64: x for j, x in marks.items() if j in pr["seen"][0][i]}
            rest = [e for e in range(dh) if e not in hit]
            assert bool(((got[i][:, rest].double() - want[i][:, rest]).abs() <= bound[i][:, rest]).all()), (C, i)
            for e, x in hit.items():
                assert bool(torch.isnan(got[i, :, e]).all() if math.isnan(x) else (got[i, :, e] == x).all()), (C, i, e)
        pr["k"][pr["table"][0, (C + 71) // 16].item(), (C + 71) % 16] = float("nan")
        got = run_attention(zq, pr)
        for i in range(72):
            assert bool(torch.isnan(got[i]).all()) == (71 in pr["seen"][0][i]), (C, i)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_wide_trees_with_steep_scores(zq, dtype):
    # the running references of both groups of queries move often
    pr = attention_problem(13, dtype, 16, 4, 128, 16, "token", [700, 2900], [48, 60], "tree", gap=1, q_scale=30.0)
    got = run_attention(zq, pr)
    want, bound = attention_oracle(pr)
    off = (got[:pr["rows"]].double() - want).abs()
    assert bool((off <= bound).all()), (float(off.max()), float((off / bound.clamp(min=1e-30)).max()))


def run_pieces(items, ctas, cost=4):
    """The runs of key tiles that the tensor-core kernels deal out: items of so many tiles, each with a constant for opening and closing it,
    laid out one after the other and cut into equal runs -> per CTA its pieces [item, first tile, tiles]."""
    total = sum(items) + cost * len(items)
    ctas = min(ctas, total)
    q, r = divmod(total, ctas)
    out, unit, c = [[] for _ in range(ctas)], 0, 0
    for i, n in enumerate(items):
        for kt in range(n):
            while unit + cost + kt >= q * (c + 1) + min(c + 1, r):
                c += 1
            if out[c] and out[c][-1][0] == i:
                out[c][-1][2] += 1
            else:
                out[c].append([i, kt, 1])
        unit += cost + n
    return out


@pytest.mark.parametrize("dtype,group,n,seed,batch,share", [("bf16", 4, 1, 133, 813, 0.305), ("f16", 4, 4, 241, 769, 0.242), ("bf16", 8, 8, 125, 770, 0.297),
                                                           ("f16", 4, 2, 212, 503, 0.218)])
def test_short_items_before_the_first_tile_of_a_long_one(zq, dtype, group, n, seed, batch, share):
    # runs that end in the first tile of a longer item, without drafts in it, behind three items of one tile: the last piece then follows
    # the ones before it at the shortest distance there is.  Drafts hold infinities, whose repair keeps the output warps longest.
    rng = np.random.default_rng(seed)
    rng.integers(500, 1100), rng.uniform(0.1, 0.5)
    cached = [int(rng.integers(0, 100)) if rng.random() > share else int(rng.integers(129, 500)) for _ in range(batch)]
    items, free = [-(-(c + n) // 128) for c in cached], [c // 128 for c in cached]
    runs = run_pieces(items, torch.cuda.get_device_properties(0).multi_processor_count)
    assert sum(len(r) >= 4 and r[-1][1:] == [0, 1] and items[r[-1][0]] > 1 and free[r[-1][0]] > 0 and all(x[2] == 1 for x in r[-4:-1]) for r in runs) > 2
    pr = attention_problem(seed, dtype, group, 1, 128, 16, "token", cached, [n] * batch, "tree")
    hit = torch.zeros((pr["rows"], 1, 128), dtype=torch.bool, device="cuda")
    for b, c in enumerate(cached):
        at = c + n - 1
        pr["v"][pr["table"][b, at // 16].item(), at % 16, :, b % 128] = float("inf")
        pr["vals"][b][n - 1 + c, :, b % 128] = float("inf")
        for i in range(n):
            hit[pr["start"][b] + i, 0, b % 128] = n - 1 in pr["seen"][b][i]
    want, bound = attention_oracle(pr)
    first = run_attention(zq, pr)
    got = first[:pr["rows"]].double()
    hit = hit.expand_as(got)
    assert bool((got[hit] == float("inf")).all()) and bool(((got - want).abs() <= bound)[~hit].all())
    for _ in range(20):
        assert torch.equal(run_attention(zq, pr)[:pr["rows"]], first[:pr["rows"]])


@pytest.mark.parametrize("dtype,dh,seed", [("bf16", 128, 1), ("f16", 64, 2)])
def test_full_and_half_filled_tiles_of_a_wide_tree_by_turns(zq, dtype, dh, seed):
    # items whose tiles of 256 queries are full, then several with up to 128: the second group of softmax warps sits pieces out.
    # Infinities stand in drafts of all of them, so that both groups repair outputs in every piece.
    new = [64, 5, 9, 1, 7, 64, 30, 3, 3, 3, 3, 40, 33, 2, 31, 64] * 6
    rng = np.random.default_rng(seed)
    cached = [int(x) for x in rng.integers(0, 300, len(new))]
    heads, kv = 12, 3
    assert 3 * sum(new) * heads // kv > 2 * 64 * len(new)                # more than 64 wanted: the wide kernel
    pr = attention_problem(seed, dtype, heads, kv, dh, 16, "token", cached, new, "tree")
    hit = torch.zeros((pr["rows"], heads, dh), dtype=torch.bool, device="cuda")
    for b, (c, n) in enumerate(zip(cached, new)):
        at, e = c + n // 2, b % dh
        pr["v"][pr["table"][b, at // 16].item(), at % 16, :, e] = -float("inf")
        pr["vals"][b][at, :, e] = -float("inf")
        for i in range(n):
            hit[pr["start"][b] + i, :, e] = n // 2 in pr["seen"][b][i]
    want, bound = attention_oracle(pr)
    first = run_attention(zq, pr)
    got = first[:pr["rows"]].double()
    assert bool((got[hit] == -float("inf")).all()) and bool(((got - want).abs() <= bound)[~hit].all())
    for _ in range(20):
        assert torch.equal(run_attention(zq, pr)[:pr["rows"]], first[:pr["rows"]])


@pytest.mark.parametrize("dtype,heads,kv,dh,new", [("bf16", 4, 4, 128, [9, 3, 7]), ("f16", 2, 1, 64, [13, 9, 5]), ("bf16", 6, 2, 64, [21, 10, 3]),
                                                   ("f16", 8, 2, 128, [30, 5, 41]), ("bf16", 14, 2, 128, [50, 33, 18])])
def test_lanes_that_see_different_drafts(zq, dtype, heads, kv, dh, new):
    # every row has a random mask of its own, a third of the rows sees no draft, tiles are partly filled, and two drafts of every request
    # hold infinities: the lanes of a warp go different ways in the masks, in the tail of V and in the repair of the outputs
    pr = attention_problem(17, dtype, heads, kv, dh, 8, "joint", [125, 0, 510], new, "random")
    hit = torch.zeros((pr["rows"], heads, dh), dtype=torch.bool, device="cuda")
    for b, (c, n) in enumerate(zip([125, 0, 510], new)):
        for j, e in ((n - 1, 3), (n // 2, dh - 1)):
            pr["v"][pr["table"][b, (c + j) // 8].item(), (c + j) % 8, :, e] = float("inf")
            pr["vals"][b][c + j, :, e] = float("inf")
            for i in range(n):
                hit[pr["start"][b] + i, :, e] = j in pr["seen"][b][i]
    want, bound = attention_oracle(pr)
    first = run_attention(zq, pr)
    got = first[:pr["rows"]].double()
    assert bool((got[hit] == float("inf")).all()) and bool(((got - want).abs() <= bound)[~hit].all())
    for _ in range(5):
        assert torch.equal(run_attention(zq, pr)[:pr["rows"]], first[:pr["rows"]])


@pytest.mark.parametrize("dtype,qa,ka", [("f16", 30000.0, 512.0), ("f16", -30000.0, 512.0), ("bf16", 2.0 ** 60, 2.0 ** 50), ("bf16", 2.0 ** 62, -2.0 ** 55),
                                         ("f32", 2.0 ** 60, -2.0 ** 50), ("f16", 2048.0, 512.0), ("bf16", 2.0 ** 12, 2.0 ** 15)])
@pytest.mark.parametrize("heads,new,cached", [(1, [2, 1], [300, 900]), (4, [6, 5], [300, 900]), (8, [6, 5], [900, 20]), (8, [40, 30], [900, 129])])
def test_scores_of_any_size(zq, dtype, qa, ka, heads, new, cached):
    # one product a score, exact in binary32, up to 2^117: the softmax is an even one over the keys with the largest score, however large
    pr = attention_problem(23, dtype, heads, 1, 128, 16, "token", cached, new, "tree")
    rng = np.random.default_rng(4)
    rows = pr["rows"]
    pr["q"][:rows] = 0
    pr["q"][:rows, :, 0] = qa
    want = torch.zeros((rows, heads, 128), dtype=torch.float64, device="cuda")
    size = want.clone()
    for b, (c, n) in enumerate(zip(cached, new)):
        step = torch.from_numpy(rng.integers(1, 90, c + n)).cuda()
        pr["keys"][b].zero_()
        pr["keys"][b][:, 0, 0] = (ka * step).to(TYPES[dtype])
        t = torch.arange(c + n, device="cuda")
        pr["k"][pr["table"][b].long()[t // 16], t % 16] = pr["keys"][b]
        v = pr["vals"][b][:, 0].double()
        s = pr["keys"][b][:, 0, 0].double() * qa
        assert bool((s.float().double() == s).all())
        for i in range(n):
            vis = t < c
            for j in pr["seen"][b][i]:
                vis[c + j] = True
            best = vis & (s == s[vis].max())
            want[pr["start"][b] + i] = v[best].mean(0)
            size[pr["start"][b] + i] = v[best].abs().mean(0)
    got, err = zq.zoqat_op_tree_attention(pr["q"], pr["k"], pr["v"], pr["table"], pr["kv_len"], pr["row_start"], tree_mask=pr["mask"], scale=1.0)
    assert err.item() == 0
    # the weights of all keys with the largest score are the same number; 16-bit weights and the output are rounded, sums are binary32
    half = torch.finfo(TYPES[dtype]).eps / 2
    bound = half * want.abs() + (0 if dtype == "f32" else half) * size * (1 + half) + 64 * 2.0 ** -24 * size + (2.0 ** -25 if dtype == "f16" else 0)
    assert bool(((got[:rows].double() - want).abs() <= bound).all())


LONG_REQUESTS = [
    # dtype, heads, kv, dh, page, layout, cached, new, mask
    ("bf16", 4, 4, 128, 16, "token", [129] + [40] * 40, [300] + [1] * 40, "tree"),     # one wide request among single tokens: tiles of 16 queries
    ("f16", 4, 2, 64, 32, "head", [0] + [300] * 40, [300] + [1] * 40, "tree"),         # of 32
    ("bf16", 8, 2, 64, 16, "joint", [250] + [7, 500] * 20, [290] + [1, 2] * 20, "random"),    # of 64
    ("f32", 4, 2, 128, 24, "token", [129] + [40] * 12, [300] + [1] * 12, "tree"),
    ("f16", 4, 2, 128, 64, "token", [0, 129], [700, 513], None),                       # chunks of a prompt
    ("bf16", 8, 2, 64, 16, "head", [129, 0], [700, 257], "tree"),
    ("f32", 2, 1, 64, 16, "head", [0, 129], [700, 513], None),
    ("bf16", 2, 2, 128, 128, "token", [0], [1000], "tree"),                            # masks of 32 words
    ("bf16", 8, 2, 128, 384, "token", [1200, 383, 0], [9, 2, 700], None),              # pages that are no power of two
    ("f16", 4, 4, 64, 640, "head", [1300, 639, 5], [1, 3, 2], "tree"),
]


@pytest.mark.parametrize("case", LONG_REQUESTS, ids=lambda c: "-".join(str(x) for x in c[:6]) + f"-n{max(c[7])}-{c[8]}")
def test_requests_with_many_rows(zq, case):
    dtype, heads, kv, dh, page, layout, cached, new, mask = case
    pr = attention_problem(29, dtype, heads, kv, dh, page, layout, cached, new, mask)
    got = run_attention(zq, pr)
    want, bound = attention_oracle(pr)
    off = (got[:pr["rows"]].double() - want).abs()
    assert bool((off <= bound).all()), (float(off.max()), float((off / bound.clamp(min=1e-30)).max()))
    assert torch.equal(run_attention(zq, pr)[:pr["rows"]], got[:pr["rows"]])


@pytest.mark.parametrize("dtype,heads,kv,new", [("bf16", 2, 2, [300] + [1] * 30), ("f16", 4, 2, [300] + [1] * 30), ("f16", 8, 2, [300, 290]), ("f32", 4, 2, [300, 3])])
@pytest.mark.parametrize("cached", [0, 70])
def test_rows_that_see_late_drafts_only(zq, dtype, heads, kv, new, cached):
    # rows whose first tiles of drafts are hidden whole, rows that see one draft, rows that see none
    pr = attention_problem(31, dtype, heads, kv, 128, 16, "token", [cached] * len(new), new, "tree")
    rng = np.random.default_rng(8)
    pr["seen"] = [[[set(range(140, n, 3)), {n - 1}, set(), set(np.nonzero(rng.random(n) < 0.1)[0].tolist())][i % 4] & set(range(n)) for i in range(n)] for n in new]
    words = pr["mask"].shape[1]
    pr["mask"][:pr["rows"]] = ints([words_of(s, words) for r in pr["seen"] for s in r])
    got = run_attention(zq, pr)
    want, bound = attention_oracle(pr)
    off = (got[:pr["rows"]].double() - want).abs()
    assert bool((off <= bound).all()), (float(off.max()), float((off / bound.clamp(min=1e-30)).max()))
    if cached == 0:
        assert bool((got[2] == 0).all())


@pytest.mark.parametrize("dtype,heads,kv,new", [("bf16", 8, 2, [5, 6, 4]), ("f16", 16, 2, [40, 33, 64]), ("f32", 4, 2, [2, 3, 1])])
def test_two_streams_at_once(zq, dtype, heads, kv, new):
    # a scratch each, eager calls and two graphs in flight; every call gives the bits of a call alone
    prs = [attention_problem(41 + i, dtype, heads, kv, 128, 16, "token", c, new, "tree") for i, c in enumerate(([900, 3000, 40], [2100, 11, 700]))]
    alone = [run_attention(zq, pr) for pr in prs]
    streams = [torch.cuda.Stream() for _ in prs]
    scratch = [torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda") for _ in prs]
    outs, errs = [torch.full_like(pr["q"], 5.0) for pr in prs], [torch.zeros(1, dtype=torch.int32, device="cuda") for _ in prs]
    torch.cuda.synchronize()

    def call(i):
        pr = prs[i]
        zq.zoqat_op_tree_attention(pr["q"], pr["k"], pr["v"], pr["table"], pr["kv_len"], pr["row_start"], tree_mask=pr["mask"], out=outs[i], scratch=scratch[i],
                                   err=errs[i])

    graphs = []
    for i, s in enumerate(streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            call(i)
        graphs.append(g)
    for rounds in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                outs[i].fill_(5.0)
                if rounds % 2:
                    call(i)
                else:
                    graphs[i].replay()
    torch.cuda.synchronize()
    for i, pr in enumerate(prs):
        assert errs[i].item() == 0 and torch.equal(outs[i][:pr["rows"]], alone[i][:pr["rows"]]) and bool((outs[i][pr["rows"]:] == 5.0).all())


def test_no_rows(zq):
    k, v = [torch.randn((4, 16, 2, 64), device="cuda").to(torch.bfloat16) for _ in range(2)]
    keep = k.clone()
    out, err = zq.zoqat_op_tree_attention(torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda"), k, v, ints([[0]]), ints([0]), ints([0, 0]),
                                          ints([[0]])[:0])
    q, err2 = zq.zoqat_op_cache_append(torch.empty((0, 512), device="cuda"), ints([0])[:0], ints([0])[:0], k, v, 4)
    assert out.shape == q.shape == (0, 4, 64) and err.item() == err2.item() == 0 and torch.equal(k, keep)


def test_attention_on_another_stream(zq):
    pr = attention_problem(2, "f16", 4, 4, 64, 32, "head", [200, 10], [3, 3], "tree")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = run_attention(zq, pr)
    side.synchronize()
    want, bound = attention_oracle(pr)
    assert bool(((got[:pr["rows"]].double() - want).abs() <= bound).all())


def test_attention_reads_the_decode_paths_own_cache_layout(zq):
    # [batch][heads][max_len][d_head] in fp32: a page per sequence
    gen = torch.Generator(device="cuda").manual_seed(1)
    B, H, M, dh, L = 3, 2, 50, 64, [50, 17, 1]
    k, v = [torch.randn((B, H, M, dh), generator=gen, device="cuda") for _ in range(2)]
    q = torch.randn((B, H, dh), generator=gen, device="cuda")
    out, err = zq.zoqat_op_tree_attention(q, k.transpose(1, 2), v.transpose(1, 2), ints([[0], [1], [2]]), ints(L), ints([0, 1, 2, 3]))
    assert err.item() == 0
    for b in range(B):
        w = torch.softmax(torch.einsum("hd,htd->ht", q[b].double(), k[b, :, :L[b]].double()) / 8.0, -1)
        want = torch.einsum("ht,htd->hd", w, v[b, :, :L[b]].double())
        assert float((out[b].double() - want).abs().max()) < 2e-5


# ---- rules ------------------------------------------------------------------------------------------------------------
def rules_oracle(x, dtype, request, rules, V):
    """The formula in numpy binary32, one rounding per operation, in the documented order."""
    x = x.float().cpu().numpy().copy()
    tokens = np.full(len(request), 99, dtype=np.int64)
    for r, b in enumerate(request):
        if b < 0:
            continue
        made, asked, bias, touched = np.zeros(V, dtype=np.int64), np.zeros(V, dtype=bool), np.zeros(V, dtype=np.float32), rules.get("bias") is not None
        if rules.get("history") is not None:
            hist, n, p = rules["history"][b], rules["history_len"][b], rules["prompt_len"][b] if rules.get("prompt_len") is not None else 0
            for k, t in enumerate(hist[:n]):
                if 0 <= t < V:
                    if k < p:
                        asked[t] = True
                    else:
                        made[t] += 1
        if rules.get("drafts") is not None:
            for j in rules["seen"][r]:
                t = rules["drafts"][rules["row_start"][b] + j]
                if 0 <= t < V:
                    made[t] += 1
        if touched:
            for t, w in rules["bias"][b]:
                if 0 <= t < V:
                    bias[t] = np.float32(bias[t] + np.float32(w))
        rep, freq, pres = [np.float32(rules[k][b]) if rules.get(k) is not None else np.float32(d) for k, d in (("repetition", 1), ("frequency", 0), ("presence", 0))]
        row = x[r]
        old = asked | (made > 0)
        with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
            row = np.where(old, np.where(row > 0, row / rep, row * rep), row).astype(np.float32)
            row = np.where(old, row - freq * made.astype(np.float32), row).astype(np.float32)
            row = np.where(made > 0, row - pres, row).astype(np.float32)
            if touched and len(rules["bias"][b]):
                row = (row + bias).astype(np.float32)
        if rules.get("allowed") is not None:
            row = np.where(rules["allowed"][r], row, np.float32(-np.inf))
        x[r] = row
        y = torch.from_numpy(row).to(TYPES[dtype]).float().numpy()
        best = -1
        for t in np.argsort(-np.where(np.isnan(y), -np.inf, y), kind="stable")[:1]:
            best = int(t) if y[t] > -np.inf else -1
        tokens[r] = best
    return torch.from_numpy(x).to(TYPES[dtype]), tokens


def pack_bits(ok):
    n = -(-ok.shape[1] // 32) * 32
    full = np.zeros((ok.shape[0], n), dtype=np.uint8)
    full[:, :ok.shape[1]] = ok
    return torch.from_numpy(np.packbits(full, axis=1, bitorder="little").view(np.int32).copy()).cuda()


@pytest.mark.parametrize("dtype,V,batch,per,groups", [
    ("f32", 1, 1, 1, "h"), ("f32", 1000, 3, 1, ""), ("f32", 32000, 2, 3, "hpdba"), ("bf16", 50257, 2, 2, "hpdba"), ("f16", 777, 5, 4, "hpdb"),
    ("f32", 131072, 1, 1, "hpb"), ("bf16", 4097, 40, 1, "a"), ("f32", 65537, 2, 1, "b"), ("f16", 8193, 3, 2, "d"), ("f32", 5000, 3, 1, "hba")])
def test_rules_match_the_formula_bit_for_bit(zq, dtype, V, batch, per, groups):
    check_rules(zq, dtype, V, batch, per, groups)


# rows on 16-byte boundaries, taken in vectors; histories of more distinct tokens than are counted at a time; a vocabulary of
# several slices (one CTA per row)
@pytest.mark.parametrize("dtype,V,batch,per,groups,hist,skew", [
    ("f32", 1000, 3, 2, "hpdba", 600, 6), ("bf16", 50264, 2, 2, "hpdba", 600, 6), ("f16", 776, 5, 4, "hpdb", 600, 6), ("bf16", 8, 2, 1, "hba", 600, 6),
    ("f32", 50272, 2, 2, "hpdba", 20000, 1), ("f16", 40000, 150, 1, "hpb", 9000, 1), ("f32", 70016, 150, 1, "hpa", 600, 1)])
def test_rules_on_aligned_rows(zq, dtype, V, batch, per, groups, hist, skew):
    check_rules(zq, dtype, V, batch, per, groups, pad=8, H=hist, skew=skew)


def check_rules(zq, dtype, V, batch, per, groups, pad=3, H=600, skew=6):
    rng = np.random.default_rng(V)
    rows = batch * per
    request = [r // per for r in range(rows)]
    if rows > 3:
        request[1] = -1                                                  # a padded row is left as it is
    slab = torch.from_numpy((4 * rng.standard_normal((rows, V + pad))).astype(np.float32)).to(TYPES[dtype]).cuda()
    logits = slab[:, :V]
    R, kw = {}, {}
    if "h" in groups:
        hist = np.minimum((V * rng.random((batch, H)) ** skew).astype(np.int64), V - 1)
        hist[:, 7], hist[:, 11] = V, -1                                  # not tokens
        R.update(history=hist.tolist(), history_len=rng.integers(0, H + 1, batch).tolist())
        kw.update(history=ints(hist.tolist()), history_len=ints(R["history_len"]))
        if "p" in groups:
            R["prompt_len"] = [n // 3 for n in R["history_len"]]
            kw["prompt_len"] = ints(R["prompt_len"])
    if "h" in groups or "d" in groups:
        for n, lo, hi in (("repetition", 0.8, 1.7), ("presence", -0.5, 1.0), ("frequency", 0.0, 0.3)):
            R[n] = rng.uniform(lo, hi, batch).astype(np.float32).tolist()
            kw[n] = torch.tensor(R[n], dtype=torch.float32, device="cuda")
    if "b" in groups:
        B = 70
        tok = rng.integers(0, V, (batch, B))
        tok[:, 1::3] = tok[:, :1]                                         # the same token many times
        tok[:, 5], tok[:, 6] = V + 5, -1
        val = (3 * rng.standard_normal((batch, B))).astype(np.float32)
        n = rng.integers(0, B + 1, batch)
        n[0] = B
        R["bias"] = [list(zip(tok[b, :n[b]].tolist(), val[b, :n[b]].tolist())) for b in range(batch)]
        kw.update(bias_token=ints(tok.tolist()), bias_value=torch.from_numpy(val).cuda(), bias_len=ints(n.tolist()))
    if "a" in groups:
        ok = rng.random((rows, V)) < 0.5
        ok[0] = False                                                     # nothing is allowed
        R["allowed"] = ok
        kw["allowed"] = pack_bits(ok)
    if "d" in groups:
        R["drafts"] = rng.integers(-1, V + 1, rows).tolist()
        R["row_start"] = [per * b for b in range(batch + 1)]
        R["seen"] = [{j for j in range(r % per + 1) if j == r % per or rng.random() < 0.5} for r in range(rows)]
        kw.update(draft_token=ints(R["drafts"]), row_start=ints(R["row_start"]), tree_mask=ints([words_of(s, 1) for s in R["seen"]]))
    want, token = rules_oracle(logits, dtype, request, R, V)
    rules = zq.LogitRules(batch=batch, row_request=ints(request), **kw)
    out, tok = zq.zoqat_op_logit_rules(logits, rules, out=torch.full_like(logits, 3.0), token=ints([99] * rows))
    want[[r for r in range(rows) if request[r] < 0]] = 3.0
    assert tok.tolist() == token.tolist()
    assert torch.equal(out.cpu(), want)
    _, only = zq.zoqat_op_logit_rules(logits, rules, want_logits=False, token=ints([99] * rows))
    assert only.tolist() == token.tolist()
    keep = slab.clone()
    zq.zoqat_op_logit_rules(logits, rules, out=logits, token=ints([99] * rows))                     # in place
    live = [r for r in range(rows) if request[r] >= 0]
    assert torch.equal(logits[live].cpu(), want[live]) and torch.equal(slab[:, V:], keep[:, V:])


def test_rules_choice_with_ties_infinities_and_nan(zq):
    V = 9000
    x = torch.zeros((4, V), device="cuda")
    x[1] = -float("inf")
    x[2] = float("nan")
    x[2, 8999] = -5.0
    x[3, 4000:] = float("inf")
    _, tok = zq.zoqat_op_logit_rules(x, zq.LogitRules(batch=4))
    assert tok.tolist() == [0, -1, 8999, 4000]


# ---- the largest sizes ---------------------------------------------------------------------------------------------------
def test_plan_of_the_largest_batch(zq):
    # 16384 requests, more rows than one pass of the grid; chains, checked in closed form
    rng = np.random.default_rng(5)
    batch, page, words = 16384, 16, 1
    cached, new = rng.integers(0, 100, batch), rng.integers(0, 32, batch)
    held, kv = -(-cached // page), cached + new
    need = -(-kv // page) - held
    start, first = np.concatenate([[0], np.cumsum(new)]), np.concatenate([[0], np.cumsum(need)])
    max_pages, n_pages, rows = 9, int(held.sum() + need.sum()) + 3, int(new.sum())
    assert rows > 148 * 1024
    order = rng.permutation(n_pages)
    table = np.full((batch, max_pages), -7)
    table[np.arange(max_pages)[None] < held[:, None]] = order[:held.sum()]
    free = order[held.sum():]
    t = torch.from_numpy(table).to(torch.int32).cuda()
    got = zq.zoqat_op_cache_plan(ints(cached.tolist()), ints(new.tolist()), page, n_pages, ints(free.tolist()), ints([len(free)]), t, rows + 7, mask_words=words)
    fresh = (np.arange(max_pages)[None] >= held[:, None]) & (np.arange(max_pages)[None] < (held + need)[:, None])
    table[fresh] = free[len(free) - 1 - np.arange(need.sum())]
    request = np.repeat(np.arange(batch), new)
    i = np.arange(rows) - start[request]
    at = cached[request] + i
    pad = lambda x, v: np.concatenate([x, np.full(7, v)])  # noqa: E731
    want = dict(kv_len=kv, row_start=start, row_request=pad(request, -1), row_pos=pad(at, -1), slot=pad(table[request, at // page] * page + at % page, -1),
                n_free=[len(free) - first[-1]], status=[0])
    for n, w in want.items():
        assert np.array_equal(got[n].cpu().numpy(), w), n
    mask = pad((1 << (i + 1).astype(np.int64)) - 1, 0)
    assert np.array_equal(got["tree_mask"][:, 0].cpu().numpy().view(np.uint32).astype(np.int64), mask) and np.array_equal(t.cpu().numpy(), table)


@pytest.mark.parametrize("dtype,layout", [("bf16", "token"), ("f16", "head"), ("f32", "token")])
def test_pages_behind_32_bits(zq, dtype, layout):
    # a cache of more than 2^32 elements, its last pages in use: append, then attention with few and with many queries
    page, kv, dh, heads = 16, 8, 128, 32
    n_pages = 2 ** 32 // (page * kv * dh) + 200
    shape = (n_pages, page, kv, dh) if layout == "token" else (n_pages, kv, page, dh)
    k, v = [torch.empty(shape, dtype=TYPES[dtype], device="cuda") for _ in range(2)]
    if layout == "head":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    gen = torch.Generator(device="cuda").manual_seed(3)
    for n in (1, 40):
        C = 300
        L, used = C + n, -(-(C + n) // page)
        pages = [n_pages - 1 - 5 * i for i in range(used)]
        qkv = torch.randn((L, (heads + 2 * kv) * dh), generator=gen, device="cuda")
        slot = [pages[t // page] * page + t % page for t in range(L)]
        q, err = zq.zoqat_op_cache_append(qkv, ints([0] * L), ints(slot), k, v, heads)
        assert err.item() == 0
        x = qkv.view(L, heads + 2 * kv, dh)
        t = torch.arange(L, device="cuda")
        at = torch.tensor(pages, device="cuda")[t // page]
        assert torch.equal(k[at, t % page], x[:, heads:heads + kv].to(TYPES[dtype])) and torch.equal(v[at, t % page], x[:, heads + kv:].to(TYPES[dtype]))
        pr = dict(dtype=dtype, q=q[C:], k=k, v=v, table=ints([pages]), kv_len=ints([L]), row_start=ints([0, n]), mask=None, rows=n, start=[0, n], new=[n], L=[L],
                  keys=[x[:, heads:heads + kv].to(TYPES[dtype])], vals=[x[:, heads + kv:].to(TYPES[dtype])], seen=[[set(range(i + 1)) for i in range(n)]],
                  heads=heads, kv=kv, dh=dh, scale=1.0 / math.sqrt(dh))
        got = run_attention(zq, pr)
        want, bound = attention_oracle(pr)
        assert bool(((got.double() - want).abs() <= bound).all())


def test_requests_that_share_pages(zq):
    # two requests with the same prefix pages, each with drafts in a page of its own; and the same request twice
    pr = attention_problem(6, "bf16", 8, 2, 128, 16, "token", [96, 96], [3, 3], "tree")
    pr["table"][1, :6] = pr["table"][0, :6]
    pr["keys"][1][:96], pr["vals"][1][:96] = pr["keys"][0][:96], pr["vals"][0][:96]
    want, bound = attention_oracle(pr)
    got = run_attention(zq, pr)
    assert bool(((got[:6].double() - want).abs() <= bound).all())
    pr["table"][1] = pr["table"][0]
    pr["q"][3:6], pr["mask"][3:6] = pr["q"][:3], pr["mask"][:3]
    got = run_attention(zq, pr)
    assert bool(((got[:3].double() - want[:3]).abs() <= bound[:3]).all()) and bool(((got[3:6].double() - want[:3]).abs() <= bound[:3]).all())


def test_rules_on_the_largest_batch(zq):
    # 65535 rows of logits, 2.6e9 elements: the last rows as in a call of their own
    rows, V, batch = 65535, 40008, 7
    gen = torch.Generator(device="cuda").manual_seed(2)
    logits = torch.empty((rows, V), dtype=torch.bfloat16, device="cuda")
    few = torch.randn((64, V), generator=gen, device="cuda").to(torch.bfloat16)
    logits.view(-1)[: 64 * V] = few.view(-1)
    logits[64:] = 0
    logits[-64:] = few.flip(0)
    allowed = torch.randint(-2 ** 31, 2 ** 31, (rows, -(-V // 32)), generator=gen, device="cuda").to(torch.int32)
    request = (torch.arange(rows, device="cuda") % batch).to(torch.int32)
    history = torch.randint(0, V, (batch, 500), generator=gen, device="cuda").to(torch.int32)
    kw = dict(history=history, history_len=ints([500, 0, 3, 77, 500, 250, 1]), repetition=torch.full((batch,), 1.2, device="cuda"),
              presence=torch.full((batch,), 0.3, device="cuda"), frequency=torch.full((batch,), 0.1, device="cuda"))
    out, tok = zq.zoqat_op_logit_rules(logits, zq.LogitRules(row_request=request, allowed=allowed, **kw))
    for part in (slice(0, 64), slice(rows - 64, rows)):
        one, t1 = zq.zoqat_op_logit_rules(logits[part].clone(), zq.LogitRules(row_request=request[part].clone(), allowed=allowed[part].clone(), **kw))
        assert torch.equal(out[part], one) and torch.equal(tok[part], t1)


# ---- the operators together ---------------------------------------------------------------------------------------------
MODELS = {
    "llama_w4a8": dict(arch="llama", n_layers=2, d_model=256, n_heads=2, d_ffn=512, vocab=600, w_bits=4, w_group=64, a_bits=8),
    "llama_w4": dict(arch="llama", n_layers=2, d_model=128, n_heads=2, d_ffn=384, vocab=600, w_bits=4, w_group=128, a_bits=0),
    "opt_w3a8": dict(arch="opt", n_layers=2, d_model=128, n_heads=2, d_ffn=256, vocab=333, w_bits=3, w_group=128, a_bits=8),
}


def packed_model(zq, name, batch, seq):
    from paper_2509_00031_b200 import synth
    shape = MODELS[name]
    params = synth.make_params(shape, seed=5, max_seq=seq, jitter=True)
    model = zq.ZoqatModel(shape, zq.params_to_device(params), max_batch=batch, max_seq=seq, first_trainable_layer=shape["n_layers"], head_trainable=False,
                          packed_frozen=True)
    model.zoqat_prequantize_frozen()
    model.zoqat_decode_begin(batch, seq)
    return shape, model


class Serving:
    """A serving loop's state: lengths, pages and their tables, advanced by the operators alone."""

    def __init__(self, zq, shape, model, batch, page, dtype, max_rows=8):
        self.zq, self.model, self.page, self.batch, self.rows = zq, model, page, batch, max_rows
        self.cached, self.n_pages = [0] * batch, 40
        dh = shape["d_model"] // shape["n_heads"]
        self.caches = [make_cache(self.n_pages, page, shape["n_heads"], dh, dtype, "token") for _ in range(shape["n_layers"])]
        self.table = torch.full((batch, 12), -1, dtype=torch.int32, device="cuda")
        self.free = torch.randperm(self.n_pages, generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda()
        self.n_free = ints([self.n_pages])

    def step(self, tokens, parents=None, rules=None, keep=True):
        """tokens, parents: one list per request.  Returns logits and choices of the live rows, and the plan."""
        flat = [t for r in tokens for t in r]
        par = [t for r in parents for t in r] if parents else None
        pad = self.rows - len(flat)
        plan = self.zq.zoqat_op_cache_plan(ints(self.cached), ints([len(r) for r in tokens]), self.page, self.n_pages, self.free, self.n_free, self.table,
                                           self.rows, parents=ints(par + [-1] * pad) if par else None, mask_words=1)
        assert plan["status"].item() == 0
        if rules is not None:
            rules = self.zq.LogitRules(row_request=plan["row_request"], draft_token=ints(flat + [0] * pad), row_start=plan["row_start"],
                                       tree_mask=plan["tree_mask"], batch=self.batch, **rules)
        logits, choice = self.model.zoqat_decode_tree_step(ints(flat + [0] * pad), plan, self.table, self.caches, rules=rules)
        self.model.zoqat_check()
        if keep:
            self.n_free = plan["n_free"]
            self.cached = plan["kv_len"].tolist()
        return logits[:len(flat)], choice[:len(flat)], plan


def sequential_logits(model, tokens, batch):
    """Logits after the last of `tokens`, by the one-token decode path."""
    for pos, t in enumerate(tokens):
        logits, _ = model.zoqat_decode_step(ints([t] * batch), pos)
    return logits[0].clone()


@pytest.mark.parametrize("name,dtype,page", [("llama_w4a8", "f32", 16), ("llama_w4", "bf16", 8), ("opt_w3a8", "f16", 16), ("llama_w4a8", "f32", 5),
                                             ("opt_w3a8", "f32", 7)])
def test_drafts_through_the_model_match_the_one_token_path(zq, name, dtype, page):
    # three requests of different lengths, prompts fed in chunks, then one step with a tree per request: every row's logits against the
    # one-token decode path fed the prompt and the row's ancestors
    batch = 2
    shape, model = packed_model(zq, name, batch, 64)
    _, other = packed_model(zq, name, batch, 64)
    rng = np.random.default_rng(1)
    prompts = [rng.integers(0, shape["vocab"], n).tolist() for n in (9, 17, 1)]
    sv = Serving(zq, shape, model, 3, page, dtype)
    todo = [list(p) for p in prompts]
    while any(todo):
        share = [min(len(t), 3) for t in todo]
        sv.step([t[:n] for t, n in zip(todo, share)])
        todo = [t[n:] for t, n in zip(todo, share)]
    assert sv.cached == [9, 17, 1]
    drafts = [rng.integers(0, shape["vocab"], n).tolist() for n in (4, 3, 1)]
    parents = [[-1, 0, 0, 2], [-1, -1, 1], [-1]]
    logits, choice, plan = sv.step(drafts, parents, keep=False)
    # a difference of one code in one activation moves a row by up to one step (1 / 127 of its largest value, 2^-8 of a bf16 value);
    # 16-bit caches round every key and value once
    tol = {"f32": 2e-2, "f16": 2e-2, "bf16": 5e-2}[dtype]
    row = 0
    for b in range(3):
        for i in range(len(drafts[b])):
            path = [drafts[b][j] for j in sorted(ancestors(parents[b], i))]
            want = sequential_logits(other, prompts[b] + path, batch)
            assert float((logits[row] - want).abs().max()) <= tol * float(want.abs().max()), (b, i)
            assert choice[row].item() == int(torch.argmax(logits[row]))
            row += 1
    # the same step again, with rules: the choices are those of the rules on these logits
    V = shape["vocab"]
    history = torch.zeros((3, 20), dtype=torch.int32, device="cuda")
    for b in range(3):
        history[b, :len(prompts[b])] = ints(prompts[b])
    rules = dict(history=history, history_len=ints([9, 17, 1]), prompt_len=ints([4, 17, 0]), repetition=torch.full((3,), 1.3, device="cuda"),
                 presence=torch.full((3,), 0.2, device="cuda"), frequency=torch.full((3,), 0.1, device="cuda"))
    ruled, token, plan = sv.step(drafts, parents, rules=dict(rules), keep=False)
    seen = [set(ancestors(parents[b], i)) for b in range(3) for i in range(len(drafts[b]))]
    want, best = rules_oracle(logits, "f32", plan["row_request"].tolist()[:8], dict(
        history=history.tolist(), history_len=[9, 17, 1], prompt_len=[4, 17, 0], repetition=[1.3] * 3, presence=[0.2] * 3, frequency=[0.1] * 3,
        drafts=[t for r in drafts for t in r], row_start=[0, 4, 7, 8], seen=seen), V)
    assert torch.equal(ruled.cpu(), want) and token.tolist() == best.tolist()
    # one request accepts a branch: its drafts' slots are overwritten by the next step, and the others go on as they were
    sv.cached = [9, 17, 1]
    logits2, _, _ = sv.step([[drafts[0][0]], [], [drafts[2][0], 5]])
    assert float((logits2[0] - logits[0]).abs().max()) <= tol * float(logits[0].abs().max())


def test_a_captured_tree_step_replays_with_new_lengths(zq):
    shape, model = packed_model(zq, "llama_w4a8", 2, 64)
    sv = Serving(zq, shape, model, 2, 16, "bf16", max_rows=4)
    sv.step([[3, 4], [5]])
    cached, new, tokens = ints(sv.cached), ints([1, 1]), ints([7, 8, 0, 0])
    n_free = sv.n_free.clone()
    out = {n: torch.empty(s, dtype=torch.int32, device="cuda") for n, s in dict(kv_len=(2,), row_start=(3,), row_request=(4,), row_pos=(4,), slot=(4,), n_free=(1,),
                                                                               tree_mask=(4, 1)).items()}
    out["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    logits, nxt = torch.empty((4, shape["vocab"]), device="cuda"), torch.empty(4, dtype=torch.int32, device="cuda")
    scratch = torch.empty(48 << 20, dtype=torch.uint8, device="cuda")

    def run():
        zq.zoqat_op_cache_plan(cached, new, 16, sv.n_pages, sv.free, n_free, sv.table, 4, mask_words=1, out=out)
        model.zoqat_decode_tree_step(tokens, out, sv.table, sv.caches, logits=logits, next_token=nxt, scratch=scratch)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for lens, n in (([2, 1], [1, 1]), ([3, 2], [2, 1]), ([5, 3], [0, 3])):
        cached.copy_(ints(lens)); new.copy_(ints(n)); tokens.copy_(ints([9, 10, 11, 12]))
        logits.fill_(0.0)
        graph.replay()
        torch.cuda.synchronize()
        model.zoqat_check()
        got = logits.clone()
        run()
        torch.cuda.synchronize()
        rows = sum(n)
        assert out["status"].item() == 0 and out["row_start"].tolist()[-1] == rows
        assert torch.equal(got[:rows], logits[:rows]) and bool(torch.isfinite(got[:rows]).all())


def test_tree_step_refuses_and_reports(zq):
    shape, model = packed_model(zq, "llama_w4a8", 2, 64)
    sv = Serving(zq, shape, model, 1, 16, "f32", max_rows=2)
    _, _, plan = sv.step([[3]])
    ok = lambda **kw: model.zoqat_decode_tree_step(kw.pop("tokens", ints([1, 2])), kw.pop("plan", plan), sv.table, kw.pop("caches", sv.caches), **kw)  # noqa: E731
    ok()
    for kw in (dict(tokens=ints([1, 2, 3])), dict(caches=sv.caches[:1]), dict(caches=[make_cache(4, 16, 1, 128, "f32", "token")] * 2),
               dict(scratch=torch.empty(4096, dtype=torch.uint8, device="cuda")), dict(caches=[make_cache(4, 12, 2, 128, "bf16", "token")] * 2),
               dict(logits=torch.empty((2, 5), device="cuda"))):
        with pytest.raises(zq.ZoqatError):
            ok(**kw)
    # a position behind the tables is reported by the check
    bad = dict(plan, row_pos=ints([64, -1]))
    ok(plan=bad)
    with pytest.raises(zq.ZoqatError) as e:
        model.zoqat_check()
    assert e.value.status == zq.ERR_INVALID_ARG
    model.zoqat_check()


@pytest.mark.parametrize("name", ["opt_w3a8", "llama_w4a8"])
def test_tree_step_leaves_the_pages_of_rows_with_a_bad_position(zq, name):
    # models with position embeddings and models with rotary tables alike: no key and no value of such a row is stored
    shape, model = packed_model(zq, name, 2, 64)
    sv = Serving(zq, shape, model, 1, 16, "f32", max_rows=2)
    _, _, plan = sv.step([[3, 4]])
    model.zoqat_check()
    for pos, kept in (([0, 64], 0), ([64, 1], 1), ([0, -1], 0)):
        for k, v in sv.caches:
            k.fill_(5.0); v.fill_(5.0)
        model.zoqat_decode_tree_step(ints([3, 4]), dict(plan, row_pos=ints(pos)), sv.table, sv.caches)
        with pytest.raises(zq.ZoqatError) as e:
            model.zoqat_check()
        assert e.value.status == zq.ERR_INVALID_ARG
        model.zoqat_check()
        page, off = [x // 16 for x in plan["slot"].tolist()], [x % 16 for x in plan["slot"].tolist()]
        for k, v in sv.caches:
            for c in (k, v):
                assert bool((c[page[kept], off[kept]] != 5.0).any())
                c[page[kept], off[kept]] = 5.0
                assert bool((c == 5.0).all()), (pos, "a row that was to be skipped")


def test_tree_step_checks_every_cache_before_it_starts(zq):
    # a cache that the attention cannot address is refused before the first layer has stored anything
    shape, model = packed_model(zq, "llama_w4a8", 2, 64)
    sv = Serving(zq, shape, model, 1, 16, "bf16", max_rows=2)
    _, _, plan = sv.step([[3]])
    for k, v in sv.caches:
        k.fill_(5.0); v.fill_(5.0)
    dev = torch.cuda.current_device()
    good = [zq._caches(dev, k, v) for k, v in sv.caches]
    tokens, nxt, scratch = ints([1, 2]), ints([9, 9]), torch.empty(48 << 20, dtype=torch.uint8, device="cuda")
    tb = zq.TreeBatch(sv.table.data_ptr(), plan["kv_len"].data_ptr(), plan["row_start"].data_ptr(), plan["row_pos"].data_ptr(), plan["slot"].data_ptr(),
                      plan["tree_mask"].data_ptr(), 1, sv.table.shape[1], 1, 0)
    for n_pages, page, slot in ((1 << 20, 128 << 12, 256), (2, 1 << 37, 1 << 36)):
        last = zq.PagedCache(good[1].k, good[1].v, good[1].type, n_pages, 16, 2, 128, 0, page, slot, 128)
        rc = zq.lib().zoqat_decode_tree_step(model.handle, tokens.data_ptr(), 2, tb, (zq.PagedCache * 2)(good[0], last), None, None, nxt.data_ptr(),
                                             scratch.data_ptr(), scratch.numel(), torch.cuda.current_stream().cuda_stream)
        assert rc == zq.ERR_UNSUPPORTED
    torch.cuda.synchronize()
    assert nxt.tolist() == [9, 9] and all(bool((c == 5.0).all()) for kv in sv.caches for c in kv)
