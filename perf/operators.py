"""The operators of serving drafted tokens over a paged key/value cache, as cases to measure.

Four operators that a serving loop runs one after the other for every step of a batch of requests:

  plan    block tables, slots, positions and tree masks from the requests' lengths and the drafts' parents
  append  rotary embedding of the new rows, their keys and values written into the pages
  attend  attention of the drafted rows over the cached positions and their own ancestors
  rules   penalties for repeated tokens, biases and grammar masks on the logits, then the greedy choice

Where ``own`` is false ``run`` computes them with elementary torch operations in 32 bits; where it is true it calls the
package's entry points.  ``exact`` gives the floating outputs from the definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


# ---- cases ------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one step of a small interactive batch: a token for each request, latency is what counts
        dict(name="plan_decode_small", op="plan", batch=8, page=16, len_lo=1, len_hi=1500, new_lo=1, new_hi=1, words=0),
        # a large serving batch, every request with a tree of drafted tokens
        dict(name="plan_trees_b1024", op="plan", batch=1024, page=16, len_lo=0, len_hi=4095, new_lo=1, new_hi=64, words=2),
        # prompts that enter the cache whole: many rows, no trees
        dict(name="plan_prompts_b64", op="plan", batch=64, page=64, len_lo=0, len_hi=777, new_lo=200, new_hi=4001, words=0),
        # the new rows of one layer in a decode step of 8 rows
        dict(name="append_decode_bf16", op="append", rows=8, heads=32, kv_heads=32, d_head=128, page=16, rope_len=2048, dtype="bf16",
             layout="token"),
        # a prompt chunk entering the cache, grouped heads, pages laid out head by head
        dict(name="append_chunk_f16", op="append", rows=8191, heads=40, kv_heads=8, d_head=128, page=64, rope_len=16384, dtype="f16",
             layout="head"),
        # one request, one token, a short context: the smallest call of a decode loop
        dict(name="attend_one_token", op="attend", batch=1, heads=32, kv_heads=32, d_head=128, page=16, len_lo=777, len_hi=777,
             new_lo=1, new_hi=1, dtype="bf16", layout="token"),
        # a serving batch with ragged contexts and small trees, grouped heads
        dict(name="attend_trees_b32", op="attend", batch=32, heads=32, kv_heads=8, d_head=128, page=16, len_lo=500, len_hi=8191,
             new_lo=1, new_hi=16, dtype="bf16", layout="token"),
        # 64-wide heads, binary16, pages laid out head by head
        dict(name="attend_d64_f16", op="attend", batch=16, heads=32, kv_heads=32, d_head=64, page=32, len_lo=100, len_hi=2047,
             new_lo=8, new_hi=8, dtype="f16", layout="head"),
        # the type of the package's own decode cache
        dict(name="attend_f32_b8", op="attend", batch=8, heads=32, kv_heads=32, d_head=128, page=64, len_lo=1, len_hi=1020,
             new_lo=1, new_hi=4, dtype="f32", layout="token"),
        # long documents with wide trees: where the products count as much as the bytes
        dict(name="attend_long_trees", op="attend", batch=4, heads=32, kv_heads=8, d_head=128, page=64, len_lo=60001, len_hi=120000,
             new_lo=64, new_hi=64, dtype="bf16", layout="token"),
        # one request's next token under penalties
        dict(name="rules_one_row", op="rules", batch=1, per=1, vocab=32000, hist=700, bias=20, mask=False, dtype="f32"),
        # the rows of a batch of drafts: penalties over history and ancestors, biases, a grammar mask
        dict(name="rules_drafts", op="rules", batch=64, per=4, vocab=50272, hist=3000, bias=200, mask=True, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choice(["plan", "append", "attend", "attend", "rules"])
        if op == "plan":
            words = rng.choice([0, 1, 2, 4])
            new_hi = _log(rng, 1, 32 * words) if words else _log(rng, 1, 4000)
            lo = rng.randrange(0, 1 + 300)
            c = dict(op=op, batch=_log(rng, 1, 2000), page=rng.choice([16, 32, 64, 128]), len_lo=lo, len_hi=lo + _log(rng, 1, 8000),
                     new_lo=rng.randrange(0, new_hi + 1), new_hi=new_hi, words=words)
            if c["batch"] * (32 * words) ** 2 > 4_200_000 or sum(_new(c)) > 130_000 or sum(_new(c)) == 0:
                continue
        elif op == "append":
            kv = rng.choice([1, 2, 8, 32])
            rows = _log(rng, 1, 8191)
            c = dict(op=op, rows=rows, heads=kv * rng.choice([1, 2, 4] if kv > 2 else [1, 4, 8]), kv_heads=kv, d_head=rng.choice([64, 128]),
                     page=rng.choice([16, 32, 64, 128]), rope_len=rng.choice([1, 2]) * 8192, dtype=rng.choice(list(DTYPES)),
                     layout=rng.choice(["token", "head"]))
            if rows * (c["heads"] + 2 * kv) * c["d_head"] > 58_000_000:
                continue
        elif op == "attend":
            dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
            kv = rng.choice([1, 2, 4, 8, 32])
            g = rng.choice([1, 2, 4, 7, 8]) if kv < 32 else 1
            new_hi = _log(rng, 1, 64 if dtype != "f32" else 8)
            lo = rng.randrange(0, 700)
            c = dict(op=op, batch=_log(rng, 1, 128), heads=kv * g, kv_heads=kv, d_head=rng.choice([64, 128]),
                     page=rng.choice([16, 32, 64, 128]), len_lo=lo, len_hi=lo + _log(rng, 1, 60000 if dtype != "f32" else 4000),
                     new_lo=rng.randrange(0, new_hi + 1), new_hi=new_hi, dtype=dtype, layout=rng.choice(["token", "head"]))
            padded = c["batch"] * (c["len_hi"] + c["new_hi"])
            if padded * kv * c["d_head"] > 490_000_000 or padded * c["heads"] * c["new_hi"] > 980_000_000:
                continue
        else:
            c = dict(op=op, batch=_log(rng, 1, 128), per=rng.choice([1, 1, 3, 8]), vocab=_log(rng, 5000, 131072), hist=_log(rng, 1, 20000),
                     bias=rng.choice([0, 1, 33, 300]), mask=rng.random() < 0.5, dtype=rng.choice(list(DTYPES)))
            if c["batch"] * c["per"] * c["vocab"] > 12_800_000:
                continue
        return c


def _spread(lo, hi, n, step):
    """n whole numbers between lo and hi (both among them where n > 1), in a scattered order."""
    if n == 1:
        return [hi]
    while math.gcd(step, n) != 1:
        step += 1
    return [lo + (hi - lo) * ((i * step) % n) // (n - 1) for i in range(n)]


def _cached(c):
    return _spread(c["len_lo"], c["len_hi"], c["batch"], 7)


def _new(c):
    return _spread(c["new_lo"], c["new_hi"], c["batch"], 11)


def _pages(n, page):
    return -(-n // page)


# ---- inputs -----------------------------------------------------------------------------------------------------
def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _parents(new, gen):
    """Drafts of every request back to back: the first hangs on the context, each other on one of the few before it."""
    local = torch.cat([torch.arange(n) for n in new])
    back = 1 + (torch.rand(local.numel(), generator=gen) * 5).long()
    return torch.clamp(local - back, min=0).where(local > 0, torch.tensor(-1)).to(torch.int32)


def _reach(parents, row_start, request, local, n_max):
    """[batch, n_max, n_max] of 0 and 1: which drafts of its request a draft sees (its ancestors and itself)."""
    batch = row_start.numel() - 1
    step = torch.zeros((batch, n_max, n_max), dtype=torch.float32, device=parents.device)
    has = (parents >= 0).float()
    step[request, local, parents.long().clamp(min=0)] = has
    reach = step + torch.eye(n_max, device=parents.device)
    for _ in range(max(1, (n_max - 1).bit_length())):        # paths of up to 2, 4, 8, ... edges
        reach = (reach @ reach).clamp(max=1.0)
    return reach


def _pack(bits):
    """0 / 1 in the last dimension (a multiple of 32) -> 32-bit words."""
    w = bits.reshape(*bits.shape[:-1], -1, 32).long() << torch.arange(32, device=bits.device)
    w = w.sum(-1)
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32)


def _cache(n_pages, page, kv_heads, d_head, dtype, layout, gen):
    if layout == "token":
        make = lambda: torch.randn((n_pages, page, kv_heads, d_head), generator=gen, device="cuda", dtype=torch.float32).to(DTYPES[dtype])  # noqa: E731
        return make(), make()
    make = lambda: torch.randn((n_pages, kv_heads, page, d_head), generator=gen, device="cuda", dtype=torch.float32).to(DTYPES[dtype])  # noqa: E731
    return make().transpose(1, 2), make().transpose(1, 2)


def prepare(case, seed):
    host = torch.Generator().manual_seed(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"plan": _prepare_plan, "append": _prepare_append, "attend": _prepare_attend, "rules": _prepare_rules}[case["op"]](case, host, gen)


def _prepare_plan(c, host, gen):
    cached, new, page = _cached(c), _new(c), c["page"]
    batch, rows = c["batch"], sum(new) + 5
    held = [_pages(x, page) for x in cached]
    need = sum(_pages(x + y, page) for x, y in zip(cached, new))
    max_pages = max(_pages(x + y, page) for x, y in zip(cached, new)) + 1
    n_pages = need + 9
    order = torch.randperm(n_pages, generator=host).to(torch.int32)
    table = torch.full((batch, max_pages), -1, dtype=torch.int32)
    taken = torch.arange(max_pages).unsqueeze(0) < torch.tensor(held).unsqueeze(1)
    table[taken] = order[: sum(held)]
    free = order[sum(held):]
    i32 = lambda *shape: torch.empty(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    out = dict(kv_len=i32(batch), row_start=i32(batch + 1), row_request=i32(rows), row_pos=i32(rows), slot=i32(rows), n_free=i32(1),
               status=i32(1))
    parents = None
    if c["words"]:
        out["tree_mask"] = i32(rows, c["words"])
        parents = torch.cat([_parents(new, host), torch.full((5,), -1, dtype=torch.int32)]).cuda()
    return dict(case=c, cached=_ints(cached), new=_ints(new), table=table.cuda(), free=free.cuda().contiguous(),
                n_free=_ints([free.numel()]), n_pages=n_pages, parents=parents, rows=rows, out=out)


def _prepare_append(c, host, gen):
    rows, page, hd = c["rows"], c["page"], c["d_head"]
    n_pages = _pages(rows, page) + 3
    k, v = _cache(n_pages, page, c["kv_heads"], hd, c["dtype"], c["layout"], gen)
    slot = torch.randperm(n_pages * page, generator=host)[:rows].to(torch.int32)
    if rows > 4:
        slot[-2:] = -1                                        # a padded batch
    pos = torch.randint(0, c["rope_len"], (rows,), generator=host).to(torch.int32)
    pos[slot < 0] = -1
    angle = torch.arange(c["rope_len"], dtype=torch.float64)[:, None] * (10000.0 ** (-torch.arange(hd // 2, dtype=torch.float64) / (hd // 2)))[None]
    qkv = torch.randn((rows, (c["heads"] + 2 * c["kv_heads"]) * hd), generator=gen, device="cuda", dtype=torch.float32)
    return dict(case=c, qkv=qkv, pos=pos.cuda(), slot=slot.cuda(), cos=angle.cos().float().cuda(), sin=angle.sin().float().cuda(), k=k, v=v,
                q=torch.zeros((rows, c["heads"], hd), dtype=DTYPES[c["dtype"]], device="cuda"),
                err=torch.zeros(1, dtype=torch.int32, device="cuda"))


def _prepare_attend(c, host, gen):
    cached, new, page = _cached(c), _new(c), c["page"]
    batch, rows = c["batch"], sum(new) + (3 if c["batch"] > 1 else 0)
    kv = [x + y for x, y in zip(cached, new)]
    used = sum(_pages(x, page) for x in kv)
    n_pages, max_pages = used + 2, max(_pages(x, page) for x in kv)
    order = torch.randperm(n_pages, generator=host).to(torch.int32)
    table = torch.full((batch, max_pages), -1, dtype=torch.int32)
    table[torch.arange(max_pages).unsqueeze(0) < torch.tensor([_pages(x, page) for x in kv]).unsqueeze(1)] = order[:used]
    k, v = _cache(n_pages, page, c["kv_heads"], c["d_head"], c["dtype"], c["layout"], gen)
    q = 1.5 * torch.randn((rows, c["heads"], c["d_head"]), generator=gen, device="cuda", dtype=torch.float32)
    row_start = [0]
    for n in new:
        row_start.append(row_start[-1] + n)
    words = _pages(max(new), 32)
    start, request = _ints(row_start), torch.repeat_interleave(torch.arange(batch), torch.tensor(new)).cuda()
    local = torch.arange(sum(new), device="cuda") - start.long()[request]
    mask = torch.zeros((rows, words), dtype=torch.int32, device="cuda")
    mask[: sum(new)] = _pack(_reach(_parents(new, host).cuda(), start, request, local, 32 * words)[request, local])
    return dict(case=c, q=q.to(DTYPES[c["dtype"]]), k=k, v=v, table=table.cuda(), kv_len=_ints(kv), row_start=start, mask=mask, n_max=max(new),
                scale=1.0 / math.sqrt(c["d_head"]), out=torch.zeros((rows, c["heads"], c["d_head"]), dtype=DTYPES[c["dtype"]], device="cuda"),
                scratch=torch.empty(64 << 20, dtype=torch.uint8, device="cuda"), err=torch.zeros(1, dtype=torch.int32, device="cuda"))


def _prepare_rules(c, host, gen):
    batch, per, V, rows = c["batch"], c["per"], c["vocab"], c["batch"] * c["per"]
    hist_len = _spread(c["hist"] // 3, c["hist"], batch, 5)
    # tokens of a text: few of them make up most of it
    history = (V * torch.rand((batch, max(1, c["hist"])), generator=gen, device="cuda") ** 4).long().clamp(max=V - 1).to(torch.int32)
    logits = 3.0 * torch.randn((rows, V), generator=gen, device="cuda", dtype=torch.float32)
    s = dict(case=c, logits=logits.to(DTYPES[c["dtype"]]), request=_ints([r // per for r in range(rows)]), history=history,
             history_len=_ints(hist_len), prompt_len=_ints([n // 2 for n in hist_len]),
             repetition=1.0 + 0.5 * torch.rand(batch, generator=gen, device="cuda"), presence=torch.rand(batch, generator=gen, device="cuda"),
             frequency=0.2 * torch.rand(batch, generator=gen, device="cuda"), bias_token=None, bias_value=None, bias_len=None, allowed=None,
             drafts=None, row_start=None, tree_mask=None, out=torch.empty((rows, V), dtype=DTYPES[c["dtype"]], device="cuda"),
             token=torch.empty(rows, dtype=torch.int32, device="cuda"))
    if c["bias"]:
        s["bias_token"] = torch.stack([torch.randperm(V, generator=gen, device="cuda")[: c["bias"]] for _ in range(batch)]).to(torch.int32)
        s["bias_value"] = 4.0 * torch.randn((batch, c["bias"]), generator=gen, device="cuda")
        s["bias_len"] = _ints(_spread(c["bias"] // 2, c["bias"], batch, 3))
    if c["mask"]:
        s["allowed"] = torch.randint(-2 ** 31, 2 ** 31, (rows, _pages(V, 32)), generator=gen, device="cuda").to(torch.int32)
    if per > 1:
        new = [per] * batch
        s["drafts"] = (V * torch.rand(rows, generator=gen, device="cuda") ** 4).long().clamp(max=V - 1).to(torch.int32)
        s["row_start"] = _ints([per * b for b in range(batch + 1)])
        local = torch.arange(rows, device="cuda") % per
        reach = _reach(_parents(new, host).cuda(), s["row_start"], s["request"].long(), local, 32)
        s["tree_mask"] = _pack(reach[s["request"].long(), local])
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------
def run(state):
    op = state["case"]["op"]
    if own:
        return {"plan": _own_plan, "append": _own_append, "attend": _own_attend, "rules": _own_rules}[op](state)
    return {"plan": _plain_plan, "append": _plain_append, "attend": _plain_attend, "rules": _plain_rules}[op](state)


def _own_plan(s):
    from paper_2509_00031_b200 import binding as zq
    if "status" not in s:                                     # the call or-s into this word: a program zeroes it once
        s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = zq.zoqat_op_cache_plan(s["cached"], s["new"], s["case"]["page"], s["n_pages"], s["free"], s["n_free"], s["table"], s["rows"],
                                 parents=s["parents"], mask_words=s["case"]["words"],
                                 out=dict(s["out"], status=s["status"]))
    return dict(out, table=s["table"])


def _own_append(s):
    from paper_2509_00031_b200 import binding as zq
    q, _ = zq.zoqat_op_cache_append(s["qkv"], s["pos"], s["slot"], s["k"], s["v"], s["case"]["heads"], cos=s["cos"], sin=s["sin"], q_out=s["q"],
                                    err=s["err"])
    return q, s["k"], s["v"]


def _own_attend(s):
    from paper_2509_00031_b200 import binding as zq
    out, _ = zq.zoqat_op_tree_attention(s["q"], s["k"], s["v"], s["table"], s["kv_len"], s["row_start"], tree_mask=s["mask"], scale=s["scale"],
                                        out=s["out"], scratch=s["scratch"], err=s["err"])
    return out


def _own_rules(s):
    from paper_2509_00031_b200 import binding as zq
    rules = zq.LogitRules(row_request=s["request"], history=s["history"], history_len=s["history_len"], prompt_len=s["prompt_len"],
                          repetition=s["repetition"], presence=s["presence"], frequency=s["frequency"], bias_token=s["bias_token"],
                          bias_value=s["bias_value"], bias_len=s["bias_len"], allowed=s["allowed"], draft_token=s["drafts"],
                          row_start=s["row_start"], tree_mask=s["tree_mask"])
    return zq.zoqat_op_logit_rules(s["logits"], rules, out=s["out"], token=s["token"])


def _plain_plan(s):
    page, rows, table = s["case"]["page"], s["rows"], s["table"]
    cached, new, free = s["cached"].long(), s["new"].long(), s["free"]
    batch, max_pages = table.shape
    kv = cached + new
    held = (cached + page - 1) // page
    need = (kv + page - 1) // page - held
    first = torch.cumsum(need, 0) - need
    k = torch.arange(max_pages, device="cuda")[None]
    fresh = (k >= held[:, None]) & (k < (held + need)[:, None])
    top = s["n_free"].long() - 1
    table.copy_(torch.where(fresh, free[(top - first[:, None] - k + held[:, None]).clamp(0, free.numel() - 1)], table))
    row_start = torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), torch.cumsum(new, 0)])
    r = torch.arange(rows, device="cuda")
    live = r < row_start[-1]
    request = torch.searchsorted(row_start[1:], r, right=True).clamp(max=batch - 1)
    local = torch.where(live, r - row_start[request], 0)
    at = (cached[request] + local).clamp(max=max_pages * page - 1)
    slot = table[request, at // page].long() * page + at % page
    pos = at
    out = dict(kv_len=kv, row_start=row_start, row_request=torch.where(live, request, -1), slot=torch.where(live, slot, -1),
               n_free=s["n_free"] - need.sum(), status=torch.zeros(1, device="cuda"))
    if s["parents"] is not None:
        n_max = 32 * s["case"]["words"]
        # rows behind the last draft go to a request of their own
        own_request = torch.where(live, request, batch)
        starts = torch.cat([row_start, row_start[-1:]])
        seen = _reach(s["parents"], starts, own_request, torch.where(live, local, r % n_max), n_max)[own_request, local]
        pos = cached[request] + seen.sum(-1).long() - 1
        out["tree_mask"] = torch.where(live[:, None], _pack(seen), 0)
    out["row_pos"] = torch.where(live, pos, -1)
    out = {n: t.to(torch.int32) for n, t in out.items()}
    return dict(out, table=table)


def _plain_append(s):
    c = s["case"]
    hd, H, kv = c["d_head"], c["heads"], c["kv_heads"]
    x = s["qkv"].view(-1, H + 2 * kv, hd)
    live = s["slot"] >= 0
    cos, sin = s["cos"][s["pos"].long().clamp(min=0)][:, None], s["sin"][s["pos"].long().clamp(min=0)][:, None]
    a, b = x[:, : H + kv, : hd // 2], x[:, : H + kv, hd // 2:]
    turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    s["q"].copy_(torch.where(live[:, None, None], turned[:, :H].to(s["q"].dtype), s["q"]))
    page, off = s["slot"].long() // c["page"], s["slot"].long() % c["page"]
    # a padded row repeats what row 0 writes
    at = torch.where(live, torch.arange(live.numel(), device="cuda"), 0)
    s["k"][page[at], off[at]] = turned[at, H:].to(s["k"].dtype)
    s["v"][page[at], off[at]] = x[at, H + kv:].to(s["v"].dtype)
    return s["q"], s["k"], s["v"]


def _bits(words, n):
    """[..., n] truth values of the first n bits of 32-bit words."""
    j = torch.arange(n, device=words.device)
    return (words[..., j // 32] >> (j % 32)) & 1 != 0


def _plain_attend(s):
    c, table, n_max = s["case"], s["table"], s["n_max"]
    B, H, kv, hd = c["batch"], c["heads"], c["kv_heads"], c["d_head"]
    g, rows, L = H // kv, s["q"].shape[0], table.shape[1] * c["page"]
    start, kv_len = s["row_start"].long(), s["kv_len"].long()
    new = start[1:] - start[:-1]
    held = table.long().clamp(min=0)
    t = torch.arange(L, device="cuda")
    inside = (t[None] < kv_len[:, None])[:, :, None, None]
    k = torch.where(inside, s["k"][held].reshape(B, L, kv, hd).float(), 0.0)
    v = torch.where(inside, s["v"][held].reshape(B, L, kv, hd).float(), 0.0)
    i = torch.arange(n_max, device="cuda")
    row = (start[:-1, None] + i[None]).clamp(max=rows - 1)                               # [B, n_max]
    q = s["q"][row].float().view(B, n_max, kv, g, hd).permute(0, 2, 1, 3, 4).reshape(B, kv, n_max * g, hd)
    score = (q @ k.permute(0, 2, 3, 1)) * s["scale"]                                     # [B, kv, n_max * g, L]
    draft = t[None, :] - (kv_len - new)[:, None]                                         # position among the drafts
    seen = _bits(s["mask"][row], n_max)                                                  # [B, n_max, n_max]
    seen = torch.gather(seen, 2, draft.clamp(0, n_max - 1)[:, None].expand(B, n_max, L))
    seen = (draft < 0)[:, None] | (seen & (t[None] < kv_len[:, None])[:, None])
    seen = seen[:, None, :, None].expand(B, 1, n_max, g, L).reshape(B, 1, n_max * g, L)
    score = score.masked_fill(~seen, -math.inf)
    top = score.max(-1, keepdim=True).values
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.where(total > 0, (p @ v.permute(0, 2, 1, 3)) / total, 0.0)                 # [B, kv, n_max * g, hd]
    o = o.view(B, kv, n_max, g, hd).permute(0, 2, 1, 3, 4).reshape(B, n_max, H, hd).to(s["out"].dtype)
    r = torch.arange(rows, device="cuda")
    request = torch.searchsorted(start[1:], r, right=True).clamp(max=B - 1)
    mine = o[request, (r - start[request]).clamp(0, n_max - 1)]
    s["out"].copy_(torch.where((r < start[-1])[:, None, None], mine, s["out"]))
    return s["out"]


def _counts(s, kind):
    """How often each token stands in a row's prompt ("prompt") or among its generated and drafted tokens ("made")."""
    c = s["case"]
    i = torch.arange(s["history"].shape[1], device="cuda")[None]
    inside = i < s["history_len"][:, None]
    prompt = i < s["prompt_len"][:, None]
    n = torch.zeros((c["batch"], c["vocab"]), dtype=torch.float32, device="cuda")
    n.scatter_add_(1, s["history"].long(), (inside & (prompt if kind == "prompt" else ~prompt)).float())
    n = n[s["request"].long()]
    if kind == "made" and s["drafts"] is not None:
        per = c["per"]
        seen = _bits(s["tree_mask"], per).float()
        n = n.scatter_add(1, s["drafts"].long().view(-1, per)[s["request"].long()], seen)
    return n


def _plain_rules(s):
    c = s["case"]
    b = s["request"].long()
    x = s["logits"].float()
    made = _counts(s, "made")
    rep = s["repetition"][b][:, None]
    x = torch.where((made > 0) | (_counts(s, "prompt") > 0), torch.where(x > 0, x / rep, x * rep), x)
    x = x - s["frequency"][b][:, None] * made
    x = torch.where(made > 0, x - s["presence"][b][:, None], x)
    if s["bias_token"] is not None:
        add = torch.where(torch.arange(c["bias"], device="cuda")[None] < s["bias_len"][:, None], s["bias_value"], 0.0)
        x = x + torch.zeros((c["batch"], c["vocab"]), device="cuda").scatter_add_(1, s["bias_token"].long(), add)[b]
    if s["allowed"] is not None:
        x = x.masked_fill(~_bits(s["allowed"], c["vocab"]), -math.inf)
    out = x.to(s["out"].dtype)
    best = out.float().max(1, keepdim=True).values
    token = torch.where(out.float() == best, torch.arange(c["vocab"], device="cuda"), c["vocab"]).min(1).values
    return out, torch.where(best[:, 0] > -math.inf, token, -1).to(torch.int32)


# ---- work and exact values ------------------------------------------------------------------------------------------
def work(case):
    c = case
    if c["op"] == "plan":
        cached, new = _cached(c), _new(c)
        fresh = sum(_pages(x + y, c["page"]) - _pages(x, c["page"]) for x, y in zip(cached, new))
        rows = sum(new)
        # lengths read, tables' new entries read and written, four words a row (with its parent), the masks
        nbytes = c["batch"] * 4 * 4 + fresh * 8 + rows * (12 + (4 + 4 * c["words"] if c["words"] else 0))
        return {"bytes": nbytes, "flops": 10 * rows}
    if c["op"] == "append":
        live = c["rows"] - (2 if c["rows"] > 4 else 0)
        wide = (c["heads"] + 2 * c["kv_heads"]) * c["d_head"]
        return {"bytes": live * (wide * (4 + BYTES[c["dtype"]]) + 8 + 4 * c["d_head"]), "flops": live * 3 * (c["heads"] + c["kv_heads"]) * c["d_head"]}
    if c["op"] == "attend":
        cached, new = _cached(c), _new(c)
        e, hd = BYTES[c["dtype"]], c["d_head"]
        keys = sum(x + y for x, y in zip(cached, new))
        nbytes = keys * c["kv_heads"] * hd * 2 * e + 2 * sum(new) * c["heads"] * hd * e + 4 * keys // c["page"] + 8 * c["batch"]
        pairs = sum(n * (x + n) for x, n in zip(cached, new))
        return {"bytes": nbytes, "flops": 4 * pairs * c["heads"] * hd}
    rows = c["batch"] * c["per"]
    hist = sum(_spread(c["hist"] // 3, c["hist"], c["batch"], 5))
    nbytes = 2 * rows * c["vocab"] * BYTES[c["dtype"]] + 4 * hist + (rows * _pages(c["vocab"], 32) * 4 if c["mask"] else 0) + c["batch"] * c["bias"] * 8
    return {"bytes": nbytes, "flops": 6 * rows * c["vocab"]}


def exact(case, seed):
    if case["op"] == "plan":
        return None
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "rules": _exact_rules}[case["op"]](case, s)


def _exact_append(c, s):
    H, kv, hd = c["heads"], c["kv_heads"], c["d_head"]
    half = hd // 2
    x = s["qkv"].double().reshape(-1, H + 2 * kv, 2, half)
    rows = [r for r, n in enumerate(s["slot"].tolist()) if n >= 0]
    where = s["slot"].long()[rows]
    turn = torch.complex(s["cos"].double(), s["sin"].double())[s["pos"].long()[rows]]
    z = torch.complex(x[rows, :, 0], x[rows, :, 1])
    z[:, : H + kv] = z[:, : H + kv] * turn[:, None, :]
    y = torch.cat([z.real, z.imag], -1)
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    q[rows] = y[:, :H]
    k[where // c["page"], where % c["page"]] = y[:, H: H + kv]
    v[where // c["page"], where % c["page"]] = y[:, H + kv:]
    return q, k, v


def _exact_attend(c, s):
    H, kv, hd = c["heads"], c["kv_heads"], c["d_head"]
    g, page = H // kv, c["page"]
    out = s["out"].double()
    start, lens, mask = s["row_start"].tolist(), s["kv_len"].tolist(), s["mask"].cpu().numpy().astype("uint32")
    if sum((start[b + 1] - start[b]) * lens[b] for b in range(c["batch"])) * H * hd > 3e12:
        return None
    for b in range(c["batch"]):
        n, L = start[b + 1] - start[b], lens[b]
        if n == 0:
            continue
        pages = s["table"][b, : _pages(L, page)].long()
        visible = torch.zeros((n, L), dtype=torch.bool)
        visible[:, : L - n] = True
        for i in range(n):
            for j in range(n):
                visible[i, L - n + j] = bool((int(mask[start[b] + i, j // 32]) >> (j % 32)) & 1)
        visible = visible.cuda()
        for h in range(kv):
            keys = s["k"][pages, :, h].reshape(-1, hd)[:L].double()
            vals = s["v"][pages, :, h].reshape(-1, hd)[:L].double()
            q = s["q"][start[b]: start[b + 1], h * g: (h + 1) * g].double()
            w = torch.einsum("ngd,td->ngt", q, keys) / math.sqrt(hd)
            w = torch.softmax(w.masked_fill(~visible[:, None, :], -math.inf), -1)
            w = torch.nan_to_num(w, nan=0.0)
            out[start[b]: start[b + 1], h * g: (h + 1) * g] = torch.einsum("ngt,td->ngd", w, vals)
    return out


def _exact_rules(c, s):
    V, per = c["vocab"], c["per"]
    x = s["logits"].double()
    hist, lens, prompts = s["history"].long(), s["history_len"].tolist(), s["prompt_len"].tolist()
    for r in range(c["batch"] * per):
        b = r // per
        made = torch.bincount(hist[b, prompts[b]: lens[b]], minlength=V).double()
        asked = torch.bincount(hist[b, : prompts[b]], minlength=V)
        if s["drafts"] is not None:
            m = int(s["tree_mask"][r, 0])
            for j in range(per):
                if (m >> j) & 1:
                    made[int(s["drafts"][b * per + j])] += 1
        rep = float(s["repetition"][b])
        old = (made > 0) | (asked > 0)
        row = x[r]
        row = torch.where(old & (row > 0), row / rep, torch.where(old, row * rep, row))
        row = row - float(s["frequency"][b]) * made - float(s["presence"][b]) * (made > 0)
        if s["bias_token"] is not None:
            n = int(s["bias_len"][b])
            row[s["bias_token"][b, :n].long()] += s["bias_value"][b, :n].double()
        if s["allowed"] is not None:
            words = s["allowed"][r].long() & 0xFFFFFFFF
            ok = ((words[:, None] >> torch.arange(32, device="cuda")) & 1).reshape(-1)[:V] != 0
            row = torch.where(ok, row, -math.inf)
        x[r] = row
    return x, None
