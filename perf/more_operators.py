"""The operators of decoding many continuations of one long prompt over a paged key/value cache, as cases to measure.

Four operators that a serving loop with beams (or many requests behind one system prompt) runs for every token:

  append   norms of the query and key heads and their rotation at (far) positions in one pass, keys and values into their slots
  attend   attention of a batch whose requests share a long prefix: the prefix is read once for all of a group
  select   the best continuations of every request's beams over the vocabulary, finished ones apart
  reorder  the states follow the beams that go on: block tables, pages given back and taken, token histories, and the slots of
           half-filled pages copied in every layer's cache

Where ``own`` is false ``run`` computes them with elementary torch operations in 32 bits (64 for angles of far positions and for the
order of scores); where it is true it calls the package's entry points.  ``exact`` gives the floating outputs from the definitions
in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


# ---- cases ------------------------------------------------------------------------------------------------------
def listed():
    return [
        # the new rows of one layer in a step of 8 beams: latency is what counts
        dict(name="append_beams_bf16", op="append", rows=8, heads=32, kv_heads=8, d_head=128, rot=128, interleaved=False, norm=True, scaled=1,
             pos_hi=4000, page=16, src="f32", dtype="bf16", layout="token"),
        # a chunk of a very long prompt: frequencies scaled for long contexts, half of each head turned, grouped heads
        dict(name="append_long_f16", op="append", rows=8191, heads=40, kv_heads=8, d_head=128, rot=64, interleaved=True, norm=True, scaled=8,
             pos_hi=1000000, page=64, src="bf16", dtype="f16", layout="head"),
        # a batch of single tokens, 64-wide heads without norms, the type of the package's own decode cache
        dict(name="append_batch_f32", op="append", rows=777, heads=32, kv_heads=32, d_head=64, rot=64, interleaved=False, norm=False, scaled=1,
             pos_hi=32000, page=32, src="f32", dtype="f32", layout="token"),
        # four beams of one request: the smallest call
        dict(name="attend_beams_b1", op="attend", groups=1, per_lo=4, per_hi=4, prefix_lo=2000, prefix_hi=2000, own_lo=33, own_hi=33, new_lo=1,
             new_hi=1, heads=32, kv_heads=32, d_head=128, page=16, dtype="bf16", layout="token"),
        # a batch of beam searches with ragged prompts, grouped heads
        dict(name="attend_beams_b8", op="attend", groups=8, per_lo=8, per_hi=8, prefix_lo=3000, prefix_hi=16000, own_lo=17, own_hi=300, new_lo=1,
             new_hi=1, heads=32, kv_heads=8, d_head=128, page=16, dtype="bf16", layout="token"),
        # a serving batch behind one long system prompt, requests of very different lengths: products count as much as bytes
        dict(name="attend_system_prompt", op="attend", groups=1, per_lo=128, per_hi=128, prefix_lo=16001, prefix_hi=16001, own_lo=1, own_hi=1500,
             new_lo=1, new_hi=1, heads=32, kv_heads=8, d_head=128, page=64, dtype="bf16", layout="head"),
        # 32-bit caches, several prompts, small trees of drafts
        dict(name="attend_f32_drafts", op="attend", groups=3, per_lo=2, per_hi=6, prefix_lo=500, prefix_hi=4000, own_lo=8, own_hi=200, new_lo=1,
             new_hi=3, heads=32, kv_heads=32, d_head=64, page=64, dtype="f32", layout="token"),
        # one request's four beams
        dict(name="select_b1", op="select", batch=1, beams=4, vocab=32000, eos=1, banned=0, dtype="f32"),
        # a batch of beam searches: the logits of 512 rows are read once
        dict(name="select_b64", op="select", batch=64, beams=8, vocab=50272, eos=1, banned=0, dtype="f32"),
        # 16-bit logits, few beams, two tokens that end a text, most of the vocabulary ruled out by a grammar
        dict(name="select_bf16_grammar", op="select", batch=96, beams=3, vocab=128256, eos=2, banned=90, dtype="bf16"),
        # the beams of a small batch change places, all layers of a model
        dict(name="reorder_b4", op="reorder", batch=4, beams=4, ctx_lo=300, ctx_hi=2000, tail=3, page=16, layers=24, kv_heads=8, d_head=128,
             dtype="bf16", layout="token"),
        # a large batch: what is copied in the caches counts
        dict(name="reorder_b64", op="reorder", batch=64, beams=8, ctx_lo=100, ctx_hi=2000, tail=2, page=32, layers=16, kv_heads=8, d_head=128,
             dtype="bf16", layout="head"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choice(["append", "attend", "attend", "select", "reorder"])
        if op == "append":
            kv, dh = rng.choice([1, 2, 8, 32]), rng.choice([64, 128])
            c = dict(op=op, rows=_log(rng, 1, 8191), heads=kv * rng.choice([1, 2, 5] if kv > 2 else [1, 4, 8]), kv_heads=kv, d_head=dh,
                     rot=rng.choice([dh, dh, dh // 2, dh // 4, 0]), interleaved=rng.random() < 0.5, norm=rng.random() < 0.7, scaled=rng.choice([1, 4, 32]),
                     pos_hi=_log(rng, 100, 1000000), page=rng.choice([16, 32, 64, 100, 128]), src=rng.choice(list(DTYPES)), dtype=rng.choice(list(DTYPES)),
                     layout=rng.choice(["token", "head"]))
            if c["rows"] * (c["heads"] + 2 * kv) * dh > 58_000_000:
                continue
        elif op == "attend":
            dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
            kv = rng.choice([1, 2, 4, 8, 32])
            g = rng.choice([1, 2, 4, 7, 8]) if kv < 32 else 1
            lo, own_lo, new_hi = rng.randrange(0, 3000), rng.randrange(1, 200), rng.choice([1, 1, 1, 2, 5])
            per_hi = _log(rng, 1, 128 if dtype != "f32" else 8)
            c = dict(op=op, groups=_log(rng, 1, 16), per_lo=rng.randrange(1, per_hi + 1), per_hi=per_hi, prefix_lo=lo,
                     prefix_hi=lo + _log(rng, 1, 24000 if dtype != "f32" else 4000), own_lo=own_lo + new_hi, own_hi=own_lo + new_hi + _log(rng, 1, 1500),
                     new_lo=rng.randrange(0, 2), new_hi=new_hi, heads=kv * g, kv_heads=kv, d_head=rng.choice([64, 128]), page=rng.choice([16, 32, 64, 128]),
                     dtype=dtype, layout=rng.choice(["token", "head"]))
            padded = c["groups"] * per_hi * (c["prefix_hi"] + c["own_hi"])
            if padded * kv * c["d_head"] > 1_900_000_000 or padded * c["heads"] * new_hi > 75_000_000:
                continue
        elif op == "select":
            c = dict(op=op, batch=_log(rng, 1, 128), beams=rng.choice([1, 2, 3, 4, 5, 8, 16]), vocab=_log(rng, 5000, 131072), eos=rng.choice([0, 1, 1, 2]),
                     banned=rng.choice([0, 0, 50, 99]), dtype=rng.choice(list(DTYPES)))
            if c["batch"] * c["beams"] * c["vocab"] > 36_900_000:
                continue
        else:
            lo = rng.randrange(1, 500)
            c = dict(op=op, batch=_log(rng, 1, 128), beams=rng.choice([1, 2, 3, 4, 6, 8, 16]), ctx_lo=lo, ctx_hi=lo + _log(rng, 1, 8000),
                     tail=rng.choice([1, 2, 4]), page=rng.choice([8, 16, 32, 48, 128]), layers=rng.choice([1, 4, 16, 24]), kv_heads=rng.choice([1, 2, 8, 32]),
                     d_head=rng.choice([64, 128]), dtype=rng.choice(list(DTYPES)), layout=rng.choice(["token", "head"]))
            pages = _reorder_pages(c)
            if pages * c["page"] * c["kv_heads"] * c["d_head"] * c["layers"] * 2 * BYTES[c["dtype"]] > 8_000_000_000:
                continue
            if c["batch"] * c["beams"] * c["page"] * c["kv_heads"] * c["d_head"] * c["layers"] * BYTES[c["dtype"]] > 540_000_000:
                continue
        return c


def _spread(lo, hi, n, step):
    """n whole numbers between lo and hi (both among them where n > 1), in a scattered order."""
    if n == 1:
        return [hi]
    while math.gcd(step, n) != 1:
        step += 1
    return [lo + (hi - lo) * ((i * step) % n) // (n - 1) for i in range(n)]


def _pages(n, page):
    return -(-n // page)


# ---- inputs -----------------------------------------------------------------------------------------------------
def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _cache(n_pages, page, kv_heads, d_head, dtype, layout, gen):
    shape = (n_pages, page, kv_heads, d_head) if layout == "token" else (n_pages, kv_heads, page, d_head)
    both = [torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(DTYPES[dtype]) for _ in range(2)]
    return tuple(both) if layout == "token" else tuple(t.transpose(1, 2) for t in both)


def prepare(case, seed):
    host = torch.Generator().manual_seed(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"append": _prepare_append, "attend": _prepare_attend, "select": _prepare_select, "reorder": _prepare_reorder}[case["op"]](case, host, gen)


def _frequencies(rot, scaled):
    """Angles per position of the pairs of a head, float64.  scaled > 1: for contexts that many times longer than those trained on (8192 of them):
    pairs that turn less than once in them are slowed down by the factor, those that turn 32 times are left, a ramp in between."""
    n = rot // 2
    freq = 10000.0 ** (-torch.arange(n, dtype=torch.float64) / max(1, n))
    if scaled > 1:
        turns = freq * 8192 / (2 * math.pi)
        keep = ((turns - 1.0) / 31.0).clamp(0.0, 1.0)
        freq = freq / scaled * (1.0 - keep) + freq * keep
    return freq


def _prepare_append(c, host, gen):
    rows, page, hd = c["rows"], c["page"], c["d_head"]
    n_pages = _pages(rows, page) + 3
    k, v = _cache(n_pages, page, c["kv_heads"], hd, c["dtype"], c["layout"], gen)
    slot = torch.randperm(n_pages * page, generator=host)[:rows].to(torch.int32)
    if rows > 4:
        slot[-2:] = -1                                        # a padded batch
    pos = torch.randint(0, c["pos_hi"], (rows,), generator=host).to(torch.int32)
    pos[slot < 0] = -1
    wide = (c["heads"] + 2 * c["kv_heads"]) * hd
    qkv = torch.randn((rows, wide), generator=gen, device="cuda", dtype=torch.float32)
    qkv *= 0.2 + 3.0 * torch.rand((rows, 1), generator=gen, device="cuda")
    gains = [1.0 + 0.3 * torch.randn(hd, generator=gen, device="cuda") for _ in range(2)] if c["norm"] else [None, None]
    return dict(case=c, qkv=qkv.to(DTYPES[c["src"]]), pos=pos.cuda(), slot=slot.cuda(), k=k, v=v, q_gain=gains[0], k_gain=gains[1], eps=1e-6,
                freq=_frequencies(c["rot"], c["scaled"]).cuda() if c["rot"] else None,
                magnitude=1.0 if c["scaled"] == 1 else 0.1 * math.log(c["scaled"]) + 1.0,
                q=torch.zeros((rows, c["heads"], hd), dtype=DTYPES[c["dtype"]], device="cuda"), err=torch.zeros(1, dtype=torch.int32, device="cuda"))


def _attend_shape(c):
    """(requests of each group, prefix of each group, own keys of each request, new rows of each request)"""
    per = _spread(c["per_lo"], c["per_hi"], c["groups"], 5)
    n = sum(per)
    own_keys = _spread(c["own_lo"], c["own_hi"], n, 7)
    return per, _spread(c["prefix_lo"], c["prefix_hi"], c["groups"], 3), own_keys, [min(x, y) for x, y in zip(_spread(c["new_lo"], c["new_hi"], n, 11), own_keys)]


def _prepare_attend(c, host, gen):
    per, prefix, own_keys, new = _attend_shape(c)
    page, batch = c["page"], sum(per)
    group = [g for g, n in enumerate(per) for _ in range(n)]
    kv = [prefix[g] + x for g, x in zip(group, own_keys)]
    held = [_pages(x, page) for x in kv]
    whole = [p // page for p in prefix]                       # pages of a group's prefix that its requests share
    n_pages = sum(whole) + sum(h - whole[g] for g, h in zip(group, held)) + 2
    order = torch.randperm(n_pages, generator=host).to(torch.int32)
    table = torch.full((batch, max(held)), -1, dtype=torch.int32)
    k, v = _cache(n_pages, page, c["kv_heads"], c["d_head"], c["dtype"], c["layout"], gen)
    at, b = 0, 0
    for g, n in enumerate(per):
        table[b: b + n, : whole[g]] = order[at: at + whole[g]]
        at += whole[g]
        for i in range(b, b + n):
            table[i, whole[g]: held[i]] = order[at: at + held[i] - whole[g]]
            at += held[i] - whole[g]
        rest = prefix[g] - whole[g] * page                    # the prefix's end lies in a page of each request's own, as a copy
        if rest:
            of = table[b: b + n, whole[g]].long().cuda()
            for t in (k, v):
                t[of, :rest] = t[of[0], :rest]
        b += n
    rows = sum(new) + (3 if batch > 1 else 0)
    row_start, group_start = [0], [0]
    for x in new:
        row_start.append(row_start[-1] + x)
    for x in per:
        group_start.append(group_start[-1] + x)
    q = 1.5 * torch.randn((rows, c["heads"], c["d_head"]), generator=gen, device="cuda", dtype=torch.float32)
    s = dict(case=c, q=q.to(DTYPES[c["dtype"]]), k=k, v=v, table=table.cuda(), kv_len=_ints(kv), row_start=_ints(row_start), group_start=_ints(group_start),
             prefix_len=_ints(prefix), request_group=_ints(group), mask=None, n_max=max(new), scale=1.0 / math.sqrt(c["d_head"]),
             out=torch.zeros((rows, c["heads"], c["d_head"]), dtype=DTYPES[c["dtype"]], device="cuda"), err=torch.zeros(1, dtype=torch.int32, device="cuda"))
    if max(new) > 1:                                          # drafts: each sees itself, and each of those before it with a chance of a half
        mask = [0] * rows
        for b in range(batch):
            for i in range(new[b]):
                mask[row_start[b] + i] = (1 << i) | (int(torch.randint(0, 1 << i, (1,), generator=host)) if i else 0)
        s["mask"] = _ints(mask)[:, None].contiguous()
    return s


def _prepare_select(c, host, gen):
    B, K, V = c["batch"], c["beams"], c["vocab"]
    logits = 3.0 * torch.randn((B * K, V), generator=gen, device="cuda", dtype=torch.float32)
    favoured = (V * torch.rand((B * K, 24), generator=gen, device="cuda") ** 3).long().clamp(max=V - 1)
    logits.scatter_reduce_(1, favoured, 3.0 + 12.0 * torch.rand((B * K, 24), generator=gen, device="cuda"), "amax")
    if c["banned"]:                                           # what a grammar rules out
        keep = torch.rand((B * K, V), generator=gen, device="cuda") * 100.0 >= c["banned"]
        logits.masked_fill_(~keep, -math.inf)
    scores = -40.0 * torch.rand((B, K), generator=gen, device="cuda")
    if B > 2:
        scores[0, 1:] = -math.inf                             # a request at its first token: one beam
    eos = [2, V - 1][: c["eos"]]
    if eos:                                                   # texts do end
        logits[:, eos] += 9.0
    return dict(case=c, logits=logits.to(DTYPES[c["dtype"]]), scores=scores, eos=_ints(eos) if eos else None)


def _reorder_len(c):
    return _spread(c["ctx_lo"], c["ctx_hi"], c["batch"], 7)


def _reorder_pages(c):
    held = [_pages(n, c["page"]) for n in _reorder_len(c)]
    return sum(max(0, h - c["tail"]) + c["beams"] * min(h, c["tail"]) for h in held) + c["batch"] * c["beams"] + 7


def _prepare_reorder(c, host, gen):
    B, K, page = c["batch"], c["beams"], c["page"]
    lens = _reorder_len(c)
    held = [_pages(n, page) for n in lens]
    M, n_pages = max(held) + 1, _reorder_pages(c)
    order = torch.randperm(n_pages, generator=host).to(torch.int32)
    table = torch.full((B, K, M), -1, dtype=torch.int32)
    at = 0
    for b, h in enumerate(held):                              # beams share all but their last pages
        same = max(0, h - c["tail"])
        table[b, :, :same] = order[at: at + same]
        at += same
        table[b, :, same:h] = order[at: at + K * (h - same)].view(K, h - same)
        at += K * (h - same)
    parent = (K * torch.rand((B, K), generator=host) ** 2).int().clamp(max=K - 1)        # good beams have more than one child
    if B > 3:
        parent[1, K - 1] = -1                                 # fewer candidates than beams
    hist = max(lens) + 1
    history = torch.randint(0, 50000, (B * K, hist), generator=gen, device="cuda").to(torch.int32)
    free = torch.full((n_pages,), -1, dtype=torch.int32)
    free[: n_pages - at] = order[at:]
    rows = B * K
    i32 = lambda *shape: torch.full(shape, -1, dtype=torch.int32, device="cuda")  # noqa: E731
    out = dict(block_table=i32(rows, M), kv_len=i32(rows), free_pages=i32(n_pages), n_free=i32(1), copy_from=i32(rows), copy_to=i32(rows), copy_len=i32(rows),
               history=i32(rows, hist), history_len=i32(rows))
    lens_row = torch.tensor(lens, dtype=torch.int32)[:, None].expand(B, K).reshape(-1)
    return dict(case=c, parent=parent.cuda(), token=torch.randint(0, 50000, (B, K), generator=host).to(torch.int32).cuda(), kv_len=lens_row.cuda(),
                table=table.view(rows, M).cuda(), shared=_ints([max(0, h - c["tail"]) * page // 2 for h in held]), free=free.cuda(),
                n_free=_ints([n_pages - at]), n_pages=n_pages, history=history, history_len=lens_row.cuda().clone(), out=out,
                caches=[_cache(n_pages, page, c["kv_heads"], c["d_head"], c["dtype"], c["layout"], gen) for _ in range(c["layers"])])


# ---- one pass -----------------------------------------------------------------------------------------------------
def run(state):
    op = state["case"]["op"]
    if own:
        return {"append": _own_append, "attend": _own_attend, "select": _own_select, "reorder": _own_reorder}[op](state)
    return {"append": _plain_append, "attend": _plain_attend, "select": _plain_select, "reorder": _plain_reorder}[op](state)


def _own_append(s):
    from paper_2509_00031_b200 import binding as zq
    q, _ = zq.zoqat_op_rotary_append(s["qkv"], s["pos"], s["slot"], s["k"], s["v"], s["case"]["heads"], freq=s["freq"], interleaved=s["case"]["interleaved"],
                                     magnitude=s["magnitude"], q_gain=s["q_gain"], k_gain=s["k_gain"], norm_eps=s["eps"], q_out=s["q"], err=s["err"])
    return q, s["k"], s["v"]


def _own_attend(s):
    from paper_2509_00031_b200 import binding as zq
    if "scratch" not in s:                                    # a program keeps it from call to call
        s["scratch"] = zq.prefix_attention_scratch(s["q"], s["k"])
    out, _ = zq.zoqat_op_prefix_attention(s["q"], s["k"], s["v"], s["table"], s["kv_len"], s["row_start"], s["group_start"], s["prefix_len"],
                                          s["request_group"], tree_mask=s["mask"], scale=s["scale"], out=s["out"], scratch=s["scratch"], err=s["err"])
    return out


def _own_select(s):
    from paper_2509_00031_b200 import binding as zq
    s["own_out"] = zq.zoqat_op_beam_select(s["logits"], s["scores"], eos=s["eos"], out=s.get("own_out"))
    return s["own_out"]


def _own_reorder(s):
    from paper_2509_00031_b200 import binding as zq
    if "layers" not in s:                                     # a program keeps these from call to call
        s["layers"] = zq.LayerCaches(s["caches"])
        s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        s["scratch"] = zq.beam_reorder_scratch(s["parent"])
    out = zq.zoqat_op_beam_reorder(s["parent"], s["kv_len"], s["table"], s["case"]["page"], s["n_pages"], s["free"], s["n_free"], shared_len=s["shared"],
                                   history=s["history"], history_len=s["history_len"], token=s["token"], out=dict(s["out"], status=s["status"]),
                                   scratch=s["scratch"])
    zq.zoqat_op_cache_copy(s["layers"], out["copy_from"], out["copy_to"], out["copy_len"], err=s["status"])
    return {n: out[n] for n in s["out"]}, s["caches"]


def _plain_append(s):
    c = s["case"]
    hd, H, kv, rot = c["d_head"], c["heads"], c["kv_heads"], c["rot"]
    x = s["qkv"].float().view(-1, H + 2 * kv, hd)
    live = s["slot"] >= 0
    y = x[:, : H + kv]
    if s["q_gain"] is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + s["eps"])
        y = torch.cat([y[:, :H] * s["q_gain"], y[:, H:] * s["k_gain"]], 1)
    if rot:
        angle = s["pos"].double().clamp(min=0)[:, None] * s["freq"][None]
        cos, sin = (angle.cos() * s["magnitude"]).float()[:, None], (angle.sin() * s["magnitude"]).float()[:, None]
        if c["interleaved"]:
            a, b = y[..., 0:rot:2], y[..., 1:rot:2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = y[..., : rot // 2], y[..., rot // 2: rot]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        y = torch.cat([turned, y[..., rot:]], -1)
    s["q"].copy_(torch.where(live[:, None, None], y[:, :H].to(s["q"].dtype), s["q"]))
    page, off = s["slot"].long() // c["page"], s["slot"].long() % c["page"]
    # a padded row repeats what row 0 writes
    at = torch.where(live, torch.arange(live.numel(), device="cuda"), 0)
    s["k"][page[at], off[at]] = y[at, H:].to(s["k"].dtype)
    s["v"][page[at], off[at]] = x[at, H + kv:].to(s["v"].dtype)
    return s["q"], s["k"], s["v"]


def _plain_attend(s):
    c, table, n_max = s["case"], s["table"], s["n_max"]
    kv, hd, H = c["kv_heads"], c["d_head"], c["heads"]
    B, g, rows, L = table.shape[0], H // kv, s["q"].shape[0], table.shape[1] * c["page"]
    start, kv_len = s["row_start"].long(), s["kv_len"].long()
    new = start[1:] - start[:-1]
    held = table.long().clamp(min=0)
    t = torch.arange(L, device="cuda")
    i = torch.arange(n_max, device="cuda")
    row = (start[:-1, None] + i[None]).clamp(max=rows - 1)                               # [B, n_max]
    draft = t[None, :] - (kv_len - new)[:, None]                                         # position among the new rows
    if s["mask"] is not None:
        seen = (s["mask"][:, 0].long()[row][:, :, None] >> torch.arange(32, device="cuda")) & 1 != 0
        seen = torch.gather(seen, 2, draft.clamp(0, 31)[:, None].expand(B, n_max, L)) & (draft < 32)[:, None]
    else:
        seen = draft[:, None, :] <= i[None, :, None]
    seen = (draft < 0)[:, None] | (seen & (t[None] < kv_len[:, None])[:, None])          # [B, n_max, L]
    o = torch.zeros((B, n_max, H, hd), device="cuda")
    step = max(1, min(kv, 400_000_000 // (B * L * hd)))                                  # key heads at once: as many as fit
    for h in range(0, kv, step):
        m = min(step, kv - h)
        inside = (t[None] < kv_len[:, None])[..., None, None]
        k = torch.where(inside, s["k"][:, :, h: h + m][held].reshape(B, L, m, hd).float(), 0.0)
        v = torch.where(inside, s["v"][:, :, h: h + m][held].reshape(B, L, m, hd).float(), 0.0)
        q = s["q"][row][:, :, h * g: (h + m) * g].float().view(B, n_max, m, g, hd).transpose(1, 2).reshape(B, m, n_max * g, hd)
        score = ((q @ k.permute(0, 2, 3, 1)) * s["scale"]).view(B, m, n_max, g, L).masked_fill(~seen[:, None, :, None], -math.inf)
        top = score.max(-1, keepdim=True).values
        p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
        total = p.sum(-1, keepdim=True)
        x = (p.view(B, m, n_max * g, L) @ v.transpose(1, 2)).view(B, m, n_max, g, hd)
        o[:, :, h * g: (h + m) * g] = torch.where(total > 0, x / total, 0.0).transpose(1, 2).reshape(B, n_max, m * g, hd)
    o = o.to(s["out"].dtype)
    r = torch.arange(rows, device="cuda")
    request = torch.searchsorted(start[1:], r, right=True).clamp(max=B - 1)
    mine = o[request, (r - start[request]).clamp(0, n_max - 1)]
    s["out"].copy_(torch.where((r < start[-1])[:, None, None], mine, s["out"]))
    return s["out"]


def _first(values, wanted, n, fill):
    """The first n wanted entries of each row of `values`, in order; `fill` behind them."""
    place = torch.cumsum(wanted, 1) - 1
    place = torch.where(wanted & (place < n), place, n)
    out = torch.full((values.shape[0], n + 1), fill, dtype=values.dtype, device=values.device)
    return out.scatter(1, place, torch.where(wanted, values, fill))[:, :n].contiguous()


def _plain_select(s):
    c = s["case"]
    B, K, V = c["batch"], c["beams"], c["vocab"]
    x = s["logits"].double().view(B, K, V)
    top = x.max(-1, keepdim=True).values.clamp(min=-1e30)
    norm = top + torch.log(torch.exp(x - top).sum(-1, keepdim=True))
    score = (s["scores"].double()[..., None] + (x - norm)).view(B, K * V)
    score = torch.where(score == score, score, -math.inf)
    score, place = torch.sort(score, dim=1, descending=True, stable=True)                 # equal ones: lowest beam, then lowest token
    n = min(K * (1 + c["eos"]), K * V)
    score, place = score[:, :n], place[:, :n]
    beam, token = (place // V).to(torch.int32), (place % V).to(torch.int32)
    some = score > -math.inf
    ends = torch.zeros_like(some)
    if s["eos"] is not None:
        ends = (token[..., None] == s["eos"]).any(-1)
    on, done = some & ~ends, some & ends & (torch.arange(n, device="cuda") < K)
    value = score.float()
    return dict(beam=_first(beam, on, K, -1), token=_first(token, on, K, -1), score=_first(value, on, K, -math.inf), done_beam=_first(beam, done, K, -1),
                done_token=_first(token, done, K, -1), done_score=_first(value, done, K, -math.inf))


def _plain_reorder(s):
    c, out = s["case"], s["out"]
    B, K, P = c["batch"], c["beams"], c["page"]
    M = s["table"].shape[1]
    old, lens, parent = s["table"].view(B, K, M).long(), s["kv_len"].view(B, K).long(), s["parent"].long()
    live, of = parent >= 0, parent.clamp(min=0)
    col = torch.arange(M, device="cuda")
    new_len = torch.where(live, lens.gather(1, of), 0)
    held, new_held = (lens + P - 1) // P, (new_len + P - 1) // P
    table = old.gather(1, of[..., None].expand(B, K, M))
    # the page that a beam writes to next: its first child keeps it, the others get a copy of what it holds
    last, part = new_len // P, new_len % P != 0
    page = table.gather(2, last.clamp(max=M - 1)[..., None])[..., 0]
    same = part[:, :, None] & part[:, None] & (page[:, :, None] == page[:, None]) & (last[:, :, None] == last[:, None])
    keep = part & ~torch.tril(same, -1).any(-1) & (last * P >= s["shared"][:, None])
    copy = part & ~keep
    # pages that nobody holds any more, in the order request, column, beam
    has = (col < held[..., None]) & (col * P >= s["shared"][:, None, None])
    still = (col < new_held[..., None]) & ~(copy[..., None] & (col == last[..., None]))
    gone = has.clone()
    for p in range(K):
        for j in range(K):
            gone[:, p] &= ~(still[:, j] & (table[:, j] == old[:, p]))
            if j < p:
                gone[:, p] &= ~(has[:, j] & (old[:, j] == old[:, p]))
    gone_by_col, old_by_col = gone.transpose(1, 2).reshape(B, M * K), old.transpose(1, 2).reshape(B, M * K)
    n_gone, n_need = gone_by_col.sum(1), copy.sum(1)
    inside = torch.minimum(n_gone, n_need)                     # a request's new pages are those it gives back, then free ones
    outside = n_need - inside
    rank = torch.cumsum(copy, 1) - 1
    mine = _first(old_by_col, gone_by_col, K, -1)
    take = s["n_free"].long() - 1 - (torch.cumsum(outside, 0) - outside)[:, None] - (rank - inside[:, None])
    fresh = torch.where(rank < inside[:, None], mine.gather(1, rank.clamp(min=0)), s["free"].long()[take.clamp(0, s["free"].numel() - 1)])
    table = torch.where(copy[..., None] & (col == last[..., None]), fresh[..., None], table)
    out["block_table"].copy_(torch.where((col < new_held[..., None]).view(B * K, M), table.view(B * K, M).int(), out["block_table"]))
    out["kv_len"].copy_(new_len.view(-1))
    left = s["n_free"].long() - outside.sum()
    given = old_by_col[gone_by_col & (torch.cumsum(gone_by_col, 1) > inside[:, None])].int()
    slot = torch.arange(s["free"].numel(), device="cuda")
    out["free_pages"].copy_(torch.where(slot < left, s["free"], out["free_pages"]))
    out["free_pages"][left + torch.arange(given.numel(), device="cuda")] = given
    out["n_free"].copy_(left + given.numel())
    out["copy_from"].copy_(torch.where(copy, page, -1).view(-1))
    out["copy_to"].copy_(torch.where(copy, fresh, -1).view(-1))
    out["copy_len"].copy_(torch.where(copy, new_len % P, 0).view(-1))
    # histories
    at = torch.arange(s["history"].shape[1], device="cuda")
    h_len = torch.where(live, s["history_len"].view(B, K).long().gather(1, of), 0).view(-1, 1)
    source = (of + K * torch.arange(B, device="cuda")[:, None]).view(-1)
    moved = torch.where(at < h_len, s["history"][source], out["history"])
    out["history"].copy_(torch.where(live.view(-1, 1) & (at == h_len), s["token"].view(-1, 1), moved))
    out["history_len"].copy_(torch.where(live.view(-1), h_len[:, 0] + 1, 0))
    # the copies, in every layer
    which = torch.nonzero(copy.view(-1))[:, 0]
    f, t, n = page.view(-1)[which], fresh.view(-1)[which], (new_len % P).view(-1)[which]
    mask = (torch.arange(P, device="cuda")[None] < n[:, None])[:, :, None, None]
    for k, v in s["caches"]:
        k[t] = torch.where(mask, k[f], k[t])
        v[t] = torch.where(mask, v[f], v[t])
    return dict(out), s["caches"]


# ---- work and exact values ------------------------------------------------------------------------------------------
def work(case):
    c = case
    if c["op"] == "append":
        live = c["rows"] - (2 if c["rows"] > 4 else 0)
        wide = (c["heads"] + 2 * c["kv_heads"]) * c["d_head"]
        return {"bytes": live * (wide * (BYTES[c["src"]] + BYTES[c["dtype"]]) + 8), "flops": live * 6 * (c["heads"] + c["kv_heads"]) * c["d_head"]}
    if c["op"] == "attend":
        per, prefix, own_keys, new = _attend_shape(c)
        e, hd = BYTES[c["dtype"]], c["d_head"]
        group = [g for g, n in enumerate(per) for _ in range(n)]
        keys = sum(prefix) + sum(own_keys)
        pairs = sum(n * (prefix[g] + x) for g, n, x in zip(group, new, own_keys))
        return {"bytes": keys * c["kv_heads"] * hd * 2 * e + 2 * sum(new) * c["heads"] * hd * e + 4 * keys // c["page"] + 12 * len(group),
                "flops": 4 * pairs * c["heads"] * hd}
    if c["op"] == "select":
        rows = c["batch"] * c["beams"]
        return {"bytes": rows * (c["vocab"] * BYTES[c["dtype"]] + 28), "flops": 4 * rows * c["vocab"]}
    lens, rows = _reorder_len(c), c["batch"] * c["beams"]
    tables = 8 * c["beams"] * sum(_pages(n, c["page"]) for n in lens)
    histories = 8 * c["beams"] * sum(lens)
    slots = c["beams"] * sum(n % c["page"] for n in lens) / 2          # about half the beams are copies
    slot = 2 * c["kv_heads"] * c["d_head"] * BYTES[c["dtype"]] * c["layers"]
    return {"bytes": int(tables + histories + 2 * slots * slot + 32 * rows), "flops": rows}


def exact(case, seed):
    if case["op"] == "reorder":
        return None                                           # nothing is computed
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "select": _exact_select}[case["op"]](case, s)


def _exact_append(c, s):
    H, kv, hd, rot = c["heads"], c["kv_heads"], c["d_head"], c["rot"]
    rows = torch.nonzero(s["slot"] >= 0)[:, 0]
    where = s["slot"].long()[rows]
    x = s["qkv"][rows].double().reshape(-1, H + 2 * kv, hd)
    if c["norm"]:
        size = x[:, : H + kv].pow(2).sum(-1, keepdim=True) / hd + s["eps"]
        x[:, : H + kv] *= size.rsqrt()
        x[:, :H] *= s["q_gain"].double()
        x[:, H: H + kv] *= s["k_gain"].double()
    if rot:
        turn = torch.polar(torch.full((rot // 2,), float(s["magnitude"]), dtype=torch.float64, device="cuda"), s["pos"][rows].double()[:, None] * s["freq"])[:, None]
        part = x[:, : H + kv, :rot]
        pairs = part.reshape(*part.shape[:2], rot // 2, 2) if c["interleaved"] else part.reshape(*part.shape[:2], 2, rot // 2).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        x[:, : H + kv, :rot] = (z if c["interleaved"] else z.transpose(-1, -2)).reshape(part.shape)
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    q[rows] = x[:, :H]
    k[where // c["page"], where % c["page"]] = x[:, H: H + kv]
    v[where // c["page"], where % c["page"]] = x[:, H + kv:]
    return q, k, v


def _exact_attend(c, s):
    H, kv, hd, page = c["heads"], c["kv_heads"], c["d_head"], c["page"]
    g, out = H // kv, s["out"].double()
    start, lens = s["row_start"].tolist(), s["kv_len"].tolist()
    masks = s["mask"][:, 0].tolist() if s["mask"] is not None else None
    if sum((start[b + 1] - start[b]) * lens[b] for b in range(len(lens))) * H * hd > 3e12 or len(lens) * kv > 20000:
        return None
    for b, L in enumerate(lens):
        n = start[b + 1] - start[b]
        if n == 0:
            continue
        pages = s["table"][b, : _pages(L, page)].long()
        hidden = torch.zeros((n, L), dtype=torch.bool)
        for i in range(n):
            for j in range(n):
                hidden[i, L - n + j] = j > i if masks is None else not (masks[start[b] + i] >> j) & 1
        hidden = hidden.cuda()
        keys = s["k"][pages].reshape(-1, kv, hd)[:L].double()
        vals = s["v"][pages].reshape(-1, kv, hd)[:L].double()
        q = s["q"][start[b]: start[b + 1]].double().view(n, kv, g, hd)
        w = torch.einsum("nhgd,thd->hgnt", q, keys) / math.sqrt(hd)
        w = torch.softmax(w.masked_fill(hidden, -math.inf), -1)
        out[start[b]: start[b + 1]] = torch.einsum("hgnt,thd->nhgd", w, vals).reshape(n, H, hd)
    return out


def _exact_select(c, s):
    B, K, V = c["batch"], c["beams"], c["vocab"]
    logp = torch.log_softmax(s["logits"].double(), -1).nan_to_num(nan=-math.inf, neginf=-math.inf)
    ends = s["eos"].tolist() if s["eos"] is not None else []
    n = min(V, K + len(ends))
    value, token = torch.topk(logp, n, 1)                      # scores alone: which of equal tokens comes first does not matter
    value = (value + s["scores"].double().view(-1, 1)).view(B, K * n).cpu()
    token = token.view(B, K * n).cpu()
    score, done = torch.full((B, K), -math.inf, dtype=torch.float64), torch.full((B, K), -math.inf, dtype=torch.float64)
    for b in range(B):
        on, over = 0, 0
        for rank, i in enumerate(torch.argsort(value[b], descending=True).tolist()):
            x = float(value[b, i])
            if x == -math.inf or on == K:
                break
            if int(token[b, i]) in ends:
                if rank < K:
                    done[b, over] = x
                    over += 1
            else:
                score[b, on] = x
                on += 1
    return dict(beam=None, token=None, score=score.cuda(), done_beam=None, done_token=None, done_score=done.cuda())
