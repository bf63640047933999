"""The operators of many continuations of one prompt on the GPU, against plain float64 (or whole-number) implementations."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def zq():
    from paper_2509_00031_b200 import binding
    binding.lib()
    return binding


def make_cache(n_pages, page, kv, dh, dtype, layout, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    shape = (n_pages, page, kv, dh) if layout == "token" else (n_pages, kv, page, dh)
    both = [torch.randn(shape, generator=gen, device="cuda").to(DTYPES[dtype]) for _ in range(2)]
    return both if layout == "token" else [t.transpose(1, 2) for t in both]


# ---- rotary append --------------------------------------------------------------------------------------------------
def append_reference(x, pos, heads, kv, dh, freq, inter, magnitude, qg, kg, eps):
    """float64 [rows, heads + 2 kv, dh], and the bound on the part of the error that fp32 arithmetic may make."""
    x = x.double().view(x.shape[0], heads + 2 * kv, dh).clone()
    for lo, hi, g in ((0, heads, qg), (heads, heads + kv, kg)):
        if g is not None:
            x[:, lo:hi] = x[:, lo:hi] / (x[:, lo:hi].pow(2).mean(-1, keepdim=True) + eps).sqrt() * g.double()
    size = x.abs()
    if freq is not None:
        r, n = 2 * freq.numel(), heads + kv
        t = pos.double()[:, None] * freq
        c, s = t.cos()[:, None] * magnitude, t.sin()[:, None] * magnitude
        i = torch.arange(r // 2, device=x.device)
        a, b = (2 * i, 2 * i + 1) if inter else (i, i + r // 2)
        va, vb = x[:, :n, a], x[:, :n, b]
        both = magnitude * (size[:, :n, a] + size[:, :n, b])
        x[:, :n, a], x[:, :n, b] = va * c - vb * s, vb * c + va * s
        size[:, :n, a], size[:, :n, b] = both, both
    # fp32: a mean square of dh terms is off by dh * 2^-24 of itself (half of that in its root), a dozen roundings of 2^-24 follow, and the sine's and
    # cosine's own errors (angles in turns rounded to fp32 and the functions: under 2^-21 together)
    return x, size * (dh * 2.0 ** -25 + 12 * 2.0 ** -24 + 2.0 ** -21)


@pytest.mark.parametrize("rows,heads,kv,dh,rot,inter,norm,src,dtype,layout,top", [
    (1, 4, 2, 128, 128, False, True, "f32", "bf16", "token", 100), (8, 32, 8, 128, 128, True, True, "bf16", "f16", "head", 5000),
    (33, 5, 5, 64, 32, False, True, "f16", "f32", "token", 1000000), (257, 8, 1, 64, 64, True, False, "f32", "f32", "head", 2 ** 31 - 1),
    (300, 3, 1, 128, 32, False, False, "bf16", "bf16", "token", 4096), (70, 24, 8, 128, 96, False, True, "f32", "f16", "head", 70000),
    (5, 160, 32, 128, 16, True, True, "f32", "bf16", "token", 128000), (1200, 2, 2, 64, 48, False, True, "bf16", "f32", "token", 9999),
    (900, 96, 96, 128, 128, False, True, "f32", "bf16", "head", 3000), (19, 7, 1, 128, 0, False, True, "f16", "f16", "token", 10)])
def test_append_is_the_formula(zq, rows, heads, kv, dh, rot, inter, norm, src, dtype, layout, top):
    gen = torch.Generator(device="cuda").manual_seed(rows + rot)
    page, n_pages = 16, rows // 16 + 3
    k, v = make_cache(n_pages, page, kv, dh, dtype, layout)
    k0, v0 = k.clone(), v.clone()
    wide = (heads + 2 * kv) * dh
    store = torch.randn((rows, wide + 24), generator=gen, device="cuda").to(DTYPES[src])      # rows stand apart
    qkv = store[:, :wide]
    pos = torch.randint(0, top, (rows,), generator=gen, device="cuda").int()
    pos[0] = top - 1
    slot = torch.randperm(n_pages * page, generator=gen, device="cuda")[:rows].int()
    if rows > 6:
        slot[3] = -1
        slot[5] = n_pages * page                                  # outside: skipped and reported
    if rows > 8 and rot:
        pos[7] = -5
    qg, kg = (1 + 0.5 * torch.randn((2, dh), generator=gen, device="cuda")) if norm else (None, None)
    freq, mag = zq.rotary_frequencies(rot, kind=zq.ROTARY_PARTS, factor=4.0, trained_len=4096) if rot else (None, 1.0)
    q_store = torch.full((rows, heads, dh), 7.0, dtype=DTYPES[dtype], device="cuda")
    q, err = zq.zoqat_op_rotary_append(qkv, pos, slot, k, v, heads, freq=freq, interleaved=inter, magnitude=mag, q_gain=qg, k_gain=kg, norm_eps=1e-5, q_out=q_store)
    want, extra = append_reference(qkv, pos, heads, kv, dh, freq, inter, mag, qg, kg, 1e-5)
    live = (slot >= 0) & (slot < n_pages * page)
    if rot:
        live &= pos >= 0
    assert int(err) == (40 if rows > 6 else 0)
    half = torch.finfo(DTYPES[dtype]).eps / 2
    tiny = torch.finfo(DTYPES[dtype]).tiny * half
    ok = lambda got, w, x: ((got.double() - w).abs() <= half * (w.abs() + x) + x + tiny).all()  # noqa: E731
    assert ok(q[live], want[live, :heads], extra[live, :heads])
    at = slot[live].long()
    assert ok(k[at // page, at % page], want[live, heads: heads + kv], extra[live, heads: heads + kv])
    assert torch.equal(v[at // page, at % page], qkv.reshape(rows, -1, dh)[live, heads + kv:].float().to(DTYPES[dtype]))
    assert (q[~live] == 7.0).all()
    untouched = torch.ones(n_pages * page, dtype=torch.bool, device="cuda")
    untouched[at] = False
    u = torch.nonzero(untouched)[:, 0]
    assert torch.equal(k[u // page, u % page], k0[u // page, u % page]) and torch.equal(v[u // page, u % page], v0[u // page, u % page])


def test_append_agrees_with_the_table_form(zq):
    """Plain half rotation without norms is what zoqat_op_cache_append does from a table."""
    rows, heads, kv, dh = 40, 4, 2, 128
    gen = torch.Generator(device="cuda").manual_seed(5)
    qkv = torch.randn((rows, (heads + 2 * kv) * dh), generator=gen, device="cuda")
    pos = torch.randint(0, 512, (rows,), generator=gen, device="cuda").int()
    slot = torch.randperm(64, generator=gen, device="cuda")[:rows].int()
    freq, mag = zq.rotary_frequencies(dh)
    assert mag == 1.0
    angle = torch.arange(512, device="cuda", dtype=torch.float64)[:, None] * freq
    a, b = make_cache(4, 16, kv, dh, "f32", "token"), make_cache(4, 16, kv, dh, "f32", "token")
    q1, _ = zq.zoqat_op_rotary_append(qkv, pos, slot, *a, heads, freq=freq)
    q2, _ = zq.zoqat_op_cache_append(qkv, pos, slot, *b, heads, cos=angle.cos().float(), sin=angle.sin().float())
    # both are within a few roundings of the same rotation of numbers below 6
    for x, y in ((q1, q2), (a[0], b[0])):
        assert (x - y).abs().max() <= 6 * 2 * (2.0 ** -21 + 4 * 2.0 ** -24)
    assert torch.equal(a[1], b[1])


def test_append_no_rows_and_zero_heads_of_zeros(zq):
    k, v = make_cache(2, 16, 1, 64, "bf16", "token")
    q, err = zq.zoqat_op_rotary_append(torch.zeros((0, 3 * 64), device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"),
                                       torch.zeros(0, dtype=torch.int32, device="cuda"), k, v, 1)
    assert q.shape == (0, 1, 64) and int(err) == 0
    one = torch.ones(64, device="cuda")
    zeros = torch.zeros((1, 3 * 64), device="cuda")
    q, err = zq.zoqat_op_rotary_append(zeros, None, torch.zeros(1, dtype=torch.int32, device="cuda"), k, v, 1, q_gain=one, k_gain=one, norm_eps=1e-6)
    assert (q == 0).all() and (k[0, 0] == 0).all() and int(err) == 0


# ---- beam select ----------------------------------------------------------------------------------------------------
def select_reference(logits, scores, eos):
    B, K = scores.shape
    V = logits.shape[1]
    x = logits.double().cpu().numpy().reshape(B, K, V).copy()
    x[np.isnan(x)] = -np.inf
    x = np.minimum(x, float(np.finfo(np.float32).max))
    out = dict(beam=[], token=[], score=[], done_beam=[], done_token=[], done_score=[])
    for b in range(B):
        cand = []
        for k in range(K):
            s = float(scores[b, k])
            top = x[b, k].max()
            if not s > -math.inf or top == -math.inf:
                continue
            lse = top + math.log(np.exp(x[b, k] - top).sum())
            order = np.argsort(-x[b, k], kind="stable")[: K + len(eos)]
            cand += [(-(s + (x[b, k, v] - lse)), k, i, int(v)) for i, v in enumerate(order) if x[b, k, v] > -math.inf]
        cand.sort()
        on = [c for c in cand[: K * (1 + len(eos))] if c[3] not in eos][:K]
        done = [c for c in cand[:K] if c[3] in eos]
        for name, part in (("", on), ("done_", done)):
            part = part + [(math.inf, -1, 0, -1)] * (K - len(part))
            out[name + "beam"].append([c[1] for c in part])
            out[name + "token"].append([c[3] for c in part])
            out[name + "score"].append([-c[0] for c in part])
    return out


def check_select(zq, logits, scores, eos=(), out=None):
    e = torch.tensor(list(eos), dtype=torch.int32, device="cuda") if eos else None
    got = zq.zoqat_op_beam_select(logits, scores, eos=e, out=out)
    want = select_reference(logits, scores, list(eos))
    for n in ("beam", "token", "done_beam", "done_token"):
        assert got[n].tolist() == want[n], n
    for n in ("score", "done_score"):
        w = torch.tensor(want[n], dtype=torch.float64)
        g = got[n].double().cpu()
        f = torch.isfinite(w)
        assert torch.equal(torch.isfinite(g), f) and (g[~f] == w[~f]).all()
        # one rounding to fp32; the sum of exponentials is off by 2^-22 (each ex2) + 2^-23 (its argument near the maximum) + additions, in all under 2^-20
        assert ((g - w)[f].abs() <= 2.0 ** -24 * w[f].abs() + 2.0 ** -20).all()
    return got


@pytest.mark.parametrize("B,K,V,eos,dtype", [
    (1, 1, 5, (), "f32"), (1, 4, 32000, (2,), "f32"), (2, 3, 1001, (0, 1000), "bf16"), (3, 5, 4999, (7,), "f16"), (1, 8, 131072, (), "f32"),
    (5, 2, 50272, (1, 2, 3), "f32"), (2, 16, 20011, (5,), "bf16"), (1, 32, 9000, (1, 2, 3, 4, 5, 6, 7), "f32"), (70, 4, 3001, (9,), "f32"), (2, 9, 70, (3,), "f16"),
    (1, 1, 200000, (2,), "bf16"), (3, 7, 12, (0, 5), "f32"), (1, 32, 33, (), "f32"), (300, 1, 4100, (0,), "f32"), (1, 2, 8192, (4,), "f32"), (1, 2, 8193, (4,), "bf16")])
def test_select_is_the_definition(zq, B, K, V, eos, dtype):
    gen = torch.Generator(device="cuda").manual_seed(V + K)
    logits = (3 * torch.randn((B * K, V), generator=gen, device="cuda")).to(DTYPES[dtype])
    scores = -20 * torch.rand((B, K), generator=gen, device="cuda")
    if eos:
        logits[::2, list(eos)] += 7
    if B > 1 and K > 1:
        scores[0, 1:] = -math.inf
        scores[-1, 0] = math.nan
    out = check_select(zq, logits, scores, eos)
    check_select(zq, torch.flip(logits, (1,)).contiguous(), scores, eos, out=out)


def test_select_rows_apart_and_unaligned(zq):
    gen = torch.Generator(device="cuda").manual_seed(1)
    for dtype, ld, off in (("f32", 5003, 1), ("bf16", 5008, 8), ("f16", 5001, 3)):
        store = torch.randn((6, ld + 16), generator=gen, device="cuda").to(DTYPES[dtype])
        check_select(zq, store[:, off: off + 4990], torch.zeros((2, 3), device="cuda"), (17,))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V,ld,off,B,K", [(1, 1, 0, 3, 2), (2, 9, 5, 2, 3), (7, 7, 0, 9, 1), (9, 11, 1, 5, 2), (255, 259, 2, 3, 4), (4095, 4097, 3, 2, 8), (20001, 20003, 7, 1, 3), (50257, 50257, 0, 4, 5),
                                          (100003, 100003, 1, 1, 16), (9000, 9001, 1, 200, 2)])
def test_select_rows_that_begin_anywhere(zq, dtype, V, ld, off, B, K):
    """What stands around a row (large numbers, infinities, NaN) is not the row's."""
    gen = torch.Generator(device="cuda").manual_seed(V)
    store = torch.empty(B * K * ld + off + 16, device="cuda", dtype=DTYPES[dtype])
    store[0::3], store[1::3], store[2::3] = 3e4, float("inf"), float("nan")
    logits = store[off: off + B * K * ld].view(B * K, ld)[:, :V]
    logits.copy_(torch.randn((B * K, V), generator=gen, device="cuda"))
    logits[0, 0], logits[B * K - 1, V - 1] = 9.0, 9.0              # the best at the ends
    check_select(zq, logits, torch.randn((B, K), generator=gen, device="cuda"), (V - 1,))


def test_select_hard_rows(zq):
    """Equal, rising, falling, masked and non-finite logits; large ones; rows whose mask leaves nothing."""
    V = 40000
    low = float(np.finfo(np.float32).min)
    ramp = torch.arange(V, device="cuda", dtype=torch.float32)
    rows = {
        "equal": torch.zeros(V, device="cuda"), "rising": ramp / 4096, "falling": -ramp / 4096, "rising steeply": ramp, "nothing": torch.full((V,), -math.inf, device="cuda"),
        "lowest": torch.full((V,), low, device="cuda"), "one of the lowest": torch.full((V,), low, device="cuda"), "one": torch.full((V,), -math.inf, device="cuda"),
        "nan": torch.randn(V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)), "inf": ramp / 8192, "two values": (ramp % 2) * 3, "large": ramp * 1e33,
        "late": -ramp, "zeros of both signs": torch.where(ramp % 3 == 1, -0.0, 0.0), "few zeros": torch.where(ramp % 1000 == 7, (ramp % 2000 == 7) * -0.0, -1.0), "blocks": torch.where((ramp / 32).long() % 8 == 3, ramp / 1000, -math.inf)}
    rows["one of the lowest"][777] = 1.5
    rows["one"][V - 1] = -3.0
    rows["nan"][::5] = math.nan
    rows["inf"][[100, 30000]] = math.inf
    rows["late"][V - 40:] = 100 + ramp[:40]
    for name, x in rows.items():
        for K in (1, 3, 8):
            logits = x.repeat(2 * K, 1)
            scores = -torch.arange(2 * K, device="cuda", dtype=torch.float32).view(2, K) * 0.37
            check_select(zq, logits, scores, (1,))
            got = check_select(zq, logits, scores)
            if name == "equal":
                assert got["token"][0].tolist() == list(range(K))[: K] or K > 1
            if name == "nothing":
                assert (got["beam"] == -1).all() and (got["score"] == -math.inf).all()


def test_select_ties_between_beams_and_repeats(zq):
    """Equal scores: the lower beam, then the lower token; the same call gives the same bits."""
    x = torch.randn(20000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    x[[5, 50, 19999]] = 9.0
    logits = x.repeat(4, 1)
    got = check_select(zq, logits, torch.zeros((1, 4), device="cuda"))
    assert got["beam"][0].tolist() == [0, 0, 0, 1] and got["token"][0].tolist() == [5, 50, 19999, 5]
    first = {n: t.clone() for n, t in got.items()}
    for _ in range(5):
        again = zq.zoqat_op_beam_select(logits, torch.zeros((1, 4), device="cuda"))
        assert all(torch.equal(first[n], again[n]) for n in first)


# ---- reorder --------------------------------------------------------------------------------------------------------
def reorder_reference(parent, kv_len, table, P, free, n_free, shared, history, history_len, token):
    B, K = len(parent), len(parent[0])
    rows, out = B * K, dict(block_table={}, kv_len=[], copy_from=[], copy_to=[], copy_len=[], history=[])
    held = lambda n: -(-n // P)  # noqa: E731
    wants, backs = [], []
    for b in range(B):
        src = [table[b * K + p][: held(kv_len[b * K + p])] for p in range(K)]
        new, copy, seen = [], [], set()
        for j in range(K):
            p = parent[b][j]
            pages = list(src[p]) if p >= 0 else []
            n = kv_len[b * K + p] if p >= 0 else 0
            c = n // P
            if n % P and ((c, pages[c]) in seen or c * P < shared[b]):
                copy.append((j, c, pages[c], n % P))
                pages[c] = None
            elif n % P:
                seen.add((c, pages[c]))
            new.append(pages)
            out["kv_len"].append(n)
        back = []
        for c in range(max(map(len, src))):
            for p in range(K):
                if c < len(src[p]) and c * P >= shared[b] and (c, src[p][c]) not in back and not any(c < len(x) and x[c] == src[p][c] for x in new):
                    back.append((c, src[p][c]))
        backs.append([x for _, x in back])
        wants.append((new, copy))
    left = list(free[:n_free])
    for b in range(B):
        new, copy = wants[b]
        for j, c, page, n in copy:
            to = backs[b].pop(0) if backs[b] else left.pop()
            new[j][c] = to
            out["copy_" + str(b * K + j)] = (page, to, n)
        for j in range(K):
            out["block_table"][b * K + j] = new[j]
            p = parent[b][j]
            f, t, n = out.get("copy_" + str(b * K + j), (-1, -1, 0))
            out["copy_from"].append(f); out["copy_to"].append(t); out["copy_len"].append(n)
            out["history"].append(history[b * K + p][: history_len[b * K + p]] + [token[b][j]] if p >= 0 else [])
    out["free"] = left + [x for back in backs for x in back]
    return out


@pytest.mark.parametrize("B,K,P,top,tail,pool,seed", [
    (1, 1, 16, 5, 1, 40, 0), (1, 4, 16, 300, 2, 400, 1), (3, 8, 8, 500, 3, 2600, 2), (40, 3, 32, 900, 1, 3000, 3), (5, 32, 16, 100, 4, 900, 4),
    (2, 5, 1, 40, 3, 200, 5), (7, 2, 48, 48 * 5, 2, 90, 6), (300, 4, 16, 64, 1, 3000, 7), (1, 8, 16, 16 * 700, 2, 740, 8)])
def test_reorder_follows_the_beams(zq, B, K, P, top, tail, pool, seed):
    rng = np.random.default_rng(seed)
    M, stride = -(-top // P) + 1, top + 3
    pages = list(rng.permutation(pool))
    kv_len = [int(x) for x in np.repeat(rng.integers(0, top + 1, B), K)]
    kv_len[0: K] = [top] * K
    table = rng.integers(0, pool, (B * K, M)).tolist()
    shared = [int(x) for x in rng.integers(0, 2 * P, B)]
    for b in range(B):
        h = -(-kv_len[b * K] // P)
        same = max(0, h - tail)
        common = [int(pages.pop()) for _ in range(same)]
        fork = [[int(pages.pop()) for _ in range(h - same)]]
        for k in range(K):                                        # some rows share the last pages too, as right after a prompt
            if k and rng.random() < 0.7:
                fork.append([int(pages.pop()) for _ in range(h - same)])
            table[b * K + k][:h] = common + fork[-1]
    parent = rng.integers(-1, K, (B, K)).tolist()
    history = rng.integers(0, 1000, (B * K, stride)).tolist()
    history_len = [int(x) for x in rng.integers(0, stride, B * K)]
    token = rng.integers(0, 1000, (B, K)).tolist()
    n_free = len(pages)
    free = [int(p) for p in pages] + [-7] * (pool - n_free)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    old_table = torch.full((B * K, M), -9, dtype=torch.int32, device="cuda")
    args = (i32(parent), i32(kv_len), i32(table), P, pool, i32(free), i32([n_free]))
    out = None
    for _ in range(2):                                            # the second time into the first's outputs
        out = zq.zoqat_op_beam_reorder(*args, shared_len=i32(shared), history=i32(history), history_len=i32(history_len), token=i32(token), out=out)
        if _ == 0:
            out["block_table"].copy_(old_table)
            out["history"].fill_(-9)
    want = reorder_reference(parent, kv_len, table, P, free, n_free, shared, history, history_len, token)
    assert int(out["status"]) == 0
    assert out["kv_len"].tolist() == want["kv_len"]
    for n in ("copy_from", "copy_to", "copy_len"):
        assert out[n].tolist() == want[n], n
    got, hist = out["block_table"].tolist(), out["history"].tolist()
    for r in range(B * K):
        w = want["block_table"][r]
        assert got[r][: len(w)] == w and all(x == -9 for x in got[r][len(w):]), r
        h = want["history"][r]
        assert out["history_len"][r] == len(h) and hist[r][: len(h)] == h and all(x == -9 for x in hist[r][len(h):])
    assert int(out["n_free"]) == len(want["free"])
    assert out["free_pages"].tolist()[: len(want["free"])] == want["free"]


def simple_reorder(zq, **kw):
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    a = dict(parent=[[0, 0]], kv_len=[5, 5], table=[[0, 1, -1], [0, 2, -1]], free=[3, 4, 5, -1, -1, -1], n_free=3)
    a.update(kw)
    return zq.zoqat_op_beam_reorder(i32(a["parent"]), i32(a["kv_len"]), i32(a["table"]), 4, 6, i32(a["free"]), i32([a["n_free"]]))


def test_reorder_reports_what_it_cannot_do(zq):
    ok = simple_reorder(zq)
    assert int(ok["status"]) == 0 and ok["block_table"].tolist() == [[0, 1, -1], [0, 2, -1]] and ok["copy_from"].tolist() == [-1, 1] and ok["copy_to"].tolist() == [-1, 2]
    assert ok["n_free"].tolist() == [3] and ok["free_pages"].tolist()[:3] == [3, 4, 5]
    short = simple_reorder(zq, table=[[0, 1, -1], [0, 1, -1]], n_free=0)                       # the page of both: one more is needed
    assert int(short["status"]) == 2 and short["kv_len"].tolist() == [0, 0] and short["copy_len"].tolist() == [0, 0] and int(short["n_free"]) == 0
    for n in (-1, 7):
        bad = simple_reorder(zq, n_free=n)
        assert int(bad["status"]) == 1 and bad["kv_len"].tolist() == [0, 0]
    assert int(simple_reorder(zq, kv_len=[13, 5])["status"]) == 1
    assert int(simple_reorder(zq, kv_len=[-1, 5])["status"]) == 1
    far = simple_reorder(zq, parent=[[2, 1]])
    assert int(far["status"]) == 8 and far["kv_len"].tolist() == [0, 5]
    page = simple_reorder(zq, table=[[0, 6, -1], [0, 2, -1]])
    assert int(page["status"]) == 4 and page["copy_len"].tolist() == [0, 0]
    ends = simple_reorder(zq, parent=[[-1, -1]])
    assert int(ends["status"]) == 0 and int(ends["n_free"]) == 6 and ends["free_pages"].tolist() == [3, 4, 5, 0, 1, 2] and ends["kv_len"].tolist() == [0, 0]


# ---- copies ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("layers,page,kv,dh,dtype,layout", [(1, 16, 2, 128, "bf16", "token"), (70, 8, 1, 64, "f16", "head"), (3, 100, 5, 64, "f32", "head"), (2, 256, 32, 128, "f32", "token"), (2, 1, 3, 128, "f16", "token")])
def test_copies_of_all_layers(zq, layers, page, kv, dh, dtype, layout):
    n_pages = 12
    caches = [make_cache(n_pages, page, kv, dh, dtype, layout, seed=l) for l in range(layers)]
    before = [(k.clone(), v.clone()) for k, v in caches]
    frm, to, n = [0, 3, -1, 5, 5, 12, 2, 4], [1, 7, -1, 8, 9, 2, 2, 6], [page, (page + 1) // 2, 0, 1, page, 1, 1, page + 1]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    err = zq.zoqat_op_cache_copy(zq.LayerCaches(caches), i32(frm), i32(to), i32(n))
    assert int(err) == 42                                         # rows 5 (a page outside), 6 (onto itself), 7 (too long): left out
    for (k, v), (k0, v0) in zip(caches, before):
        for r in (0, 1, 3, 4):
            k0[to[r], : n[r]] = k0[frm[r], : n[r]]
            v0[to[r], : n[r]] = v0[frm[r], : n[r]]
        assert torch.equal(k, k0) and torch.equal(v, v0)
    empty = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert int(zq.zoqat_op_cache_copy(zq.LayerCaches(caches), empty, empty, empty)) == 0


# ---- attention over a shared prefix ---------------------------------------------------------------------------------
def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prefix_problem(seed, dtype, heads, kv, dh, page, layout, prefix, per, cached, new, mask="tree", pad=2, gap=0, q_scale=1.0, share=True):
    """cached: keys of each request between the prefix and its new rows.  Everything that no row may see is NaN."""
    from test_gpu_serve import ancestors, rand_parents, words_of
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    group = [g for g, n in enumerate(per) for _ in range(n)]
    L = [prefix[g] + c + n for g, c, n in zip(group, cached, new)]
    whole = [p // page if share else 0 for p in prefix]
    held = [-(-x // page) for x in L]
    n_pages = sum(w for w, n in zip(whole, per) if n) + sum(h - whole[g] for g, h in zip(group, held)) + 2
    order = rng.permutation(n_pages).tolist()
    shape = (n_pages, kv, page, dh) if layout == "head" else (n_pages, page, kv, dh)
    k, v = [torch.full(shape, float("nan"), device="cuda", dtype=DTYPES[dtype]) for _ in range(2)]
    if layout == "head":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    rand = lambda n: torch.randn((n, kv, dh), generator=gen, device="cuda").to(DTYPES[dtype])  # noqa: E731
    first = [(rand(p), rand(p)) for p in prefix]
    pages_of = []
    for w, n in zip(whole, per):
        w = w if n else 0
        pages_of.append(order[:w])
        order = order[w:]
    table, keys, vals = [], [], []
    for b, g in enumerate(group):
        mine = pages_of[g] + order[: held[b] - whole[g]]
        order = order[held[b] - whole[g]:]
        table.append(mine + [-3] * (max(held) + 1 - len(mine)))
        keys.append(torch.cat([first[g][0], rand(L[b] - prefix[g])]))
        vals.append(torch.cat([first[g][1], rand(L[b] - prefix[g])]))
        t = torch.arange(L[b], device="cuda")
        pg = torch.tensor(mine + [0], device="cuda")[t // page]
        k[pg, t % page], v[pg, t % page] = keys[-1], vals[-1]
    rows = sum(new)
    q = torch.full((rows + pad, heads + gap, dh), float("nan"), dtype=DTYPES[dtype], device="cuda")[:, :heads]
    q[:rows] = (q_scale * torch.randn((rows, heads, dh), generator=gen, device="cuda")).to(DTYPES[dtype])
    words = max(1, -(-max(new) // 32))
    seen = []
    for n in new:
        if mask == "tree":
            par = rand_parents(rng, [n])
            seen.append([set(ancestors(par, i)) for i in range(n)])
        elif mask == "random":
            seen.append([set(np.nonzero(rng.random(n) < 0.3)[0].tolist()) if i % 3 else set() for i in range(n)])
        else:
            seen.append([set(range(i + 1)) for i in range(n)])
    start, gs = [0], [0]
    for n in new:
        start.append(start[-1] + n)
    for n in per:
        gs.append(gs[-1] + n)
    bits = [words_of(s, words) for r in seen for s in r] + [[-1] * words] * pad
    return dict(dtype=dtype, q=q, k=k, v=v, table=ints(table), kv_len=ints(L), row_start=ints(start), mask=ints(bits) if mask else None, rows=rows, start=start, new=new, L=L,
                keys=keys, vals=vals, seen=seen, heads=heads, kv=kv, dh=dh, scale=1.0 / math.sqrt(dh), group_start=ints(gs), prefix_len=ints(prefix), group=ints(group))


def run_prefix(zq, pr, out=None, **kw):
    out = torch.full_like(pr["q"], 5.0) if out is None else out
    got, err = zq.zoqat_op_prefix_attention(pr["q"], pr["k"], pr["v"], pr["table"], pr["kv_len"], pr["row_start"], pr["group_start"], pr["prefix_len"], pr["group"],
                                            tree_mask=pr["mask"], out=out, **kw)
    assert int(err) == 0
    assert (got[pr["rows"]:] == 5.0).all()                        # rows behind the last request
    return got


def check_prefix(zq, pr, **kw):
    from test_gpu_serve import attention_oracle
    got = run_prefix(zq, pr, **kw)
    want, bound = attention_oracle(pr)                            # (joining two parts is a few of the roundings its bound allows for sums)
    off = (got[: pr["rows"]].double() - want).abs()
    assert bool((off <= bound).all()), (float(off.max()), float((off / bound.clamp(min=1e-30)).max()))
    assert torch.equal(run_prefix(zq, pr, **kw)[: pr["rows"]], got[: pr["rows"]])
    return got


PREFIX = [
    # dtype, heads, kv, dh, page, layout, prefix, per, own cached, new, mask
    ("bf16", 2, 2, 128, 16, "token", [300], [1], [0], [1], "tree"),
    ("f32", 4, 2, 64, 16, "token", [300], [3], [0, 5, 40], [1, 1, 1], None),
    ("bf16", 8, 2, 128, 16, "token", [1000, 0, 127], [4, 3, 2], [0, 1, 2, 300, 0, 9, 200, 0, 5], [1, 1, 1, 1, 1, 1, 1, 1, 1], None),     # groups without a whole tile
    ("f16", 8, 2, 64, 64, "head", [128, 129, 1280], [1, 5, 0], [0, 1, 2, 300, 0, 9], [1, 2, 0, 3, 1, 4], "random"),                      # a group without requests
    ("bf16", 14, 2, 128, 32, "token", [700, 650], [9, 3], list(range(12)), [1] * 12, None),       # 7 query heads per key head, tiles that cut a request's heads apart
    ("f16", 16, 1, 128, 16, "token", [2000], [40], [3 * i for i in range(40)], [1] * 40, None),     # many queries of one prefix: the wide kernel
    ("bf16", 8, 2, 64, 128, "head", [900, 400], [50, 60], [i % 7 for i in range(110)], [1 + i % 3 for i in range(110)], "tree"),
    ("bf16", 32, 8, 128, 64, "token", [3000], [33], [50 * i for i in range(33)], [1] * 33, None),
    ("f16", 4, 4, 128, 16, "token", [513], [130], [i for i in range(130)], [1] * 130, None),
    ("bf16", 4, 4, 64, 16, "token", [100] * 70, [1] * 70, [i for i in range(70)], [1] * 70, None),  # nothing worth sharing
    ("bf16", 8, 1, 128, 16, "token", [20000], [2], [0, 1], [1, 1], None),                          # one prefix over all CTAs
    ("f32", 8, 1, 128, 64, "head", [9000, 31], [4, 2], [0, 100, 7, 8, 0, 1], [1, 2, 1, 1, 3, 1], "tree"),
    ("f32", 6, 2, 64, 24, "token", [200, 95, 96], [3, 1, 6], [i for i in range(10)], [1] * 10, None),
    ("bf16", 20, 1, 64, 8, "token", [640, 260], [3, 4], [5, 0, 7, 130, 0, 64, 1], [33, 2, 40, 1, 0, 5, 17], "random"),          # wide own parts too
    ("f16", 8, 2, 128, 256, "head", [1023, 1024, 1025], [5, 5, 5], [0, 0, 1, 255, 256] * 3, [1] * 15, None),
    # groups and requests in kernels of their own, which share the SMs out
    ("bf16", 8, 2, 128, 16, "token", [100], [40], [i for i in range(40)], [1] * 40, None),                                      # nothing for the groups' kernel
    ("f16", 60, 60, 64, 16, "token", [400], [700], [i % 50 for i in range(700)], [1] * 700, None),                              # a group with more items than CTAs
    ("bf16", 8, 2, 64, 32, "head", [128 + i for i in range(70)], [6] * 70, [i % 40 for i in range(420)], [1] * 420, None),      # more parts than a CTA keeps
    ("f16", 20, 1, 128, 16, "token", [700, 300], [1, 1], [5, 200], [3, 3], "tree"),                                             # wide tiles for requests, narrower for groups
    ("bf16", 8, 8, 128, 8, "token", [5000], [150], [0] * 150, [1] * 150, None),                                                 # next to nothing of their own
    ("f16", 4, 2, 64, 8, "head", [1, 260], [2, 3], [0, 30, 31, 32, 33], [1, 2, 1, 3, 2], "random"),                             # four boxes a tile
]


@pytest.mark.parametrize("case", PREFIX, ids=lambda c: "-".join(str(x) for x in c[:6]) + f"-g{len(c[6])}-b{len(c[8])}-{c[10]}")
def test_prefix_attention_is_the_definition(zq, case):
    check_prefix(zq, prefix_problem(11, *case))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_prefix_attention_steep_scores_strided_rows_and_copied_prefixes(zq, dtype):
    pr = prefix_problem(5, dtype, 8, 2, 128, 16, "token", [520, 300], [6, 4], [i for i in range(10)], [2] * 10, "tree", gap=3, q_scale=20.0, share=False)
    store = torch.full((pr["q"].shape[0], pr["heads"] + 1, 128), 5.0, dtype=DTYPES[dtype], device="cuda")
    got = check_prefix(zq, pr, out=store[:, : pr["heads"]])
    assert (store[:, pr["heads"]:] == 5.0).all()
    scratch = torch.full((zq.prefix_attention_scratch(pr["q"], pr["k"], rows=4 * pr["q"].shape[0]).numel(),), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(run_prefix(zq, pr, scratch=scratch), got)  # what the scratch held does not matter


@pytest.mark.parametrize("dtype,per", [("bf16", [6, 4]), ("f16", [40, 30]), ("f32", [3, 2])])
def test_prefix_attention_is_tree_attention(zq, dtype, per):
    n = sum(per)
    pr = prefix_problem(3, dtype, 8, 2, 128, 16, "token", [700, 140], per, [5 * i for i in range(n)], [1 + i % 2 for i in range(n)], "tree")
    got = run_prefix(zq, pr)
    other, _ = zq.zoqat_op_tree_attention(pr["q"], pr["k"], pr["v"], pr["table"], pr["kv_len"], pr["row_start"], tree_mask=pr["mask"])
    from test_gpu_serve import attention_oracle
    _, bound = attention_oracle(pr)
    assert bool(((got[: pr["rows"]].double() - other[: pr["rows"]].double()).abs() <= 2 * bound).all())


@pytest.mark.parametrize("dtype,per", [("bf16", [2, 3, 2]), ("f16", [30, 40, 30]), ("f32", [2, 3, 2])])
def test_prefix_attention_reports_contradictions_and_leaves_rows(zq, dtype, per):
    from test_gpu_serve import attention_oracle
    n = sum(per)
    pr = prefix_problem(4, dtype, 4, 2, 64, 16, "token", [300, 200, 150], per, [3] * n, [1] * n, None)
    good = run_prefix(zq, pr)
    g1, g2 = per[0], per[0] + per[1]
    def call(**kw):
        a = dict(pr, **kw)
        out = torch.full_like(pr["q"], 5.0)
        _, err = zq.zoqat_op_prefix_attention(a["q"], a["k"], a["v"], a["table"], a["kv_len"], a["row_start"], a["group_start"], a["prefix_len"], a["group"], out=out)
        return out, int(err)
    def changed(t, i, x):
        t = t.clone()
        t[i] = x
        return t
    # (where the parts of a request are cut depends on all requests' lengths, so the others' outputs are held to the definition, not to the bits of another batch)
    want, bound = attention_oracle(pr)
    same = lambda out, rows: bool(((out[: pr["rows"]].double() - want).abs() <= bound)[rows].all())  # noqa: E731
    assert same(good, slice(0, n))
    first, last = slice(0, g1), slice(g2, n)
    for bad in (changed(pr["prefix_len"], 1, -1), changed(pr["prefix_len"], 1, 10 ** 6), changed(pr["prefix_len"], 1, 204)):      # group 1: more than its requests hold
        out, err = call(prefix_len=bad)
        assert err == 41 and same(out, first) and same(out, last) and (out[g1:g2] == 5.0).all()
    for bad in (-1, 3, 0, 2 ** 30):                               # a request in no group, or in one that is not its own
        out, err = call(group=changed(pr["group"], g1, bad))
        assert err == 41 and (out[g1] == 5.0).all() and same(out, first) and same(out, slice(g1 + 1, n))
    out, err = call(group_start=changed(pr["group_start"], 3, n + 5))
    assert err == 41 and same(out, slice(0, g2)) and (out[g2:] == 5.0).all()
    out, err = call(kv_len=changed(pr["kv_len"], g1, 10 ** 7))
    assert err == 41 and (out[g1] == 5.0).all() and same(out, first) and same(out, slice(g1 + 1, n))
    page = pr["table"].clone()
    page[0, 1] = 10 ** 6                                          # in the shared part: its keys and values count as zeros
    out, err = call(table=page)
    assert err == 42 and torch.isfinite(out[:n].float()).all() and same(out, slice(g1, n))


def test_prefix_attention_captured_as_lengths_change(zq):
    from test_gpu_serve import attention_oracle
    n = 9
    pr = prefix_problem(9, "bf16", 8, 2, 128, 16, "token", [900, 300], [5, 4], [40] * n, [1] * n, None)
    out, err, scratch = torch.zeros_like(pr["q"]), torch.zeros(1, dtype=torch.int32, device="cuda"), zq.prefix_attention_scratch(pr["q"], pr["k"])
    call = lambda: zq.zoqat_op_prefix_attention(pr["q"], pr["k"], pr["v"], pr["table"], pr["kv_len"], pr["row_start"], pr["group_start"], pr["prefix_len"],  # noqa: E731
                                                pr["group"], out=out, scratch=scratch, err=err)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for prefix, own in (([900, 300], [10, 41, 1, 2, 3, 40, 30, 20, 1]), ([130, 127], [1] * 9), ([0, 0], [30] * 9)):
        L = [prefix[0 if b < 5 else 1] + own[b] for b in range(n)]
        pr["kv_len"].copy_(ints(L))
        pr["prefix_len"].copy_(ints(prefix))
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        now = dict(pr, L=L, keys=[k[:x] for k, x in zip(pr["keys"], L)], vals=[v[:x] for v, x in zip(pr["vals"], L)])
        want, bound = attention_oracle(now)
        assert int(err) == 0 and bool(((out[:n].double() - want).abs() <= bound).all()) and (out[n:] == 5.0).all()


def test_prefix_attention_two_streams_at_once(zq):
    prs = [prefix_problem(21 + i, "bf16", 8, 2, 128, 16, "token", [1500 - 700 * i], [40], [7 * j for j in range(40)], [1] * 40, None) for i in range(2)]
    alone = [run_prefix(zq, pr) for pr in prs]
    streams = [torch.cuda.Stream() for _ in prs]
    outs = [torch.full_like(pr["q"], 5.0) for pr in prs]
    torch.cuda.synchronize()
    for _ in range(10):
        for pr, s, o in zip(prs, streams, outs):
            with torch.cuda.stream(s):
                zq.zoqat_op_prefix_attention(pr["q"], pr["k"], pr["v"], pr["table"], pr["kv_len"], pr["row_start"], pr["group_start"], pr["prefix_len"], pr["group"], out=o)
    torch.cuda.synchronize()
    assert all(torch.equal(o, a) for o, a in zip(outs, alone))


def test_prefix_attention_no_rows(zq):
    k, v = make_cache(4, 16, 2, 64, "bf16", "token")
    out, err = zq.zoqat_op_prefix_attention(torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda"), k, v, ints([[0]]), ints([0]), ints([0, 0]), ints([0, 1]), ints([0]), ints([0]))
    assert out.shape == (0, 4, 64) and int(err) == 0


# ---- a beam search through a packed model ---------------------------------------------------------------------------
def beam_search(zq, shape, model, prompts, K, page, dtype, steps, eos, shared):
    """Beams of all prompts as requests of one batch, advanced by the operators alone.  shared: the prompts' keys are attended to once (zoqat_decode_prefix_step).
    Returns (tokens, score) of every beam at the end, the finished ones as (tokens, score), and the number of pages copied."""
    G, B, V, n_pages, M = len(prompts), len(prompts) * K, shape["vocab"], 400, 24
    dh, longest = shape["d_model"] // shape["n_heads"], max(map(len, prompts)) + steps + 1
    caches = [make_cache(n_pages, page, shape["n_heads"], dh, dtype, "token", seed=l) for l in range(shape["n_layers"])]
    M = -(-longest // page) + 1
    layers = zq.LayerCaches(caches)
    table = torch.full((B, M), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(n_pages, generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda()
    n_free, cached = ints([n_pages]), ints([0] * B)
    # the prompts, through the first beam of each
    todo, last = [list(p) for p in prompts], [None] * G
    while any(todo):
        share = [min(len(t), 8 // G) for t in todo]
        flat = [x for t, n in zip(todo, share) for x in t[:n]]
        plan = zq.zoqat_op_cache_plan(cached, ints([share[b // K] if b % K == 0 else 0 for b in range(B)]), page, n_pages, free, n_free, table, 8)
        logits, _ = model.zoqat_decode_tree_step(ints(flat + [0] * (8 - len(flat))), plan, table, caches)
        at = 0
        for g in range(G):
            at += share[g]
            if share[g]:
                last[g] = logits[at - 1].clone()
        todo = [t[n:] for t, n in zip(todo, share)]
        cached, n_free = plan["kv_len"], plan["n_free"]
    groups = (ints([g * K for g in range(G + 1)]), ints([len(p) for p in prompts]), ints([b // K for b in range(B)]))
    logits = torch.stack(last).repeat_interleave(K, 0)
    score = torch.full((G, K), -math.inf, device="cuda")
    score[:, 0] = 0.0
    history = torch.zeros((B, longest), dtype=torch.int32, device="cuda")
    for b in range(B):
        history[b, : len(prompts[b // K])] = ints(prompts[b // K])
    history_len = ints([len(prompts[b // K]) if b % K == 0 else 0 for b in range(B)])
    done, copies = [], 0
    for step in range(steps):
        best = zq.zoqat_op_beam_select(logits, score, eos=ints(eos))
        for g in range(G):                                        # finished ones: the parent's tokens, then the one that ends
            for k in range(K):
                if int(best["done_beam"][g, k]) >= 0:
                    row = g * K + int(best["done_beam"][g, k])
                    done.append((history[row, : int(history_len[row])].tolist() + [int(best["done_token"][g, k])], float(best["done_score"][g, k])))
        out = zq.zoqat_op_beam_reorder(best["beam"], cached, table, page, n_pages, free, n_free, history=history, history_len=history_len, token=best["token"])
        zq.zoqat_op_cache_copy(layers, out["copy_from"], out["copy_to"], out["copy_len"], err=out["status"])
        assert int(out["status"]) == 0
        table, cached, free, n_free, history, history_len = (out[n] for n in ("block_table", "kv_len", "free_pages", "n_free", "history", "history_len"))
        copies += int((out["copy_len"] > 0).sum())
        held = {p for b in range(B) for p in table[b, : -(-int(cached[b]) // page)].tolist()}
        spare = free[: int(n_free)].tolist()
        assert len(held) + len(spare) == n_pages and held.isdisjoint(spare) and held | set(spare) == set(range(n_pages))      # no page is lost or held twice
        score = best["score"]
        plan = zq.zoqat_op_cache_plan(cached, ints([1] * B), page, n_pages, free, n_free, table, B)
        assert int(plan["status"]) == 0
        if shared:
            logits, _ = model.zoqat_decode_prefix_step(best["token"].view(-1).clamp(min=0), plan, table, *groups, caches)
        else:
            logits, _ = model.zoqat_decode_tree_step(best["token"].view(-1).clamp(min=0), plan, table, caches)
        model.zoqat_check()
        cached, n_free = plan["kv_len"], plan["n_free"]
    live = [(history[b, : int(history_len[b])].tolist(), float(score.view(-1)[b])) for b in range(B)]
    return live, done, copies


@pytest.mark.parametrize("name,dtype,page,K,lengths", [("llama_w4a8", "f32", 16, 4, (37, 70)), ("llama_w4", "bf16", 16, 4, (135, 150)), ("opt_w3a8", "f32", 5, 8, (40,)),
                                                       ("llama_w4a8", "f16", 8, 2, (5, 130, 140, 131))])
def test_beam_search_through_a_packed_model(zq, name, dtype, page, K, lengths):
    from test_gpu_serve import packed_model, sequential_logits
    shape, model = packed_model(zq, name, 8, 192)
    _, other = packed_model(zq, name, 2, 192)
    rng = np.random.default_rng(4)
    prompts = [rng.integers(3, shape["vocab"], n).tolist() for n in lengths]
    eos = [int(x) for x in rng.integers(3, shape["vocab"], 2)]
    live, done, copies = beam_search(zq, shape, model, prompts, K, page, dtype, 7, eos, shared=True)
    assert copies > 0
    # every hypothesis' score is the sum of its tokens' log-probabilities by the one-token path, which keeps no pages: a row that followed the wrong
    # beam, or lost a key of its page, is off by whole units.  Per token the logits differ by up to 2 % (5 % with bf16 keys) of their scale
    # (a difference of one code in one activation; see the test of drafts), the log of their sum by as much again.
    tol = {"f32": 2e-2, "f16": 2e-2, "bf16": 5e-2}[dtype]
    for tokens, score in (live[:: max(1, len(live) // 4)] + done[:2]):
        p = next(p for p in prompts if tokens[: len(p)] == p)
        want, bound = 0.0, 0.0
        for i in range(len(p), len(tokens)):
            logits = sequential_logits(other, tokens[:i], 2).double()
            want += float(torch.log_softmax(logits, 0)[tokens[i]])
            bound += 2 * tol * float(logits.abs().max())
        assert abs(score - want) <= bound, (score, want, bound)
    for g in range(len(prompts)):
        mine = [s for _, s in live[g * K: (g + 1) * K]]
        assert mine == sorted(mine, reverse=True) and len({tuple(t) for t, _ in live[g * K: (g + 1) * K]}) == K


def test_prefix_step_is_the_tree_step(zq):
    """The same search with and without the shared prefix: the same first beams, the same scores up to the attention's rounding."""
    from test_gpu_serve import packed_model
    shape, model = packed_model(zq, "llama_w4a8", 8, 192)
    prompts = [list(range(3, 60)), list(range(100, 190))]
    one, two = [beam_search(zq, shape, model, prompts, 4, 16, "f32", 3, [1], shared) for shared in (True, False)]
    for (a, x), (b, y) in zip(one[0], two[0]):
        assert abs(x - y) <= 0.05 * max(1.0, abs(y))
    with pytest.raises(zq.ZoqatError):
        model.zoqat_decode_prefix_step(ints([1]), dict(kv_len=ints([1]), row_start=ints([0, 1]), row_pos=ints([0]), slot=ints([0])), ints([[0]]), ints([0, 1]), ints([0]),
                                       ints([0]), [make_cache(4, 16, 2, 64, "f32", "token")] * 2, scratch=torch.empty(1 << 16, dtype=torch.uint8, device="cuda"))


def test_the_operators_of_a_layer_in_a_row(zq):
    """A layer's new rows with head norms and interleaved rotation at far positions, into pages and through the shared-prefix attention: against float64 from end to end."""
    G, K, prefix, heads, kv, dh, page = 2, 3, [300, 170], 4, 2, 64, 16
    B, gen = G * K, torch.Generator(device="cuda").manual_seed(8)
    freq, mag = zq.rotary_frequencies(32, kind=zq.ROTARY_LINEAR, factor=8.0)
    qg, kg = 1 + 0.2 * torch.randn((2, dh), generator=gen, device="cuda")
    L = [prefix[b // K] + 1 for b in range(B)]
    n_pages = 100
    k, v = make_cache(n_pages, page, kv, dh, "bf16", "token")
    table, free = torch.full((B, 24), -1, dtype=torch.int32, device="cuda"), torch.arange(n_pages, dtype=torch.int32, device="cuda")
    wide = (heads + 2 * kv) * dh
    # the prompts' rows through the first beam of each group, then their pages for all beams
    plan = zq.zoqat_op_cache_plan(ints([0] * B), ints([prefix[b // K] if b % K == 0 else 0 for b in range(B)]), page, n_pages, free, ints([n_pages]), table, sum(prefix))
    x = torch.randn((sum(prefix), wide), generator=gen, device="cuda")
    far = 100000
    zq.zoqat_op_rotary_append(x, plan["row_pos"] + far, plan["slot"], k, v, heads, freq=freq, interleaved=True, magnitude=mag, q_gain=qg, k_gain=kg)
    out = zq.zoqat_op_beam_reorder(ints([[0] * K] * G), plan["kv_len"], table, page, n_pages, free, plan["n_free"])
    zq.zoqat_op_cache_copy(zq.LayerCaches([(k, v)]), out["copy_from"], out["copy_to"], out["copy_len"])
    step = zq.zoqat_op_cache_plan(out["kv_len"], ints([1] * B), page, n_pages, out["free_pages"], out["n_free"], out["block_table"], B)
    y = torch.randn((B, wide), generator=gen, device="cuda")
    q, err = zq.zoqat_op_rotary_append(y, step["row_pos"] + far, step["slot"], k, v, heads, freq=freq, interleaved=True, magnitude=mag, q_gain=qg, k_gain=kg)
    got, err2 = zq.zoqat_op_prefix_attention(q, k, v, out["block_table"], step["kv_len"], step["row_start"], ints([0, K, 2 * K]), ints(prefix), ints([0] * K + [1] * K))
    assert int(err) == int(err2) == 0 and step["kv_len"].tolist() == L
    ref = lambda z, pos: append_reference(z, pos, heads, kv, dh, freq, True, mag, qg, kg, 1e-6)[0]  # noqa: E731
    start = [0, prefix[0]]
    for b in range(B):
        g = b // K
        pos = torch.arange(prefix[g] + 1, device="cuda") + far
        rows = ref(torch.cat([x[start[g]: start[g] + prefix[g]], y[b: b + 1]]), pos)
        for h in range(heads):
            qq, kk, vv = rows[-1, h], rows[:, heads + h // 2], rows[:, heads + kv + h // 2]
            w = torch.softmax(kk @ qq / math.sqrt(dh), 0)
            want, size = w @ vv, w @ vv.abs()
            # queries, keys, values, weights and outputs are rounded to bf16 once (2^-8 each): a score moves by two of those of the sum of its products'
            # sizes, a weight relatively by twice that, and fp32's share (angles of far positions among it) is under a tenth of it
            half, products = 2.0 ** -8, float((kk.abs() @ qq.abs()).max()) / math.sqrt(dh)
            bound = 1.1 * ((4 * half * products + 2 * half) * size + half * want.abs())
            assert bool(((got[b, h].double() - want).abs() <= bound).all())


def test_a_captured_step_of_beams(zq):
    """Selection, reordering, copies and attention in one graph: replayed on new logits and scores it gives what the calls give."""
    G, K, V, page, n_pages, prefix = 2, 4, 9000, 16, 120, 200
    B, rng = G * K, torch.Generator(device="cuda").manual_seed(6)
    caches = [make_cache(n_pages, page, 2, 64, "bf16", "token", seed=l) for l in range(3)]
    keep = [(k.clone(), v.clone()) for k, v in caches]
    layers = zq.LayerCaches(caches)
    common = list(range(12))
    table = torch.full((B, 20), -1, dtype=torch.int32, device="cuda")
    for b in range(B):
        table[b, :13] = ints([x + 40 * (b // K) for x in common] + [20 + b % K + 40 * (b // K)])
    kv_len = ints([prefix + 3] * B)
    free, n_free = torch.arange(80, 120, dtype=torch.int32, device="cuda"), ints([40])
    logits, score = torch.zeros((B, V), device="cuda"), torch.zeros((G, K), device="cuda")
    q = torch.randn((B, 4, 64), generator=rng, device="cuda").to(torch.bfloat16)
    rows, groups = ints(list(range(B + 1))), (ints([0, K, B]), ints([prefix - 8] * G), ints([0] * K + [1] * K))
    scratch, attention, err = zq.beam_reorder_scratch(score), zq.prefix_attention_scratch(q, caches[0][0]), torch.zeros(1, dtype=torch.int32, device="cuda")
    state = {}

    def step(best=None, out=None, att=None):
        best = zq.zoqat_op_beam_select(logits, score, eos=None, out=best)
        out = zq.zoqat_op_beam_reorder(best["beam"], kv_len, table, page, n_pages, free, n_free, out=out, scratch=scratch)
        zq.zoqat_op_cache_copy(layers, out["copy_from"], out["copy_to"], out["copy_len"], err=err)
        att, _ = zq.zoqat_op_prefix_attention(q, *caches[0], out["block_table"], out["kv_len"], rows, *groups, out=att, scratch=attention, err=err)
        return best, out, att

    state = step()                                                # warm, and buffers for the graph
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(*state)
    for i in range(4):
        logits.copy_(3 * torch.randn((B, V), generator=rng, device="cuda"))
        score.copy_(-5 * torch.rand((G, K), generator=rng, device="cuda"))
        for (k, v), (k0, v0) in zip(caches, keep):
            k.copy_(k0)
            v.copy_(v0)
        graph.replay()
        torch.cuda.synchronize()
        got = [{n: t.clone() for n, t in d.items()} for d in state[:2]] + [state[2].clone()] + [t.clone() for kv in caches for t in kv]
        for (k, v), (k0, v0) in zip(caches, keep):
            k.copy_(k0)
            v.copy_(v0)
        best, out, att = step()
        live = lambda d: {n: t for n, t in d.items() if n not in ("block_table", "free_pages")}  # noqa: E731
        assert all(torch.equal(got[0][n], best[n]) for n in best) and all(torch.equal(got[1][n], out[n]) for n in live(out))
        assert torch.equal(got[1]["block_table"][:, :13], out["block_table"][:, :13]) and torch.equal(got[2], att)
        assert all(torch.equal(x, y) for x, y in zip(got[3:], [t for kv in caches for t in kv])) and int(err) == 0 and int(out["status"]) == 0


def test_large_batches_and_far_pages(zq):
    """The largest batch of the selection's and the reordering's rules, and copies in pages that lie behind 2^32 elements."""
    B, K = 16384, 4
    gen = torch.Generator(device="cuda").manual_seed(1)
    parent = torch.randint(-1, K, (B, K), generator=gen, device="cuda").int()
    table = torch.arange(B * K, dtype=torch.int32, device="cuda").view(B * K, 1)
    kv_len = torch.randint(0, 5, (B * K,), generator=gen, device="cuda").int()
    kv_len = kv_len.view(B, K)[:, :1].expand(B, K).contiguous().view(-1)
    n_pages = 3 * B * K
    free = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    free[: 2 * B * K] = torch.arange(B * K, n_pages, dtype=torch.int32, device="cuda")
    out = zq.zoqat_op_beam_reorder(parent, kv_len, table, 4, n_pages, free, ints([2 * B * K]))
    want = reorder_reference(parent.tolist(), kv_len.tolist(), table.tolist(), 4, free.tolist(), 2 * B * K, [0] * B, [[0]] * (B * K), [0] * (B * K), [[0] * K] * B)
    assert int(out["status"]) == 0 and out["kv_len"].tolist() == want["kv_len"] and int(out["n_free"]) == len(want["free"])
    for n in ("copy_from", "copy_to", "copy_len"):
        assert out[n].tolist() == want[n], n
    assert out["free_pages"].tolist()[: len(want["free"])] == want["free"]
    logits = torch.randn((B * 2, 700), generator=gen, device="cuda")
    got = zq.zoqat_op_beam_select(logits, torch.zeros((B, 2), device="cuda"))
    both = torch.log_softmax(logits.double(), 1).view(B, 2, 700).flatten(1)
    top = both.max(1)
    assert torch.equal(got["beam"][:, 0].long() * 700 + got["token"][:, 0], top.indices) and bool(((got["score"][:, 0].double() - top.values).abs() < 1e-5).all())
    # 2 pages of 2^31 elements and more apart
    stride = (1 << 31) + 4096
    store = torch.empty(3 * stride, dtype=torch.bfloat16, device="cuda")
    k = torch.as_strided(store, (3, 16, 2, 64), (stride, 128, 64, 1))
    v = torch.as_strided(store, (3, 16, 2, 64), (stride, 128, 64, 1), 2048)
    for t in (k, v):
        t.copy_(torch.randn((3, 16, 2, 64), generator=gen, device="cuda").to(torch.bfloat16))
    k0, v0 = k.clone(), v.clone()
    err = zq.zoqat_op_cache_copy(zq.LayerCaches([(k, v)]), ints([0]), ints([2]), ints([9]))
    assert int(err) == 0 and torch.equal(k[2, :9], k0[0, :9]) and torch.equal(k[2, 9:], k0[2, 9:]) and torch.equal(v[2, :9], v0[0, :9]) and torch.equal(v[1], v0[1])
    qkv = torch.randn((2, 4 * 64 + 2 * 2 * 64), generator=gen, device="cuda")
    q, err = zq.zoqat_op_rotary_append(qkv, ints([3, 4]), ints([2 * 16 + 15, 16]), k, v, 4, freq=zq.rotary_frequencies(64)[0])
    assert int(err) == 0 and torch.equal(v[2, 15], qkv.view(2, -1, 64)[0, 6:].to(torch.bfloat16)) and torch.equal(v[1, 0], qkv.view(2, -1, 64)[1, 6:].to(torch.bfloat16))
    out, err = zq.zoqat_op_prefix_attention(q, k, v, ints([[0, 2], [0, 1]]), ints([32, 17]), ints([0, 1, 2]), ints([0, 2]), ints([16]), ints([0, 0]))
    other, _ = zq.zoqat_op_tree_attention(q, k, v, ints([[0, 2], [0, 1]]), ints([32, 17]), ints([0, 1, 2]))
    # each of the two is off by the rounding of its weights and of its output: 2^-8 of the values' sizes, twice, and fp32's share
    assert int(err) == 0 and float((out.double() - other.double()).abs().max()) <= 2 * 2.1 * 2.0 ** -8 * float(v[[0, 1, 2]].abs().max())
