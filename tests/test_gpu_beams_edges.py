"""Batches that change while they run: requests that have ended, beams of different lengths, equal scores, and the step of a model compared with the one without groups."""
import math

import numpy as np
import pytest
import torch

from test_gpu_beams import check_select, ints, make_cache, prefix_problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def zq():
    from paper_2509_00031_b200 import binding
    binding.lib()
    return binding


# ---- attention over a shared prefix: requests that have ended -----------------------------------------------------------
def attend(zq, pr, **kw):
    a = dict(pr, **kw)
    out = torch.full_like(pr["q"], 5.0)
    _, err = zq.zoqat_op_prefix_attention(a["q"], a["k"], a["v"], a["table"], a["kv_len"], a["row_start"], a["group_start"], a["prefix_len"], a["group"], tree_mask=a["mask"], out=out)
    return out, int(err)


def held_to(pr, out, requests, untouched=()):
    from test_gpu_serve import attention_oracle
    want, bound = attention_oracle(pr)
    off = (out[: pr["rows"]].double() - want).abs() <= bound
    for b in requests:
        assert bool(off[pr["start"][b]: pr["start"][b + 1]].all()), b
    for b in untouched:
        assert bool((out[pr["start"][b]: pr["start"][b + 1]] == 5.0).all()), b
    assert bool((out[pr["rows"]:] == 5.0).all())


ENDED = [
    # dtype, heads, kv, dh, page, layout, prefix, per, own cached, new, mask: the requests without rows have ended
    ("bf16", 8, 2, 128, 16, "token", [700, 300], [4, 3], [3] * 7, [0, 1, 1, 1, 0, 0, 2], "random"),       # few queries: a run per warp, both sides in one launch
    ("f32", 4, 2, 64, 64, "head", [700, 300], [4, 3], [3] * 7, [0, 1, 1, 1, 0, 0, 2], None),
    ("f32", 8, 1, 128, 16, "token", [500], [3], [0, 1, 2], [0, 0, 3], None),
    ("f16", 8, 2, 128, 32, "token", [640], [12], [i for i in range(12)], [0] * 3 + [1] * 9, None),          # keys as rows
    ("bf16", 16, 1, 64, 16, "token", [900], [40], [2 * i for i in range(40)], [0] * 17 + [1] * 23, None),   # 256 queries a tile
    ("f16", 20, 1, 128, 16, "head", [600], [2], [5, 9], [0, 30], None),                                    # 256 queries a tile, both sides in one launch
    ("bf16", 4, 4, 64, 16, "token", [400, 200], [70, 30], [1] * 100, [0] * 66 + [1] * 4 + [0, 1] * 15, None),
    ("f16", 8, 2, 64, 16, "token", [300, 260, 200], [3, 2, 1], [1] * 6, [0, 0, 0, 1, 1, 0], None),          # groups that have ended whole
    ("bf16", 8, 2, 64, 32, "head", [128 + i for i in range(70)], [6] * 70, [i % 40 for i in range(420)], [0, 0, 1, 0, 1, 1] * 70, None),   # more parts than a CTA keeps
]


@pytest.mark.parametrize("row", ["gone", "reused", "short"])
@pytest.mark.parametrize("case", ENDED, ids=lambda c: "-".join(str(x) for x in c[:6]) + f"-b{len(c[8])}")
def test_a_prefix_is_read_through_a_request_that_holds_it(zq, case, row):
    """A request that has ended keeps its place in the batch: no rows, no keys, and a row of the table that names no pages, or pages that are others' by now."""
    pr = prefix_problem(13, *case)
    ended = [b for b, n in enumerate(pr["new"]) if n == 0]
    table, kv_len = pr["table"].clone(), pr["kv_len"].clone()
    table[ended] = -1 if row == "gone" else int(pr["table"][pr["new"].index(1) if 1 in pr["new"] else -1, 2])
    kv_len[ended] = 100 if row == "short" else 0
    out, err = attend(zq, pr, table=table, kv_len=kv_len)
    assert err == 0
    held_to(pr, out, range(len(pr["new"])))


@pytest.mark.parametrize("case", ENDED[:6], ids=lambda c: "-".join(str(x) for x in c[:6]) + f"-b{len(c[8])}")
def test_requests_that_have_ended_may_say_anything(zq, case):
    pr = prefix_problem(16, *case)
    ended = [b for b, n in enumerate(pr["new"]) if n == 0]
    for length, of in ((2 ** 31 - 1, -1), (-2 ** 31, 2 ** 31 - 1), (10 ** 6, 1), (-1, -2 ** 31)):
        kv_len, group = pr["kv_len"].clone(), pr["group"].clone()
        kv_len[ended], group[ended] = length, of
        out, err = attend(zq, pr, kv_len=kv_len, group=group)
        assert err == 0
        held_to(pr, out, range(len(pr["new"])))


@pytest.mark.parametrize("dtype,per,new", [("bf16", [3, 2], 1), ("f16", [40, 30], 1), ("f16", [12, 12], 2), ("f32", [3, 2], 1)])
def test_a_first_request_that_contradicts_its_group_is_left_out_alone(zq, dtype, per, new):
    n = sum(per)
    pr = prefix_problem(14, dtype, 8, 2, 64, 16, "token", [400, 300], per, [4] * n, [new] * n, None)
    table, kv_len = pr["table"].clone(), pr["kv_len"].clone()
    table[:2] = -1
    kv_len[:2] = 400 + new - 1                                    # a key short of the prefix
    out, err = attend(zq, pr, table=table, kv_len=kv_len)
    assert err == 41
    held_to(pr, out, range(2, n), untouched=(0, 1))
    group = pr["group"].clone()
    group[per[0]] = 0                                             # the second group's first request names the other one
    table = pr["table"].clone()
    table[per[0]] = -1
    out, err = attend(zq, pr, table=table, group=group)
    assert err == 41
    held_to(pr, out, [b for b in range(n) if b != per[0]], untouched=(per[0],))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_lengths_at_the_ends_of_their_type_are_left_out(zq, dtype):
    """A length less its rows has to be formed in more than 32 bits: the least number less one is the largest."""
    n = 5
    pr = prefix_problem(15, dtype, 8, 2, 64, 16, "token", [300], [n], [4] * n, [1, 2, 1, 3, 1], None)
    for length in (-2 ** 31, -2 ** 31 + 2, 2 ** 31 - 1, -1):
        for b in (0, 3):
            kv_len = pr["kv_len"].clone()
            kv_len[b] = length
            out, err = attend(zq, pr, kv_len=kv_len)
            assert err == 41
            held_to(pr, out, [i for i in range(n) if i != b], untouched=(b,))


# ---- selection: equal scores -------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("K,V", [(4, 32000), (1, 32000), (3, 20003), (2, 40001)])
def test_equal_scores_come_larger_logit_first_wherever_a_row_is_cut(zq, K, V, dtype):
    """Beside a beam score of large magnitude every logit of a row gives the same score, or nearly: the order within a beam is that of logits all the same.  Rows
    of one request are cut into slices, those of a hundred are not."""
    gen = torch.Generator(device="cuda").manual_seed(K)
    x = torch.randn((K, V), generator=gen, device="cuda")
    at = torch.linspace(7, V - 3, 40, device="cuda").long()
    x[:, at] = 9.0 + torch.arange(40, device="cuda") * (2.0 ** -20 if dtype == "f32" else 2.0 ** -7)       # rising to the end of the row
    x[:, at[::5] + 1] = x[:, at[20]].clone()[:, None]                     # some of them twice and more
    x = x.to({"f32": torch.float32, "f16": torch.float16}[dtype])
    few = x.clone()
    few[0] = -math.inf
    few[0, V // 2: V // 2 + 2] = 1.0                              # two continuations of the first beam: the others have to step in
    for logits in (x, few):
        for first, others in ((-1e30, -1e30), (0.0, -1e30), (-1e10, -math.inf), (-1e10, -1e30)):
            scores = torch.full((1, K), others, device="cuda")
            scores[0, 0] = first
            one = check_select(zq, logits, scores, (int(at[37]), 3))
            many = zq.zoqat_op_beam_select(logits.repeat(100, 1), scores.repeat(100, 1), eos=ints([int(at[37]), 3]))
            # (the order is the same to the last; a row's sum is cut where the row is, so each of two scores is off by up to what check_select allows)
            for n, t in one.items():
                other = t.expand(100, K)
                if t.dtype is torch.int32:
                    assert torch.equal(many[n], other), n
                else:
                    live = torch.isfinite(other)
                    assert torch.equal(torch.isfinite(many[n]), live)
                    assert ((many[n].double() - other.double())[live].abs() <= 2 * (2.0 ** -24 * other.double()[live].abs() + 2.0 ** -20)).all()


def test_equal_logits_come_in_the_order_of_tokens(zq):
    for K in (1, 3, 8):
        got = zq.zoqat_op_beam_select(torch.zeros((2 * K, 40000), device="cuda"), -torch.arange(2 * K, device="cuda", dtype=torch.float32).view(2, K) * 0.37)
        assert got["token"].tolist() == [list(range(K))] * 2 and got["beam"].tolist() == [[0] * K] * 2


def test_bounds_that_pass_a_threads_own_logits(zq):
    """Rows whose first thousands of logits are low, and whose rest rises with a few steps: the bound of the best passes what most threads have met."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    V = 120000
    for low, step, spread in ((-300.0, 290.0, 1.0), (-40.0, 40.0, 20.0), (-1e9, 1e9, 3.0)):
        x = spread * torch.randn((6, V), generator=gen, device="cuda")
        x[:, :9000] += low
        x[:, 9000:] += low + step * (torch.arange(V - 9000, device="cuda") // 20000 + 1) / 6
        check_select(zq, x, torch.zeros((2, 3), device="cuda"), (5,))
        check_select(zq, x.repeat(40, 1), torch.zeros((80, 3), device="cuda"), (5,))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("ld", [131072, 131073])
def test_sums_of_many_equal_logits(zq, dtype, ld):
    """Few different logits: the roundings of a sum's equal terms do not cancel out."""
    V, rows = 131072, 160
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((rows, ld), generator=gen, device="cuda")
    one = torch.full_like(x, 0.37)
    one[:, 5] = 1.3
    for y in (one, (x > 0).float() * -0.6, x.round()):
        y = y.to({"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype])[:, :V]
        got = zq.zoqat_op_beam_select(y, torch.zeros((rows, 1), device="cuda"))["score"][:, 0].double()
        want = y.double().amax(1) - torch.logsumexp(y.double(), 1)
        # an exponential is off by 2^-22, its argument (up to 8) by 2^-22 ln 2.  A term goes through at most 32 additions within its part of the row, then the thread's parts
        # (8192 logits each, with rows that do not begin on 16 bytes 2048), 5 steps over the lanes and 8 over the warps, each off by 2^-24; and the score is rounded once
        steps = 32 + V // (8192 if ld % 8 == 0 else 2048) + 13
        assert bool(((got - want).abs() <= 2 * 2.0 ** -22 + steps * 2.0 ** -24 + 2.0 ** -24 * want.abs()).all())


# ---- reordering: rows of different lengths -----------------------------------------------------------------------------
@pytest.mark.parametrize("B,K,P,longest,seed", [(1, 4, 4, 30, 0), (3, 8, 8, 90, 1), (4, 32, 4, 60, 2), (40, 6, 16, 200, 3), (2, 5, 16, 5000, 4), (200, 3, 2, 12, 5)])
def test_rows_of_any_length_keep_their_keys(zq, B, K, P, longest, seed):
    """Rows of a request that hold beginnings of one text, of different lengths, in the same pages.  Slots are followed through the reordering, the copies and the rows' next
    keys: every row reads its own."""
    rng = np.random.default_rng(seed)
    M = -(-longest // P) + 1
    pool = B * K * (M + 1)
    pages, rows = rng.permutation(pool).tolist(), B * K
    store = np.full((pool, P), -1, dtype=np.int64)
    kv_len, table, text = [0] * rows, np.full((rows, M), -1, dtype=np.int64), [[] for _ in range(rows)]
    for b in range(B):
        whole = [pages.pop() for _ in range(M)]
        base = rng.integers(0, 1 << 40, longest)
        for i, t in enumerate(base):
            store[whole[i // P], i % P] = t
        for k in range(K):
            r, n = b * K + k, int(rng.integers(0, longest + 1))
            kv_len[r], text[r] = n, base[:n].tolist()
            table[r, : -(-n // P)] = whole[: -(-n // P)]
        last = max(kv_len[b * K: b * K + K])
        pages += whole[-(-last // P):]                            # (pages that nobody holds)
    rng.shuffle(pages)
    free = pages + [-7] * (pool - len(pages))
    parent = rng.integers(-1, K, (B, K))
    parent[:, 0] = np.where(rng.random(B) < 0.5, rng.integers(0, K, B), parent[:, 0])
    out = zq.zoqat_op_beam_reorder(ints(parent.tolist()), ints(kv_len), ints(table.tolist()), P, pool, ints(free), ints([len(pages)]))
    assert int(out["status"]) == 0
    new_len, new_table = out["kv_len"].tolist(), out["block_table"].cpu().numpy()
    for f, t, n in zip(out["copy_from"].tolist(), out["copy_to"].tolist(), out["copy_len"].tolist()):
        if n:
            store[t, :n] = store[f, :n]
    want = []
    for r in range(rows):
        p = parent[r // K, r % K]
        want.append(list(text[r // K * K + p]) if p >= 0 else [])
        assert new_len[r] == len(want[r])
        if new_len[r] % P:                                        # the next key, where the page has room
            want[r].append(int(1 << 41) + r)
            store[new_table[r, new_len[r] // P], new_len[r] % P] = want[r][-1]
    held = set()
    for r in range(rows):
        i = np.arange(len(want[r]))
        assert bool((store[new_table[r, i // P], i % P] == np.array(want[r], dtype=np.int64)).all()), r
        held |= set(new_table[r, : -(-new_len[r] // P)].tolist())
    left = out["free_pages"][: int(out["n_free"])].tolist()
    assert len(set(left)) == len(left) and held.isdisjoint(left) and held | set(left) == set(range(pool))


# ---- the step of a packed model ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("name,dtype,prefix,own", [("llama_w4a8", "f32", [150, 90], [5, 0]), ("llama_w4a8", "bf16", [140, 131], [9, 30]), ("llama_w4", "f16", [160, 129], [1, 2])])
def test_one_step_with_and_without_the_shared_prefix(zq, name, dtype, prefix, own):
    """The same tokens, plan and caches through both steps: logits agree, and do not where a tile of the prefix is another one."""
    from test_gpu_serve import packed_model
    shape, model = packed_model(zq, name, 8, 192)
    H, dh, page, n_pages, K = shape["n_heads"], shape["d_model"] // shape["n_heads"], 16, 80, 4
    B = 2 * K
    caches = [make_cache(n_pages, page, H, dh, dtype, "token", seed=l) for l in range(shape["n_layers"])]
    cached = [prefix[b // K] + own[b // K] for b in range(B)]
    rng = np.random.default_rng(2)
    order = rng.permutation(n_pages).tolist()
    table = torch.full((B, 13), -1, dtype=torch.int32, device="cuda")
    for g in range(2):
        whole = [order.pop() for _ in range(prefix[g] // page)]
        for b in range(g * K, g * K + K):
            rest = -(-cached[b] // page) - len(whole)
            mine = whole + [order.pop() for _ in range(rest)]
            table[b, : len(mine)] = ints(mine)
            for k, v in caches:                                   # what is left of the prefix lies in a page of each request's own
                for t in (k, v):
                    t[mine[len(whole)], : prefix[g] % page] = t[int(table[g * K, len(whole)]), : prefix[g] % page]
    plan = zq.zoqat_op_cache_plan(ints(cached), ints([1] * B), page, n_pages, ints(order), ints([len(order)]), table, B)
    assert int(plan["status"]) == 0
    tokens = ints(rng.integers(0, shape["vocab"], B).tolist())
    groups = (ints([0, K, B]), ints(prefix), ints([0] * K + [1] * K))

    def step(groups, table):
        mine = [(k.clone(), v.clone()) for k, v in caches]
        if groups is None:
            got = model.zoqat_decode_tree_step(tokens, plan, table, mine)
        else:
            got = model.zoqat_decode_prefix_step(tokens, plan, table, *groups, mine)
        model.zoqat_check()
        return got

    want, best = step(None, table)
    got, choice = step(groups, table)
    # The attentions of the two differ by a few roundings (of their weights with 16-bit caches); behind them an activation may come out one code further, which moves
    # logits by up to 2 % of their scale (5 % with bf16 keys), as in the test of drafts.
    tol = {"f32": 2e-2, "f16": 2e-2, "bf16": 5e-2}[dtype] * float(want.abs().max())
    assert float((got - want).abs().max()) <= tol
    top = want.topk(2, 1).values
    clear = top[:, 0] - top[:, 1] > 2 * tol
    assert torch.equal(choice[clear], best[clear])
    # the control: the second half of the shared tile of 128 keys names the pages of the first
    other = table.clone()
    other[:, 4:8] = table[:, 0:4]
    wrong, _ = step(groups, other)
    for g, n in enumerate(prefix):
        if n >= 128:
            assert float((wrong - want)[g * K: g * K + K].abs().max()) > 2 * tol
