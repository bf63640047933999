"""Host-side argument checks of the serving operators: everything here is refused before a launch (no device needed)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def zq():
    import __graft_entry__ as ge
    ge.build()
    from paper_2509_00031_b200 import binding
    binding.lib()
    return binding


A = 1 << 20          # an aligned address that is never read: every call below is refused


def cache(zq, **kw):
    c = zq.PagedCache(A, 2 * A, zq.TYPE_BF16, 8, 16, 2, 128, 0, 16 * 2 * 128, 2 * 128, 128)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def plan(zq, **kw):
    a = dict(cached=A, new=2 * A, batch=2, page=16, n_pages=8, free=3 * A, cap=8, n_free=4 * A, table=5 * A, max_pages=4, parents=None, rows=8, words=0,
             kv=6 * A, start=7 * A, req=8 * A, pos=9 * A, slot=10 * A, mask=None, n_out=11 * A, status=12 * A, stream=None)
    a.update(kw)
    return zq.lib().zoqat_op_cache_plan(*a.values())


@pytest.mark.parametrize("kw", [dict(cached=None), dict(new=None), dict(n_free=None), dict(table=None), dict(kv=None), dict(start=None), dict(req=None),
                                dict(pos=None), dict(slot=None), dict(n_out=None), dict(status=None), dict(free=None), dict(batch=0), dict(page=0),
                                dict(n_pages=0), dict(max_pages=0), dict(rows=0), dict(cap=-1), dict(words=1), dict(mask=A), dict(kv=A), dict(kv=2 * A),
                                dict(n_out=4 * A), dict(table=3 * A), dict(parents=8 * A), dict(parents=10 * A)])
def test_plan_refuses_bad_arguments(zq, kw):
    assert plan(zq, **kw) == zq.ERR_INVALID_ARG and zq.lib().zoqat_last_error()


@pytest.mark.parametrize("kw", [dict(batch=16385), dict(words=33, mask=A), dict(words=-1), dict(page=1 << 20, n_pages=1 << 12), dict(page=1 << 20, max_pages=1 << 12)])
def test_plan_refuses_what_is_not_built(zq, kw):
    assert plan(zq, **kw) == zq.ERR_UNSUPPORTED


def append(zq, c, **kw):
    a = dict(qkv=A, ld=1024, pos=2 * A, slot=3 * A, rows=4, heads=4, cos=4 * A, sin=5 * A, rope=64)
    b = dict(q=6 * A, q_stride=512, err=7 * A, stream=None)
    for d in (a, b):
        d.update({k: v for k, v in kw.items() if k in d})
    return zq.lib().zoqat_op_cache_append(*a.values(), ctypes.byref(c) if c is not None else None, *b.values())


@pytest.mark.parametrize("kw", [dict(qkv=None), dict(slot=None), dict(q=None), dict(err=None), dict(rows=-1), dict(heads=0), dict(cos=None), dict(pos=None),
                                dict(rope=0), dict(ld=1020), dict(ld=1025), dict(q_stride=511), dict(q_stride=516), dict(qkv=A + 4), dict(q=A + 2), dict(cos=A + 4)])
def test_append_refuses_bad_arguments(zq, kw):
    assert append(zq, cache(zq), **kw) == zq.ERR_INVALID_ARG


BAD_CACHES = [(dict(k=None), "INVALID_ARG"), (dict(v=None), "INVALID_ARG"), (dict(type=3), "INVALID_ARG"), (dict(n_pages=0), "INVALID_ARG"),
              (dict(page_size=-1), "INVALID_ARG"), (dict(n_kv_heads=0), "INVALID_ARG"), (dict(d_head=32), "UNSUPPORTED"), (dict(d_head=96), "UNSUPPORTED"),
              (dict(slot_stride=260), "INVALID_ARG"), (dict(slot_stride=0), "INVALID_ARG"), (dict(head_stride=64), "INVALID_ARG"), (dict(page_stride=-4096), "INVALID_ARG"),
              (dict(k=A + 8), "INVALID_ARG"), (dict(n_pages=1 << 28), "UNSUPPORTED")]


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_caches_are_checked(zq, kw, code):
    assert append(zq, cache(zq, **kw)) == getattr(zq, "ERR_" + code)
    assert attend(zq, cache(zq, **kw)) == getattr(zq, "ERR_" + code)


def attend(zq, c, **kw):
    a = dict(q=A, q_stride=512)
    b = dict(table=2 * A, max_pages=4, kv=3 * A, start=4 * A, mask=5 * A, words=1, batch=2, rows=4, heads=4, scale=0.1, out=6 * A, out_stride=512,
             scratch=7 * A, nbytes=64 << 20, err=8 * A, stream=None)
    for d in (a, b):
        d.update({k: v for k, v in kw.items() if k in d})
    return zq.lib().zoqat_op_tree_attention(*a.values(), ctypes.byref(c) if c is not None else None, *b.values())


def test_no_rows_are_nothing_to_do(zq):
    # an empty tensor's address is NULL
    assert append(zq, cache(zq), rows=0, qkv=None, pos=None, slot=None, q=None) == zq.OK
    assert attend(zq, cache(zq), rows=0, q=None, out=None, mask=None) == zq.OK
    assert attend(zq, cache(zq), rows=0, q=None, out=None, kv=None) == zq.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(q=None), dict(table=None), dict(kv=None), dict(start=None), dict(out=None), dict(scratch=None), dict(err=None), dict(batch=0),
                                dict(rows=-1), dict(heads=0), dict(heads=3), dict(max_pages=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")),
                                dict(scale=float("nan")), dict(mask=None), dict(words=0), dict(words=-1), dict(q_stride=500), dict(q_stride=515), dict(out_stride=516),
                                dict(q=A + 8), dict(out=A), dict(scratch=A + 16)])
def test_attention_refuses_bad_arguments(zq, kw):
    assert attend(zq, cache(zq), **kw) == zq.ERR_INVALID_ARG


def test_attention_refuses_what_is_not_built_and_small_scratch(zq):
    assert attend(zq, None) == zq.ERR_INVALID_ARG
    for page in (1, 4, 24, 48, 96, 192):
        assert attend(zq, cache(zq, page_size=page, page_stride=page * 256)) == zq.ERR_UNSUPPORTED
    assert attend(zq, cache(zq), nbytes=1 << 20) == zq.ERR_WORKSPACE_SMALL
    assert attend(zq, cache(zq), rows=1 << 30) == zq.ERR_UNSUPPORTED
    assert attend(zq, cache(zq, n_pages=1 << 10), max_pages=1 << 28) == zq.ERR_UNSUPPORTED
    n = ctypes.c_size_t()
    L = zq.lib()
    for t in (zq.TYPE_F32, zq.TYPE_BF16, zq.TYPE_F16):
        assert L.zoqat_op_tree_attention_scratch_bytes(t, 128, ctypes.byref(n)) == zq.OK and 0 < n.value < 64 << 20
    assert L.zoqat_op_tree_attention_scratch_bytes(3, 128, ctypes.byref(n)) == zq.ERR_INVALID_ARG
    assert L.zoqat_op_tree_attention_scratch_bytes(0, 96, ctypes.byref(n)) == zq.ERR_UNSUPPORTED
    assert L.zoqat_op_tree_attention_scratch_bytes(0, 64, None) == zq.ERR_INVALID_ARG


def test_attention_refuses_caches_that_tensor_maps_do_not_hold(zq):
    for kw in (dict(slot_stride=1 << 36, page_stride=1 << 37), dict(slot_stride=1 << 37, page_stride=1 << 37),
               dict(n_pages=1 << 20, page_stride=128 << 12), dict(n_pages=3, page_stride=128 << 30)):
        assert attend(zq, cache(zq, **kw)) == zq.ERR_UNSUPPORTED, kw
    # one page, or one key head: the strides of what is there once do not count
    assert attend(zq, cache(zq, n_pages=1, page_stride=1 << 37, slot_stride=1 << 36)) == zq.ERR_UNSUPPORTED
    assert attend(zq, cache(zq, n_pages=1 << 20, page_stride=128 << 12, type=zq.TYPE_F32), nbytes=1 << 10) == zq.ERR_WORKSPACE_SMALL
    assert attend(zq, cache(zq, n_pages=1 << 20, page_stride=128 << 12, n_kv_heads=1), nbytes=1 << 10) == zq.ERR_WORKSPACE_SMALL


def rules(zq, desc=None, **kw):
    a = dict(logits=A, type=0, ld=100, rows=4, vocab=100)
    b = dict(out=2 * A, out_ld=100, token=3 * A, stream=None)
    for d in (a, b):
        d.update({k: v for k, v in kw.items() if k in d})
    r = zq.LogitRulesDesc(batch=4)
    for k, v in (desc or {}).items():
        setattr(r, k, v)
    return zq.lib().zoqat_op_logit_rules(*a.values(), ctypes.byref(r), *b.values())


@pytest.mark.parametrize("kw,desc", [(dict(logits=None), {}), (dict(out=None, token=None), {}), (dict(type=5), {}), (dict(ld=99), {}), (dict(out_ld=99), {}),
                                     (dict(out=A, out_ld=128), {}), (dict(logits=A + 2), {}), ({}, dict(batch=0)), ({}, dict(batch=3)),
                                     ({}, dict(history=A)), ({}, dict(history=A, history_len=A)), ({}, dict(history=A, history_len=A, history_stride=(1 << 30) + 1)),
                                     ({}, dict(bias_token=A, bias_stride=4)),
                                     ({}, dict(bias_token=A, bias_value=A, bias_len=A)), ({}, dict(bias_token=A, bias_value=A, bias_len=A, bias_stride=(1 << 30) + 1)),
                                     ({}, dict(allowed=A, allowed_stride=3)),
                                     ({}, dict(draft_token=A)), ({}, dict(draft_token=A, row_start=A, tree_mask=A, mask_words=0))])
def test_rules_refuse_bad_arguments(zq, kw, desc):
    assert rules(zq, desc, **kw) == zq.ERR_INVALID_ARG


def test_rules_refuse_sizes_that_are_not_built(zq):
    for kw in (dict(rows=0), dict(rows=65536), dict(vocab=0), dict(vocab=(1 << 30) + 1)):
        assert rules(zq, dict(row_request=A), **kw) == zq.ERR_UNSUPPORTED
    assert zq.lib().zoqat_op_logit_rules(A, 0, 100, 4, 100, None, A, 100, A, None) == zq.ERR_INVALID_ARG


def test_a_launch_that_fails_names_the_cuda_error(zq):
    import torch
    if torch.cuda.is_available():
        pytest.skip("the calls would run")
    for call, who in ((lambda: plan(zq), b"cache plan: "), (lambda: attend(zq, cache(zq, type=zq.TYPE_F32)), b"tree attention: "), (lambda: rules(zq), b"logit rules: ")):
        assert call() == zq.ERR_CUDA
        text = zq.lib().zoqat_last_error()
        assert text.startswith(who) and len(text) > len(who) + 5, text
