"""Host-side argument checks of the operators for many continuations of one prompt: everything here is refused before a launch (no device needed)."""
import ctypes
import math

import pytest

from test_serve_abi import A, BAD_CACHES, cache, zq  # noqa: F401


# ---- rotary frequencies ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rot,base", [(128, 10000.0), (64, 500000.0), (16, 100.0)])
def test_frequencies_are_the_formulas(zq, rot, base):  # noqa: F811
    plain, one = zq.rotary_frequencies(rot, base, device="cpu")
    want = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    close = lambda a, b: all(abs(x - y) <= 1e-14 * abs(y) for x, y in zip(a.tolist(), b))  # noqa: E731
    assert close(plain, want) and one == 1.0
    linear, one = zq.rotary_frequencies(rot, base, zq.ROTARY_LINEAR, 4.0, device="cpu")
    assert close(linear, [x / 4.0 for x in want]) and one == 1.0
    based, one = zq.rotary_frequencies(rot, base, zq.ROTARY_BASE, 8.0, device="cpu")
    assert abs(float(based[-1]) * 8.0 / want[-1] - 1.0) < 1e-12 and float(based[0]) == 1.0 and one == 1.0
    parts, m = zq.rotary_frequencies(rot, base, zq.ROTARY_PARTS, 16.0, 4096, device="cpu")
    assert abs(m - (0.1 * math.log(16.0) + 1.0)) < 1e-6
    for f, x in zip(want, parts.tolist()):
        r = 4096 * f / (2 * math.pi)
        keep = min(1.0, max(0.0, (r - 1.0) / 31.0))
        assert abs(x - (f * keep + f / 16.0 * (1.0 - keep))) <= 1e-13 * f
    assert torch_equal(zq.rotary_frequencies(rot, base, zq.ROTARY_PARTS, 1.0, 4096, device="cpu")[0], plain)


def torch_equal(a, b):
    return bool(((a - b).abs() <= 1e-15 * b.abs()).all())


@pytest.mark.parametrize("args", [(0, 10000.0, 0, 1.0, 0), (7, 10000.0, 0, 1.0, 0), (-2, 10000.0, 0, 1.0, 0), (8, 1.0, 0, 1.0, 0), (8, float("nan"), 0, 1.0, 0),
                                  (8, float("inf"), 0, 1.0, 0), (8, 1e4, 4, 1.0, 0), (8, 1e4, -1, 1.0, 0), (8, 1e4, 1, 0.5, 0), (8, 1e4, 1, float("nan"), 0),
                                  (8, 1e4, 3, 2.0, 0), (2, 1e4, 2, 2.0, 0), (1 << 20, 1e4, 0, 1.0, 0)])
def test_frequencies_refuse_bad_arguments(zq, args):  # noqa: F811
    rot, base, kind, factor, trained = args
    buf, mag = (ctypes.c_double * 64)(), ctypes.c_float()
    assert zq.lib().zoqat_rotary_frequencies(rot, base, kind, factor, trained, buf, ctypes.byref(mag)) == zq.ERR_INVALID_ARG
    assert zq.lib().zoqat_rotary_frequencies(8, 1e4, 0, 1.0, 0, None, ctypes.byref(mag)) == zq.ERR_INVALID_ARG


# ---- rotary append --------------------------------------------------------------------------------------------------
def append(zq, c, **kw):  # noqa: F811
    a = dict(qkv=A, type=0, ld=1024, pos=2 * A, slot=3 * A, rows=4, heads=4, freq=4 * A, rot=64, inter=0, mag=1.0, qg=5 * A, kg=6 * A, eps=1e-6)
    b = dict(q=7 * A, q_stride=512, err=8 * A, stream=None)
    for d in (a, b):
        d.update({k: v for k, v in kw.items() if k in d})
    return zq.lib().zoqat_op_rotary_append(*a.values(), ctypes.byref(c) if c is not None else None, *b.values())


@pytest.mark.parametrize("kw", [dict(qkv=None), dict(slot=None), dict(q=None), dict(err=None), dict(type=3), dict(rows=-1), dict(heads=0), dict(heads=1 << 17), dict(freq=None),
                                dict(rot=0), dict(pos=None), dict(mag=float("nan")), dict(eps=-1.0), dict(eps=float("inf")), dict(ld=1020), dict(ld=1026), dict(q_stride=511),
                                dict(q_stride=516), dict(qkv=A + 4), dict(q=A + 2), dict(qg=A + 4), dict(kg=A + 8), dict(freq=A + 4), dict(q=A)])
def test_append_refuses_bad_arguments(zq, kw):  # noqa: F811
    assert append(zq, cache(zq), **kw) == zq.ERR_INVALID_ARG and zq.lib().zoqat_last_error()


@pytest.mark.parametrize("rot", [-16, 8, 24, 144])
def test_append_refuses_rotations_that_are_not_built(zq, rot):  # noqa: F811
    assert append(zq, cache(zq), rot=rot) == zq.ERR_UNSUPPORTED


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_caches_are_checked(zq, kw, code):  # noqa: F811
    want = getattr(zq, "ERR_" + code)
    bad = cache(zq, **kw)
    assert append(zq, bad) == want and attend(zq, bad) == want
    assert zq.lib().zoqat_op_cache_copy(ctypes.byref(bad), 1, A, 2 * A, 3 * A, 4, 4 * A, None) == want
    both = (zq.PagedCache * 2)(cache(zq), bad)
    assert zq.lib().zoqat_op_cache_copy(both, 2, A, 2 * A, 3 * A, 4, 4 * A, None) == want


def test_nothing_to_do(zq):  # noqa: F811
    assert append(zq, cache(zq), rows=0, qkv=None, pos=None, slot=None, q=None) == zq.OK
    assert attend(zq, cache(zq), rows=0, q=None, out=None, mask=None) == zq.OK
    assert zq.lib().zoqat_op_cache_copy(ctypes.byref(cache(zq)), 1, None, None, None, 0, 4 * A, None) == zq.OK
    assert append(zq, cache(zq), qg=None, kg=None, eps=-1.0, rows=0) == zq.OK


# ---- shared prefixes ------------------------------------------------------------------------------------------------
def attend(zq, c, **kw):  # noqa: F811
    a = dict(q=A, q_stride=512)
    b = dict(table=2 * A, max_pages=4, kv=3 * A, start=4 * A, gs=9 * A, plen=10 * A, rg=11 * A, groups=2, mask=5 * A, words=1, batch=2, rows=4, heads=4, scale=0.1,
             out=6 * A, out_stride=512, scratch=7 * A, nbytes=256 << 20, err=8 * A, stream=None)
    for d in (a, b):
        d.update({k: v for k, v in kw.items() if k in d})
    return zq.lib().zoqat_op_prefix_attention(*a.values(), ctypes.byref(c) if c is not None else None, *b.values())


@pytest.mark.parametrize("kw", [dict(q=None), dict(table=None), dict(kv=None), dict(start=None), dict(out=None), dict(scratch=None), dict(err=None), dict(batch=0),
                                dict(rows=-1), dict(heads=0), dict(heads=3), dict(max_pages=0), dict(scale=0.0), dict(scale=float("nan")), dict(mask=None), dict(words=0),
                                dict(q_stride=500), dict(out_stride=516), dict(q=A + 8), dict(out=A), dict(scratch=A + 16), dict(gs=None), dict(plen=None), dict(rg=None),
                                dict(groups=0), dict(groups=-3)])
def test_prefix_attention_refuses_bad_arguments(zq, kw):  # noqa: F811
    assert attend(zq, cache(zq), **kw) == zq.ERR_INVALID_ARG


def test_prefix_attention_refuses_what_is_not_built_and_small_scratch(zq):  # noqa: F811
    for page in (1, 4, 24, 96, 192):
        assert attend(zq, cache(zq, page_size=page, page_stride=page * 256)) == zq.ERR_UNSUPPORTED
    assert attend(zq, cache(zq), groups=(1 << 31) - 1) == zq.ERR_UNSUPPORTED
    assert attend(zq, cache(zq), nbytes=1 << 20) == zq.ERR_WORKSPACE_SMALL
    n, L = ctypes.c_size_t(), zq.lib()
    last = 0
    for rows in (0, 1, 100, 5000):
        for t in (zq.TYPE_F32, zq.TYPE_BF16, zq.TYPE_F16):
            assert L.zoqat_op_prefix_attention_scratch_bytes(t, 128, rows, 32, ctypes.byref(n)) == zq.OK and 0 < n.value
        assert n.value >= last
        last = n.value
    assert attend(zq, cache(zq), rows=5000, heads=32, q_stride=4096, out_stride=4096, nbytes=last - 1) == zq.ERR_WORKSPACE_SMALL
    assert L.zoqat_op_prefix_attention_scratch_bytes(3, 128, 4, 4, ctypes.byref(n)) == zq.ERR_INVALID_ARG
    assert L.zoqat_op_prefix_attention_scratch_bytes(0, 128, -1, 4, ctypes.byref(n)) == zq.ERR_INVALID_ARG
    assert L.zoqat_op_prefix_attention_scratch_bytes(0, 96, 4, 4, ctypes.byref(n)) == zq.ERR_UNSUPPORTED
    assert L.zoqat_op_prefix_attention_scratch_bytes(0, 64, 1 << 30, 4, ctypes.byref(n)) == zq.ERR_UNSUPPORTED
    assert L.zoqat_op_prefix_attention_scratch_bytes(0, 64, 4, 4, None) == zq.ERR_INVALID_ARG


# ---- beams ----------------------------------------------------------------------------------------------------------
def select(zq, **kw):  # noqa: F811
    a = dict(logits=A, type=0, ld=100, batch=2, beams=4, vocab=100, score=2 * A, eos=3 * A, n_eos=1, beam=4 * A, token=5 * A, out=6 * A, db=7 * A, dt=8 * A, ds=9 * A, stream=None)
    a.update(kw)
    return zq.lib().zoqat_op_beam_select(*a.values())


@pytest.mark.parametrize("kw", [dict(logits=None), dict(score=None), dict(beam=None), dict(token=None), dict(out=None), dict(db=None), dict(dt=None), dict(ds=None), dict(type=4),
                                dict(batch=0), dict(beams=0), dict(vocab=0), dict(n_eos=-1), dict(eos=None), dict(n_eos=0), dict(ld=99), dict(logits=A + 2), dict(out=2 * A), dict(ds=2 * A)])
def test_select_refuses_bad_arguments(zq, kw):  # noqa: F811
    assert select(zq, **kw) == zq.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(beams=33), dict(batch=(1 << 24) + 1), dict(vocab=(1 << 30) + 1, ld=1 << 31), dict(n_eos=8)])
def test_select_refuses_what_is_not_built(zq, kw):  # noqa: F811
    assert select(zq, **kw) == zq.ERR_UNSUPPORTED


def reorder(zq, scratch=40 * A, nbytes=1 << 20, **kw):  # noqa: F811
    names = [n for n, t in zq.BeamReorder._fields_ if t is ctypes.c_void_p]
    d = {n: (i + 1) * A for i, n in enumerate(names)}
    d.update(history_stride=50, batch=2, beams=4, page_size=16, n_pages=64, max_pages=8, free_capacity=64)
    d.update(kw)
    r = zq.BeamReorder(**d)
    return zq.lib().zoqat_op_beam_reorder(ctypes.byref(r), scratch, nbytes, None)


@pytest.mark.parametrize("kw", [{n: None} for n in ("parent", "kv_len", "block_table", "free_pages", "n_free", "block_table_out", "kv_len_out", "free_pages_out", "n_free_out",
                                                    "copy_from", "copy_to", "copy_len", "status", "history_len", "history_out", "history_len_out", "history")] +
                         [dict(batch=0), dict(beams=0), dict(page_size=0), dict(n_pages=0), dict(max_pages=0), dict(free_capacity=0), dict(history_stride=0),
                          dict(history_stride=(1 << 30) + 1), dict(block_table_out=3 * A), dict(kv_len_out=2 * A), dict(free_pages_out=5 * A), dict(n_free_out=6 * A),
                          dict(history_out=7 * A), dict(copy_to=1 * A), dict(scratch=None), dict(scratch=40 * A + 4)])
def test_reorder_refuses_bad_arguments(zq, kw):  # noqa: F811
    assert reorder(zq, **kw) == zq.ERR_INVALID_ARG and zq.lib().zoqat_last_error()


def test_reorder_refuses_what_is_not_built_and_small_scratch(zq):  # noqa: F811
    for kw in (dict(batch=16385), dict(beams=33), dict(page_size=1 << 20, n_pages=1 << 12), dict(page_size=1 << 20, max_pages=1 << 12)):
        assert reorder(zq, **kw) == zq.ERR_UNSUPPORTED
    assert reorder(zq, nbytes=8) == zq.ERR_WORKSPACE_SMALL
    n = ctypes.c_size_t()
    assert zq.lib().zoqat_op_beam_reorder_scratch_bytes(16384, ctypes.byref(n)) == zq.OK and n.value >= 16384 * 8
    for batch in (0, -1, 16385):
        assert zq.lib().zoqat_op_beam_reorder_scratch_bytes(batch, ctypes.byref(n)) == zq.ERR_INVALID_ARG
    assert zq.lib().zoqat_op_beam_reorder_scratch_bytes(4, None) == zq.ERR_INVALID_ARG
    assert zq.lib().zoqat_op_beam_reorder(None, 40 * A, 1 << 20, None) == zq.ERR_INVALID_ARG


def test_copies_refuse_bad_arguments(zq):  # noqa: F811
    c = cache(zq)
    call = lambda *a: zq.lib().zoqat_op_cache_copy(*a, None)  # noqa: E731
    for a in ((None, 1, A, A, A, 4, A), (ctypes.byref(c), 1, None, A, A, 4, A), (ctypes.byref(c), 1, A, None, A, 4, A), (ctypes.byref(c), 1, A, A, None, 4, A),
              (ctypes.byref(c), 1, A, A, A, 4, None), (ctypes.byref(c), 0, A, A, A, 4, A), (ctypes.byref(c), 1, A, A, A, -1, A)):
        assert call(*a) == zq.ERR_INVALID_ARG
    assert call(ctypes.byref(c), 4097, A, A, A, 4, A) == zq.ERR_UNSUPPORTED


def test_a_prefix_step_needs_groups(zq):  # noqa: F811
    assert zq.lib().zoqat_decode_prefix_step(None, A, 4, None, None, None, None, None, None, A, 1 << 20, None) == zq.ERR_INVALID_ARG


def test_a_launch_that_fails_names_the_cuda_error(zq):  # noqa: F811
    import torch
    if torch.cuda.is_available():
        pytest.skip("the calls would run")
    for call, who in ((lambda: append(zq, cache(zq)), b"rotary append: "), (lambda: attend(zq, cache(zq, type=zq.TYPE_F32)), b"prefix attention: "),
                      (lambda: select(zq), b"beam select: "), (lambda: reorder(zq), b"beam reorder: "),
                      (lambda: zq.lib().zoqat_op_cache_copy(ctypes.byref(cache(zq)), 1, A, 2 * A, 3 * A, 4, 4 * A, None), b"cache copy: ")):
        assert call() == zq.ERR_CUDA
        text = zq.lib().zoqat_last_error()
        assert text.startswith(who) and len(text) > len(who) + 5, text
