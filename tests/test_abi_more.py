"""C-ABI checks, without a GPU, of the calls on a cache in 4 bits, of page tables and of logits: the argument structs' layouts, and
the refusal of invalid arguments before anything is launched."""
import pytest

from paper_2609_21858_gb300 import pps

P = 256  # an aligned address that is never dereferenced: every call below fails validation, or has nothing to do


def _cache(pages=3, page=16, kv=2, d=64, k=P, ks=P, strides=(1024, 64, 32), scale_strides=(128, 8, 4)):
    return (k, P, ks, P, 0, 0, pages, page, kv, d, *strides, *scale_strides)


CACHE = {"pages", "page", "kv", "d", "k", "ks", "strides", "scale_strides"}


def _split(kw):
    return {k: v for k, v in kw.items() if k in CACHE}, {k: v for k, v in kw.items() if k not in CACHE}


def _append(**kw):
    c, kw = _split(kw)

    def call(n=0, size=None, dtype=pps.BF16, heads=4, rot=64, max_pos=10, eps=1e-6, q=P, slot=P, pos=P, rope=P, q_strides=(256, 64)):
        s, view = pps._APPEND_Q4_ARGS, (P,) + q_strides
        return pps.lib().pps_kv_append_q4(s.pack(s.size if size is None else size, q, *q_strides, *view, *view, *view, *_cache(**c), 0,
                                                 0, rope, pos, slot, 0, n, max_pos, dtype, heads, rot, 0, eps), None)
    return call(**kw)


def _read(**kw):
    c, kw = _split(kw)

    def call(n=0, size=None, dtype=pps.BF16, out=P, slot=P, out_strides=(128, 64)):
        s = pps._READ_Q4_ARGS
        return pps.lib().pps_kv_read_q4(s.pack(s.size if size is None else size, out, *out_strides, P, *out_strides, *_cache(**c), slot,
                                               0, n, dtype), None)
    return call(**kw)


def _attention(**kw):
    c, kw = _split(kw)

    def call(n=0, size=None, dtype=pps.BF16, heads=4, n_seq=2, columns=3, table=P, stride=3, ws=P, ws_bytes=1 << 40, scale=0.125, mask=0,
             words=0, q=P, q_strides=(256, 64), lens=P):
        s = pps._ATTENTION_Q4_ARGS
        return pps.lib().pps_paged_attention_q4(s.pack(s.size if size is None else size, q, *q_strides, P, 256, 64, *_cache(**c), table,
                                                       lens, P, mask, 0, 0, ws, ws_bytes, n, stride, dtype, heads, columns, n_seq,
                                                       words, scale), None)
    return call(**kw)


def _reserve(size=None, n_tok=0, n_seq=0, columns=3, stride=3, page=16, cap=5, pages=P, held=P, free_list=P, count=P, lens=P, new=P,
             q_off=P, out_len=P, slot=P, pos=P):
    s = pps._RESERVE_ARGS
    return pps.lib().pps_kv_reserve(s.pack(s.size if size is None else size, pages, held, free_list, count, lens, new, 0, q_off, out_len,
                                           slot, pos, 0, 0, n_tok, stride, n_seq, columns, page, cap), None)


def _trim(size=None, n_seq=0, columns=3, stride=3, page=16, cap=5, pages=P, held=P, free_list=P, count=P, keep=P):
    s = pps._TRIM_ARGS
    return pps.lib().pps_kv_trim(s.pack(s.size if size is None else size, pages, held, free_list, count, keep, 0, stride, n_seq, columns,
                                        page, cap), None)


def _adjust(size=None, n=0, V=100, dtype=pps.BF16, n_seq=0, x=P, out=P + 2048, off=P, text=0, lens=0, prompt=0, node_tok=0, mask=0,
            rep=0, bias_off=0, bias_tok=0, bias_val=0, allowed=0, in_stride=100, out_stride=100, text_stride=0, allowed_stride=0,
            cap=0, words=0, n_bias=0):
    s = pps._ADJUST_ARGS
    return pps.lib().pps_adjust_logits(s.pack(s.size if size is None else size, x, out, off, text, lens, prompt, node_tok, mask, rep, 0, 0,
                                              bias_off, bias_tok, bias_val, allowed, 0, n, V, in_stride, out_stride, text_stride,
                                              allowed_stride, dtype, n_seq, cap, words, n_bias), None)


def test_struct_sizes_agree_and_empty_calls_succeed():
    for call in (_append, _read, _attention, _trim, _adjust):
        assert call() == pps.OK
    for call, s in ((_append, pps._APPEND_Q4_ARGS), (_read, pps._READ_Q4_ARGS), (_attention, pps._ATTENTION_Q4_ARGS),
                    (_reserve, pps._RESERVE_ARGS), (_trim, pps._TRIM_ARGS), (_adjust, pps._ADJUST_ARGS)):
        assert call(size=0) == pps.ERR_INVALID_ARG and call(size=s.size + 8) == pps.ERR_INVALID_ARG
    for name in ("kv_append_q4", "kv_read_q4", "paged_attention_q4", "kv_reserve", "kv_trim", "adjust_logits"):
        assert getattr(pps.lib(), "pps_" + name)(None, None) == pps.ERR_INVALID_ARG


CACHE_BAD = [dict(pages=-1), dict(page=0), dict(kv=0), dict(k=0), dict(ks=0), dict(strides=(-8, 64, 32)), dict(strides=(1024, 68, 32)),
             dict(strides=(1024, 64, 36)), dict(scale_strides=(128, 6, 4)), dict(scale_strides=(126, 8, 4)), dict(k=260), dict(ks=258),
             dict(strides=(2 ** 62, 64, 32)), dict(scale_strides=(2 ** 62, 8, 4))]


@pytest.mark.parametrize("bad", CACHE_BAD)
def test_caches_that_are_refused(bad):
    for call in (_append, _read, _attention):
        assert call(**bad) == pps.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [dict(heads=0), dict(rot=7), dict(rot=66), dict(rot=-2), dict(max_pos=0), dict(rope=0), dict(eps=-1.0),
                                 dict(eps=float("nan")), dict(n=-1), dict(n=1, q=0), dict(n=1, slot=0), dict(n=1, pos=0),
                                 dict(n=5, q_strides=(2 ** 62, 64))])
def test_append_refuses(bad):
    assert _append(**bad) == pps.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [dict(n=-1), dict(n=1, out=0), dict(n=1, slot=0), dict(out=264), dict(out_strides=(128, 60)),
                                 dict(n=3, out_strides=(124, 64))])
def test_read_refuses(bad):
    assert _read(**bad) == pps.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [dict(heads=3), dict(heads=0), dict(n=-1), dict(n_seq=-1), dict(columns=-1), dict(stride=2),
                                 dict(scale=float("inf")), dict(mask=P, words=0), dict(words=-1), dict(q=8),
                                 dict(n=2, q_strides=(260, 64)), dict(n=1, q=0), dict(n=1, lens=0), dict(n=1, table=0),
                                 dict(columns=2 ** 28), dict(n=2 ** 30)])
def test_attention_refuses(bad):
    assert _attention(**{"stride": max(3, bad.get("columns", 3)), **bad}) == pps.ERR_INVALID_ARG


def test_what_is_not_supported_and_workspaces():
    for call in (_append, _read, _attention):
        for bad in (dict(dtype=pps.F32), dict(dtype=9), dict(d=24), dict(d=272), dict(d=8)):
            assert call(**bad) == pps.ERR_UNSUPPORTED
    for bad in (dict(d=144), dict(page=12), dict(page=4)):
        assert _attention(**bad) == pps.ERR_UNSUPPORTED
    size = pps.lib().pps_attention_q4_workspace_size
    for n in (3, 300):
        for bad in (dict(ws=0), dict(ws_bytes=size(n, 4, 2, 64) - 1), dict(ws=264)):
            assert _attention(n=n, **bad) == pps.ERR_WORKSPACE
    assert size(3, 4, 2, 64) > 0 and size(-1, 4, 2, 64) == 0
    # the size is enough for any smaller call, too
    sizes = [size(n, 32, 8, 128) for n in (1, 2, 3, 4, 5, 31, 32, 33, 64, 65, 1000, 100000)]
    assert sizes == sorted(sizes)


@pytest.mark.parametrize("bad", [dict(n_tok=-1), dict(n_seq=-1), dict(columns=-1), dict(stride=2), dict(page=0), dict(cap=-1), dict(count=0),
                                 dict(q_off=0), dict(free_list=0), dict(n_tok=1, slot=0), dict(n_tok=1, pos=0), dict(n_seq=1, held=0),
                                 dict(n_seq=1, lens=0), dict(n_seq=1, new=0), dict(n_seq=1, out_len=0), dict(n_seq=1, pages=0),
                                 dict(n_seq=9, stride=2 ** 62)])
def test_reserve_refuses(bad):
    assert _reserve(**bad) == pps.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [dict(n_seq=-1), dict(columns=-1), dict(stride=2), dict(page=0), dict(cap=-1), dict(n_seq=1, count=0),
                                 dict(n_seq=1, held=0), dict(n_seq=1, keep=0), dict(n_seq=1, pages=0), dict(n_seq=1, free_list=0)])
def test_trim_refuses(bad):
    assert _trim(**bad) == pps.ERR_INVALID_ARG


def test_too_many_sequences_for_page_tables():
    assert _reserve(n_seq=8193) == pps.ERR_UNSUPPORTED and _trim(n_seq=8193) == pps.ERR_UNSUPPORTED


@pytest.mark.parametrize("bad", [dict(n=-1), dict(V=0), dict(n_seq=-1), dict(in_stride=99), dict(out_stride=99), dict(cap=-1), dict(words=-1),
                                 dict(n_bias=-1), dict(x=P + 1), dict(out=P + 1), dict(text=P), dict(text=P, lens=P, cap=4, text_stride=3),
                                 dict(mask=P, words=1), dict(mask=P, node_tok=P), dict(rep=P), dict(bias_off=P, n_bias=2),
                                 dict(allowed=P, allowed_stride=3), dict(n=2, n_seq=1, x=0), dict(n=2, n_seq=1, out=0),
                                 dict(n=2, n_seq=1, off=0), dict(n=2, n_seq=1, out=P, out_stride=101), dict(n=9, in_stride=2 ** 62)])
def test_adjust_refuses(bad):
    assert _adjust(**bad) == pps.ERR_INVALID_ARG


def test_adjust_does_not_support():
    for dtype in (pps.F16, 7):
        assert _adjust(dtype=dtype) == pps.ERR_UNSUPPORTED
