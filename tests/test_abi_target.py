"""C-ABI checks of the target-side calls that need no GPU: the argument structs' layouts, and the refusal of
invalid arguments before anything is launched."""
import ctypes

import pytest

from paper_2609_21858_gb300 import pps

P = 256  # an aligned address that is never dereferenced: every call below fails validation, or has nothing to do


def _append(n=0, size=None, dtype=pps.BF16, heads=4, kv=2, d=64, rot=64, max_pos=10, eps=1e-6, q=P, slot=P, pos=P, rope=P,
            pages=3, page=16, strides=(2048, 128, 64), k=P, q_strides=(256, 64)):
    view = (P,) + q_strides
    s = pps._APPEND_ARGS
    return pps.lib().pps_kv_append(s.pack(s.size if size is None else size, q, *q_strides, *view, *view, *view, k, P, pages,
                                          page, kv, d, *strides, 0, 0, rope, pos, slot, 0, n, max_pos, dtype, heads, rot, 0,
                                          eps), None)


def _attention(n=0, size=None, dtype=pps.BF16, heads=4, kv=2, d=64, page=16, n_seq=2, columns=3, table=P, stride=3, ws=P,
               ws_bytes=1 << 40, scale=0.125, mask=0, words=0, q=P, q_strides=(256, 64), strides=(2048, 128, 64), k=P,
               lens=P):
    s = pps._ATTENTION_ARGS
    return pps.lib().pps_paged_attention(s.pack(s.size if size is None else size, q, *q_strides, P, 256, 64, k, P, 3, page,
                                                kv, d, *strides, table, lens, P, mask, 0, 0, ws, ws_bytes, n, stride, dtype,
                                                heads, columns, n_seq, words, scale), None)


def _chain(n=0, size=None, dtype=pps.BF16, n_draft=0, V=100, strides=(100, 100, 100), n_seq=0, gamma=3, T=1.0, p=P, q=P,
           noise=P, ws=P, ws_bytes=1 << 40):
    s = pps._CHAIN_ARGS
    return pps.lib().pps_verify_chain(s.pack(s.size if size is None else size, p, q, P, P, P, P, noise, P, P, P, 0, 0, ws,
                                             ws_bytes, n, n_draft, V, *strides, dtype, n_seq, gamma, T), None)


def test_struct_sizes_agree_and_empty_calls_succeed():
    # the library compares the size it is given with its own sizeof
    for call in (_append, _attention, _chain):
        assert call() == pps.OK
        assert call(size=0) == pps.ERR_INVALID_ARG
        assert call(size=8 + pps._APPEND_ARGS.size) == pps.ERR_INVALID_ARG
    for fn in (pps.lib().pps_kv_append, pps.lib().pps_paged_attention, pps.lib().pps_verify_chain):
        assert fn(None, None) == pps.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [dict(heads=0), dict(kv=0), dict(rot=7), dict(rot=66), dict(rot=-2), dict(max_pos=0),
                                 dict(rope=0), dict(eps=-1.0), dict(eps=float("nan")), dict(n=-1), dict(n=1, q=0),
                                 dict(n=1, slot=0), dict(n=1, pos=0), dict(pages=-1), dict(page=0), dict(k=0),
                                 dict(strides=(-1, 128, 64)), dict(n=5, q_strides=(2 ** 62, 64))])
def test_append_refuses(bad):
    assert _append(**bad) == pps.ERR_INVALID_ARG


def test_append_does_not_support():
    for bad in (dict(dtype=pps.F32), dict(dtype=9), dict(d=60), dict(d=264)):
        assert _append(**bad) == pps.ERR_UNSUPPORTED


@pytest.mark.parametrize("bad", [dict(heads=3), dict(heads=0), dict(kv=0), dict(n=-1), dict(n_seq=-1), dict(columns=-1),
                                 dict(stride=2), dict(scale=float("inf")), dict(mask=P, words=0), dict(words=-1),
                                 dict(k=264), dict(q=8), dict(n=2, q_strides=(260, 64)), dict(strides=(2048, 132, 64)),
                                 dict(n=1, q=0), dict(n=1, lens=0), dict(n=1, table=0), dict(columns=2 ** 28),
                                 dict(n=2 ** 30)])
def test_attention_refuses(bad):
    bad = {"stride": max(3, bad.get("columns", 3)), **bad}
    assert _attention(**bad) == pps.ERR_INVALID_ARG


def test_attention_does_not_support_and_needs_its_workspace():
    for bad in (dict(dtype=pps.F32), dict(d=136), dict(d=12), dict(page=12), dict(page=4)):
        assert _attention(**bad) == pps.ERR_UNSUPPORTED
    need = pps.lib().pps_attention_workspace_size(3, 4, 2, 64)
    for bad in (dict(ws=0), dict(ws_bytes=need - 1), dict(ws=264)):
        assert _attention(n=3, **bad) == pps.ERR_WORKSPACE
    assert need > 0 and pps.lib().pps_attention_workspace_size(-1, 4, 2, 64) == 0
    # the size is enough for any smaller call, too
    sizes = [pps.lib().pps_attention_workspace_size(n, 32, 8, 128) for n in (1, 2, 31, 32, 33, 64, 65, 1000, 100000)]
    assert sizes == sorted(sizes)


@pytest.mark.parametrize("bad", [dict(V=0), dict(strides=(99, 100, 100)), dict(strides=(100, 99, 100)),
                                 dict(strides=(100, 100, 99)), dict(T=0.0), dict(T=-1.0), dict(T=float("nan")),
                                 dict(gamma=-1), dict(gamma=65), dict(n=-1), dict(n_seq=-1), dict(n_seq=1),
                                 dict(n=1, n_seq=2), dict(n=2, n_seq=1, p=0), dict(n=2, n_seq=1, noise=0),
                                 dict(n=2, n_seq=1, n_draft=1, q=0), dict(n_draft=-1)])
def test_chain_refuses(bad):
    assert _chain(**bad) == pps.ERR_INVALID_ARG


def test_chain_does_not_support_and_needs_its_workspace():
    for dtype in (pps.F16, 7):
        assert _chain(dtype=dtype) == pps.ERR_UNSUPPORTED
    need = pps.lib().pps_chain_workspace_size(2, 1, 1)
    for bad in (dict(ws=0), dict(ws_bytes=need - 1), dict(ws=264)):
        assert _chain(n=2, n_seq=1, n_draft=1, **bad) == pps.ERR_WORKSPACE


def test_the_race_calls_still_refuse_half_precision():
    L, ids, fake = pps.lib(), pps.RowIds(P, P, P), ctypes.c_void_p(P)
    assert L.pps_draft_list(fake, pps.F16, 4, 100, 100, ids, 1.0, 4, None, pps.DISTINCT, fake, None, fake, fake, None, None,
                            fake, 1 << 30, None) == pps.ERR_UNSUPPORTED
