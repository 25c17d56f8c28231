"""Trees of drafted tokens and moved tokens without a GPU: the oracle's own rules, and what the calls refuse before anything is launched."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import pace_oracle as O
from paper_2608_27206_gb300 import pace as P
from test_kv_cpu import BAD_CACHE, FALLING, LATE, call  # noqa: F401

A = 1 << 20     # an address that is never followed
INVALID = P.PACE_ERR_INVALID_ARG


# ---- the oracle ------------------------------------------------------------------------------
@pytest.mark.parametrize("window,sinks", [(0, 0), (3, 0), (4, 2), (1, 0), (50, 7)])
def test_a_line_of_nodes_sees_what_queries_in_a_line_see(window, sinks):
    np.testing.assert_array_equal(O.kv_tree_visible(20, list(range(-1, 6)), window, sinks), O.kv_visible(20, 7, window, sinks))


def test_visibility_of_a_tree():
    parents = [-1, 0, 0, 1, 2, -1]
    see = O.kv_tree_visible(8, parents)
    assert [np.nonzero(r)[0].tolist() for r in see] == [[0, 1, 2], [0, 1, 2, 3], [0, 1, 2, 4], [0, 1, 2, 3, 5], [0, 1, 2, 4, 6], [0, 1, 7]]
    # a node's window is the one that the path to it would have as the sequence's end
    see = O.kv_tree_visible(8, parents, window=3, sinks=1)
    assert [np.nonzero(r)[0].tolist() for r in see] == [[0, 1, 2], [0, 1, 2, 3], [0, 1, 2, 4], [0, 2, 3, 5], [0, 2, 4, 6], [0, 1, 7]]
    assert not O.kv_tree_visible(2, [-1, 0, 1])[0].any()      # a node before the first slot


@pytest.mark.parametrize("scale", [0.2, 1e4])
def test_attention_by_matrices_is_attention_row_by_row(scale):
    rng = np.random.default_rng(3)
    Q, K, V = rng.normal(size=(9, 6, 16)), rng.normal(size=(40, 2, 16)), rng.normal(size=(40, 2, 16))
    see = O.kv_tree_visible(40, [-1, 0, 0, 1, 2, -1, 5, 3, 1], window=11, sinks=3)
    see[4] = False
    a, b = O.kv_attention(Q, K, V, see, scale), O.kv_attention_dense(Q, K, V, see, scale)
    for n in a:
        np.testing.assert_allclose(b[n], a[n], rtol=1e-11, atol=1e-300)


def test_walk():
    tokens, parents = [5, 7, 8, 7, 9, 9], [-1, 0, 0, 0, 2, 2]
    assert O.draft_accept(tokens, parents, [8, 0, 9, 0, 1, 1]) == [0, 2, 4]
    assert O.draft_accept(tokens, parents, [7, 9, 0, 0, 0, 0]) == [0, 1]
    assert O.draft_accept(tokens, parents, [3, 0, 0, 0, 0, 0]) == [0]
    assert O.draft_accept([], [], []) == []


def test_moved_tokens_keep_their_values_to_half_a_step():
    rng = np.random.default_rng(1)
    values = O.e4m3_round(rng.normal(0, 60, (6, 2, 32, 64)))
    scales = 2.0 ** rng.integers(-3, 4, (6, 2, 2)).astype(float)
    was = O.kv_read(values, scales, [4, 1, 3], 90)
    kept = np.sort(rng.permutation(69)[:30])
    O.kv_compact(values, scales, [4, 1, 3], [4, 1, 3], 21, kept)
    now = O.kv_read(values, scales, [4, 1, 3], 51)
    want = np.concatenate([was[:21], was[21 + kept]])
    np.testing.assert_array_equal(now[:16], want[:16])
    step = np.repeat(np.stack([scales[p, :, i] for p, i in ((4, 1), (1, 0), (1, 1))]), 16, axis=0)[:35, :, None] * 2.0 ** -10
    assert np.all(np.abs(now - want)[16:] <= np.maximum(np.abs(want)[16:] * 2.0 ** -4, step))
    # each touched block: the smallest power that covers it
    for i, (p, s) in enumerate(((4, 1), (1, 0), (1, 1))):
        np.testing.assert_array_equal(scales[p, :, s], O.kv_scale(np.abs(want[16 * i + 16:16 * i + 32]).max(axis=(0, 2))))


# ---- refusals: before the device is looked at ------------------------------------------------
CU = (ctypes.c_int32 * 3)(0, 2, 3)
MANY = (ctypes.c_int32 * 3)(0, 2, 2 + P.TREE_MAX + 1)
FULL = (ctypes.c_int32 * 3)(0, 2, 2 + P.TREE_MAX)
MORE = (ctypes.c_int32 * 3)(0, 3, 3)


def attend(call, c=None, **kw):  # noqa: F811
    f = dict(Q=A, qs=28 * 128, cu=ctypes.addressof(CU), B=2, hq=28, parents=A, lens=A, table=A, ts=4, max_len=256, scale=0.1, window=0, sinks=0,
             out=A, lse=None, ws=A, ws_bytes=1 << 40)
    f.update(kw)
    c = c or call.cache()
    return call.L.pace_kv_tree_attention(ctypes.addressof(c), f["Q"], f["qs"], f["cu"], f["B"], f["hq"], f["parents"], f["lens"], f["table"],
                                         f["ts"], f["max_len"], f["scale"], f["window"], f["sinks"], f["out"], f["lse"], f["ws"],
                                         f["ws_bytes"], None)


@pytest.mark.parametrize("bad", [dict(B=-1), dict(Q=None), dict(Q=A + 8), dict(qs=28 * 128 - 8), dict(cu=None), dict(cu=ctypes.addressof(FALLING)),
                                 dict(cu=ctypes.addressof(MANY)), dict(hq=0), dict(hq=30), dict(parents=None), dict(parents=A + 2), dict(lens=None),
                                 dict(table=None), dict(ts=0), dict(max_len=-1), dict(max_len=257), dict(scale=0.0), dict(scale=float("inf")),
                                 dict(sinks=-1), dict(out=None), dict(out=A + 2)])
def test_tree_attention_refuses(call, bad):  # noqa: F811
    assert attend(call, **bad) == INVALID


@pytest.mark.parametrize("bad", BAD_CACHE)
def test_the_calls_refuse_a_bad_cache(call, bad):  # noqa: F811
    assert attend(call, c=call.cache(**bad)) == INVALID
    assert compact(call, c=[call.cache(), call.cache(**bad)]) == INVALID


def test_tree_attention_workspace(call):  # noqa: F811
    def size(cu, hq=28, c=call.cache()):
        return call.L.pace_kv_tree_attention_workspace_size(ctypes.addressof(c), ctypes.addressof(cu), 2, hq, 256)
    need = size(CU)
    assert need >= call.L.pace_kv_attention_workspace_size(ctypes.addressof(call.cache()), ctypes.addressof(CU), 2, 28, 256) + 3 * 8
    for bad in (dict(ws_bytes=need - 1), dict(ws=None), dict(ws=A + 8)):
        assert attend(call, **bad) == P.PACE_ERR_WORKSPACE
    assert size(FULL) > 0 and size(MANY) == 0 and size(FALLING) == 0 and size(CU, hq=30) == 0 and size(CU, c=call.cache(head_dim=80)) == 0


def accept(call, **kw):  # noqa: F811
    f = dict(tokens=A, parents=A + 4096, picked=A + 8192, cu=ctypes.addressof(CU), B=2, rows=A + 12288, counts=A + 16384, after=A + 20480)
    f.update(kw)
    return call.L.pace_draft_accept(f["tokens"], f["parents"], f["picked"], f["cu"], f["B"], f["rows"], f["counts"], f["after"], None)


@pytest.mark.parametrize("bad", [dict(B=-1), dict(tokens=None), dict(parents=None), dict(picked=None), dict(cu=None), dict(cu=ctypes.addressof(LATE)),
                                 dict(cu=ctypes.addressof(FALLING)), dict(rows=None), dict(counts=None), dict(after=None), dict(tokens=A + 1),
                                 dict(rows=A + 12290), dict(after=A + 20481), dict(rows=A), dict(rows=A + 8), dict(counts=A + 8192), dict(after=A + 4104),
                                 dict(rows=A + 16380), dict(counts=A + 20480)])
def test_accept_refuses(call, bad):  # noqa: F811
    assert accept(call, **bad) == INVALID


def compact(call, c=None, **kw):  # noqa: F811
    f = dict(cu=ctypes.addressof(CU), B=2, lens=A, table=A + 4096, ts=4, cu_rows=None, rows=A + 8192, counts=A + 12288, dst=None, ds=0,
             new=A + 16384, n=None)
    f.update(kw)
    c = c or [call.cache()]
    views = (P.KvCacheView * len(c))(*c)
    return call.L.pace_kv_compact(ctypes.addressof(views), len(c) if f["n"] is None else f["n"], f["cu"], f["B"], f["lens"], f["table"], f["ts"],
                                  f["cu_rows"], f["rows"], f["counts"], f["dst"], f["ds"], f["new"], None)


@pytest.mark.parametrize("bad", [dict(B=-1), dict(n=-1), dict(n=0), dict(cu=None), dict(cu=ctypes.addressof(FALLING)), dict(cu_rows=ctypes.addressof(LATE)),
                                 dict(cu_rows=ctypes.addressof(MORE)), dict(lens=None), dict(lens=A + 2), dict(table=None), dict(ts=0),
                                 dict(ts=1 << 31), dict(rows=A + 8194), dict(counts=A + 12289), dict(dst=A + 20480, ds=0),
                                 dict(dst=A + 4096, ds=5), dict(dst=A + 20482, ds=4), dict(new=None), dict(new=A + 16386), dict(new=A),
                                 dict(new=A + 4096 + 28), dict(new=A + 8192 + 8), dict(new=A + 12288 - 4),
                                 dict(dst=A + 20480, ds=4, new=A + 20480 + 24)])
def test_compact_refuses(call, bad):  # noqa: F811
    assert compact(call, **bad) == INVALID


@pytest.mark.parametrize("other", [dict(n_pages=9), dict(page_stride=4 * 64 * 128 + 16), dict(scale_stride=17), dict(n_kv_heads=2),
                                   dict(page_size=32), dict(head_dim=64)])
def test_compact_refuses_layers_that_differ(call, other):  # noqa: F811
    assert compact(call, c=[call.cache(), call.cache(**other)]) == INVALID


def test_nothing_to_do_is_no_error(call):  # noqa: F811
    none = (ctypes.c_int32 * 3)(0, 0, 0)
    assert attend(call, B=0) == P.PACE_OK and attend(call, cu=ctypes.addressof(none), parents=None) == P.PACE_OK
    assert accept(call, B=0) == P.PACE_OK
    assert compact(call, B=0) == P.PACE_OK


def test_binding_refuses_what_does_not_fit():
    ids = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):     # (not on a GPU)
        P.pace_draft_accept(ids, ids, ids, [0, 4])
    for layers in ([], [None]):
        with pytest.raises(ValueError):
            P.KvLayers(layers)
