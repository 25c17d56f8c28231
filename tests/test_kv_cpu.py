"""The paged 8-bit cache without a GPU: the oracle's own rules, and what the calls refuse before anything is launched."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import pace_oracle as O
from paper_2608_27206_gb300 import build as pace_build
from paper_2608_27206_gb300 import pace as P


# ---- the oracle ------------------------------------------------------------------------------
def test_e4m3_rounding_is_nearest_even_of_all_codes():
    v = O.e4m3_values()
    fin = np.unique(v[np.isfinite(v)])
    assert fin.max() == 448.0 and np.isnan(v[0x7F]) and np.isnan(v[0xFF]) and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6
    np.testing.assert_array_equal(O.e4m3_round(fin), fin)
    mid = (fin[1:] + fin[:-1]) / 2
    got = O.e4m3_round(mid)
    even = [fin[i] if int(np.abs(fin[i]) / (fin[i + 1] - fin[i])) % 2 == 0 else fin[i + 1] for i in range(len(mid))]
    np.testing.assert_array_equal(got, even)
    assert O.e4m3_round(1e9) == 448.0
    x = np.random.default_rng(0).normal(0, 3, 4096).astype(np.float32)
    np.testing.assert_array_equal(O.e4m3_round(x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())


def test_scale_is_the_smallest_power_that_covers():
    for amax in (448.0, 448.0 * (1 + 2 ** -20), 1.0, 1.75, 1.7500001, 3e38, 2.0 ** -133, 2.0 ** -70, 0.0):
        s = float(O.kv_scale(amax))
        assert np.log2(s) == round(np.log2(s)) and 2.0 ** -64 <= s <= 2.0 ** 120
        assert amax <= 448 * s and (s == 2.0 ** -64 or amax > 224 * s)


def test_rotation_keeps_lengths_and_relative_angles():
    rng = np.random.default_rng(1)
    x, y = rng.normal(size=(1, 1, 64)), rng.normal(size=(1, 1, 64))
    f = 1e6 ** (-np.arange(32) / 32)
    turn = lambda v, p: O.rope_rotate(v, np.cos(p * f)[None], np.sin(p * f)[None])   # noqa: E731
    assert np.linalg.norm(turn(x, 77)) == pytest.approx(np.linalg.norm(x))
    assert np.sum(turn(x, 100) * turn(y, 93)) == pytest.approx(np.sum(turn(x, 7) * y))


def test_appending_in_pieces_covers_the_same_values():
    """Token by token or at once: the block ends with the same scale, and each value within the roundings it took."""
    rng = np.random.default_rng(2)
    x = rng.normal(size=(37, 2, 64)) * np.exp(rng.normal(size=(37, 1, 1)))
    whole, parts = (dict(v=np.zeros((4, 2, 16, 64)), s=np.full((4, 2, 1), np.nan)) for _ in range(2))
    pages = [2, 0, 3]
    O.kv_append(whole["v"], whole["s"], x, 0, pages)
    for i in range(37):
        O.kv_append(parts["v"], parts["s"], x[i:i + 1], i, pages)
    np.testing.assert_array_equal(whole["s"][pages], parts["s"][pages])
    a, b = (O.kv_read(c["v"], c["s"], pages, 37) for c in (whole, parts))
    lsb = np.repeat(np.maximum(1e-30, np.concatenate([whole["s"][p, :, 0][None] for p in pages])), 16, axis=0)[:37, :, None] * 2.0 ** -9
    assert np.all(np.abs(a - x) <= np.maximum(np.abs(x) * 2.0 ** -4, lsb / 2))
    assert np.all(np.abs(b - a) <= lsb)     # a growing scale moves a code by less than one subnormal step


def test_visibility():
    np.testing.assert_array_equal(O.kv_visible(3, 3), np.tril(np.ones((3, 3), bool)))
    v = O.kv_visible(10, 2, window=3, sinks=2)
    assert [np.nonzero(r)[0].tolist() for r in v] == [[0, 1, 6, 7, 8], [0, 1, 7, 8, 9]]
    assert not O.kv_visible(2, 3)[0].any()      # a query before the first slot sees nothing


# ---- refusals: before the device is looked at ------------------------------------------------
@pytest.fixture(scope="module")
def call():
    pace_build.build()
    L = P.lib()
    A = 1 << 20     # an address that is never followed
    cu = (ctypes.c_int32 * 3)(0, 2, 3)

    def cache(**kw):
        f = dict(k=A, v=A, k_scale=A, v_scale=A, n_pages=8, page_stride=4 * 64 * 128, scale_stride=16, page_size=64, n_kv_heads=4,
                 head_dim=128)
        f.update(kw)
        return P.KvCacheView(*[f[n] for n, _ in P.KvCacheView._fields_])

    def append(c=None, rope=None, **kw):
        f = dict(K=A, V=A, ks=512, vs=512, n_src=3, cu=ctypes.addressof(cu), B=2, lens=A, table=A, ts=4, rows=None, Q=None, qs=0,
                 hq=0, q_out=None)
        f.update(kw)
        c = c or cache()
        return L.pace_kv_append(ctypes.addressof(c), f["K"], f["V"], f["ks"], f["vs"], f["n_src"], f["cu"], f["B"], f["lens"],
                                f["table"], f["ts"], f["rows"], None if rope is None else ctypes.addressof(rope), f["Q"], f["qs"],
                                f["hq"], f["q_out"], None)

    def attend(c=None, **kw):
        f = dict(Q=A, qs=28 * 128, cu=ctypes.addressof(cu), B=2, hq=28, lens=A, table=A, ts=4, max_len=256, scale=0.1, window=0,
                 sinks=0, out=A, lse=None, ws=A, ws_bytes=1 << 40)
        f.update(kw)
        c = c or cache()
        return L.pace_kv_attention(ctypes.addressof(c), f["Q"], f["qs"], f["cu"], f["B"], f["hq"], f["lens"], f["table"], f["ts"],
                                   f["max_len"], f["scale"], f["window"], f["sinks"], f["out"], f["lse"], f["ws"], f["ws_bytes"], None)

    class Calls:
        pass
    Calls.L, Calls.A, Calls.cache, Calls.append, Calls.attend = L, A, staticmethod(cache), staticmethod(append), staticmethod(attend)
    return Calls


BAD_CACHE = [dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(k=(1 << 20) + 8), dict(v_scale=(1 << 20) + 2),
             dict(n_pages=0), dict(n_pages=1 << 31), dict(page_size=0), dict(page_size=48), dict(page_size=512), dict(n_kv_heads=0),
             dict(n_kv_heads=257), dict(head_dim=80), dict(head_dim=0), dict(page_stride=4 * 64 * 128 - 16),
             dict(page_stride=4 * 64 * 128 + 8), dict(scale_stride=15), dict(page_stride=1 << 62)]


@pytest.mark.parametrize("bad", BAD_CACHE)
def test_both_calls_refuse_a_bad_cache(call, bad):
    assert call.append(c=call.cache(**bad)) == P.PACE_ERR_INVALID_ARG
    assert call.attend(c=call.cache(**bad)) == P.PACE_ERR_INVALID_ARG


A = 1 << 20
FALLING = (ctypes.c_int32 * 3)(0, 2, 1)
LATE = (ctypes.c_int32 * 3)(1, 2, 3)


@pytest.mark.parametrize("bad", [dict(B=-1), dict(K=None), dict(V=None), dict(K=A + 8), dict(ks=511), dict(ks=516), dict(vs=504), dict(cu=None),
                                 dict(cu=ctypes.addressof(FALLING)), dict(cu=ctypes.addressof(LATE)), dict(lens=None), dict(table=None),
                                 dict(ts=0), dict(n_src=0), dict(n_src=2), dict(Q=A), dict(q_out=A), dict(Q=A, q_out=A, qs=128, hq=0),
                                 dict(Q=A, q_out=A, qs=128, hq=2), dict(Q=A, q_out=A + 2, qs=256, hq=2)])
def test_append_refuses(call, bad):
    assert call.append(**bad) == P.PACE_ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [dict(table=None), dict(table=A + 8), dict(positions=None), dict(n_positions=0), dict(positions_stride=-1),
                                 dict(sections=(64, 64, 0)), dict(sections=(16, 24, 23)), dict(sections=(-1, 65, 0))])
def test_append_refuses_a_bad_rotation(call, bad):
    f = dict(table=A, positions=A, n_positions=100, positions_stride=3, sections=(16, 24, 24))
    f.update(bad)
    r = P.Rope(f["table"], f["positions"], f["n_positions"], f["positions_stride"], (ctypes.c_int32 * 3)(*f["sections"]))
    assert call.append(rope=r) == P.PACE_ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [dict(B=-1), dict(Q=None), dict(Q=A + 8), dict(qs=28 * 128 - 8), dict(qs=28 * 128 + 4), dict(cu=None),
                                 dict(cu=ctypes.addressof(FALLING)), dict(hq=0), dict(hq=30), dict(hq=4 * 65, qs=4 * 65 * 128), dict(lens=None), dict(table=None), dict(ts=0),
                                 dict(max_len=-1), dict(max_len=257), dict(scale=0.0), dict(scale=float("nan")), dict(sinks=-1),
                                 dict(out=None), dict(out=A + 2)])
def test_attention_refuses(call, bad):
    assert call.attend(**bad) == P.PACE_ERR_INVALID_ARG


def test_attention_refuses_a_small_workspace(call):
    c = call.cache()
    cu = (ctypes.c_int32 * 3)(0, 2, 3)
    need = call.L.pace_kv_attention_workspace_size(ctypes.addressof(c), ctypes.addressof(cu), 2, 28, 256)
    assert need >= 16
    for bad in (dict(ws_bytes=need - 1), dict(ws=None), dict(ws=A + 8)):
        assert call.attend(**bad) == P.PACE_ERR_WORKSPACE
    assert call.L.pace_kv_attention_workspace_size(ctypes.addressof(c), ctypes.addressof(cu), 2, 30, 256) == 0
    assert call.L.pace_kv_attention_workspace_size(ctypes.addressof(call.cache(head_dim=80)), ctypes.addressof(cu), 2, 28, 256) == 0


def test_nothing_to_do_is_no_error(call):
    none = (ctypes.c_int32 * 3)(0, 0, 0)
    assert call.append(B=0) == P.PACE_OK and call.attend(B=0) == P.PACE_OK
    assert call.append(cu=ctypes.addressof(none)) == P.PACE_OK and call.attend(cu=ctypes.addressof(none)) == P.PACE_OK
    assert call.L.pace_rope_table(None, 0, 128, 1e6, None) == P.PACE_OK


@pytest.mark.parametrize("bad", [(A, -1, 128, 1e6), (A, 4, 80, 1e6), (A, 4, 128, 0.0), (A, 4, 128, float("inf")), (None, 4, 128, 1e6),
                                 (A + 4, 4, 128, 1e6)])
def test_rope_table_refuses(call, bad):
    assert call.L.pace_rope_table(*bad, None) == P.PACE_ERR_INVALID_ARG


def test_binding_refuses_tensors_that_do_not_fit():
    codes, scales = torch.zeros(2, 4, 32, 64, dtype=torch.uint8), torch.zeros(2, 4, 2)
    for k, s in ((codes, scales[..., :1]), (codes[0], scales), (codes.float(), scales), (codes, scales.double()), (codes, scales)):
        with pytest.raises(ValueError):     # (the last: not on a GPU)
            P.KvCache(k, codes, s, scales)
