"""Trees of one row tile on long contexts, where the two halves of a CTA share an item's slots: batches that give every CTA eight slot tiles
of an item and more, whole items and parts of them, with odd and even numbers of tiles."""
import math

import numpy as np
import pytest
import torch

from oracle import pace_oracle as O
from test_gpu_kv import BF16, Pool, _cu, _f64, _tokens, _upload, pace  # noqa: F401
from test_gpu_kv_range import _pattern, _set_keys
from test_gpu_kv_tree import _ids, check_tree, tree

pytestmark = pytest.mark.gpu


# rows of a tile on both sides of 16, 32, 64, 96 and 128; a second tile of few rows
@pytest.mark.parametrize("nodes,group", [(17, 1), (11, 3), (9, 2), (16, 2), (17, 2), (31, 2), (32, 2), (33, 2), (13, 7), (18, 7), (19, 7), (63, 2), (130, 2)])
@pytest.mark.parametrize("dim,page", [(128, 64), (64, 16)])
def test_rows(pace, nodes, group, dim, page):  # noqa: F811
    heads = 8
    lens = [nodes + 1200 + 61 * (i % 9) for i in range(24)]
    pool = Pool(pace, 90, lens, heads, dim, page)
    # (the oracle looks at some of the sequences; all are there to fill the line)
    Q = _tokens(91, 24 * nodes, heads * group, dim)
    check_some(pace, pool, Q, [tree("random" if i % 2 else "forest", nodes, i) for i in range(24)], [0, 7, 16, 23])


def check_some(P, pool, Q, parents, which, **kw):
    """check_tree of all sequences' call for a few of them: the others' results are compared with theirs alone."""
    cu = _cu([len(p) for p in parents])
    out = P.pace_kv_tree_attention(pool.cache, Q, cu, _ids(sum(parents, [])), pool.lens, pool.table, max(pool.host_lens), **kw)
    lse = torch.empty(Q.shape[:2], device="cuda")
    P.pace_kv_tree_attention(pool.cache, Q, cu, _ids(sum(parents, [])), pool.lens, pool.table, max(pool.host_lens), lse=lse, **kw)
    D, window, sinks = Q.shape[2], kw.get("window", 0), kw.get("sinks", 0)
    for b in which:
        k, v = pool.read("k", b), pool.read("v", b)
        see = O.kv_tree_visible(pool.host_lens[b], parents[b], window, sinks)
        hidden = ~see.any(0)
        k[hidden] = v[hidden] = 0
        r = O.kv_attention_dense(_f64(Q[cu[b]:cu[b + 1]]), k, v, see, D ** -0.5)
        score = 2.0 ** -23 * (D + 8) * r["abs_score"] + 2.0 ** -20      # (the bounds of check_tree)
        tol = 2.0 ** -8 * np.abs(r["out"]) + (2.0 ** -8 + 2 * score[..., None]) * r["abs_out"] + 2.0 ** -17 * r["peak"][..., None]
        assert np.all(np.abs(_f64(out[cu[b]:cu[b + 1]]) - r["out"]) <= tol), b
        got = lse[cu[b]:cu[b + 1]].cpu().numpy().astype(np.float64)
        assert np.all(np.abs(got - r["lse"]) <= score + 2.0 ** -22 * np.abs(r["lse"])), b
    return out


@pytest.mark.parametrize("window,sinks", [(1100, 0), (1500, 200), (1030, 4), (20, 1250)])
@pytest.mark.parametrize("dim", [64, 128])
def test_windows(pace, window, sinks, dim):  # noqa: F811
    nodes = [9 + i % 30 for i in range(24)]
    lens = [n + 1400 + 53 * (i % 11) for i, n in enumerate(nodes)]
    pool = Pool(pace, 92, lens, 8, dim, 32)
    check_some(pace, pool, _tokens(93, sum(nodes), 16, dim), [tree("chain" if i % 3 == 0 else "random", n, i) for i, n in enumerate(nodes)],
               [0, 5, 22], window=window, sinks=sinks)


@pytest.mark.parametrize("gain", [1.0, 30.0])
def test_uneven_scales(pace, gain):  # noqa: F811
    nodes = [12] * 24
    pool = Pool(pace, 94, [1300 + 40 * i for i in range(24)], 8, 128, 16, spread=6)
    check_some(pace, pool, _tokens(95, sum(nodes), 24, 128) * gain, [tree("random", 12, i) for i in range(24)], [1, 12, 23])


@pytest.mark.parametrize("dim", [64, 128])
def test_rows_that_see_one_half_or_nothing(pace, dim):  # noqa: F811
    """Windows so short that most of a context's tiles hold nothing for a row, and sequences shorter than their nodes."""
    nodes = [40] * 24
    lens = [1640 + 20 * i if i % 4 else 25 for i in range(24)]
    pool = Pool(pace, 96, lens, 8, dim, 64)
    Q = _tokens(97, sum(nodes), 16, dim)
    parents = [tree("random", 40, i) for i in range(24)]
    cu = _cu(nodes)
    lse = torch.empty(sum(nodes), 16, device="cuda")
    out = pace.pace_kv_tree_attention(pool.cache, Q, cu, _ids(sum(parents, [])), pool.lens, pool.table, max(lens), window=8, sinks=1400, lse=lse)
    for b in (0, 1, 4, 9, 23):
        k, v = pool.read("k", b), pool.read("v", b)
        see = O.kv_tree_visible(lens[b], parents[b], 8, 1400)
        hidden = ~see.any(0)
        k[hidden] = v[hidden] = 0
        r = O.kv_attention_dense(_f64(Q[cu[b]:cu[b + 1]]), k, v, see, dim ** -0.5)
        none = ~see.any(1)
        got = out[cu[b]:cu[b + 1]]
        assert not got[none].any() and torch.isneginf(lse[cu[b]:cu[b + 1]][none]).all() and none.any() == (lens[b] < 40)
        score = 2.0 ** -23 * (dim + 8) * r["abs_score"] + 2.0 ** -20
        tol = 2.0 ** -8 * np.abs(r["out"]) + (2.0 ** -8 + 2 * score[..., None]) * r["abs_out"] + 2.0 ** -17 * r["peak"][..., None]
        assert np.all(np.abs(_f64(got) - r["out"]) <= tol)


@pytest.mark.parametrize("dim", [64, 128])
def test_nan_in_one_half(pace, dim):  # noqa: F811
    """A NaN reaches the rows that see it, by whichever half it comes, and no others."""
    nodes = [20] * 24
    lens = [1400 + 20] * 24
    pool = Pool(pace, 98, lens, 8, dim, 16)
    Q = _tokens(99, sum(nodes), 16, dim)
    parents = [[-1] + [0] * 19 for _ in range(24)]
    args = (_cu(nodes), _ids(sum(parents, [])), pool.lens, pool.table, 1420)
    clean = pace.pace_kv_tree_attention(pool.cache, Q, *args).clone()
    for b, slot in ((3, 1400 + 5), (4, 130), (5, 300)):      # a node; context slots of a tile with an odd and with an even number
        pool.raw["v"][pool.pages[b][slot // 16], :, slot % 16, 7] = 0x7F
    _upload(pool)
    got = pace.pace_kv_tree_attention(pool.cache, Q, *args)
    for b in range(24):
        rows = slice(20 * b, 20 * b + 20)
        if b == 3:
            assert torch.isnan(got[rows][5, :, 7]).all()
            keep = [t for t in range(20) if t != 5]
            assert torch.equal(got[rows][keep], clean[rows][keep])
        elif b in (4, 5):
            assert torch.isnan(got[rows][:, :, 7]).all()
        else:
            assert torch.equal(got[rows], clean[rows])


# Scores in base 2 of up to +-mantissa 2^log2_size along one long sequence, V scales of 2^-8 to 2^8: the halves' bases are far apart
@pytest.mark.parametrize("log2_size,mantissa", [(4, 1.0), (12, 1.0), (13, 1.0), (14, 1.9), (16, 1.3), (21, 1.9), (23, 1.0), (26, 1.7320508), (32, 1.0), (80, 1.3), (110, 1.1)])
@pytest.mark.parametrize("shape", ["rise", "fall", "saw"])
@pytest.mark.parametrize("dim", [64, 128])
def test_scores_of_any_size(pace, shape, log2_size, mantissa, dim):  # noqa: F811
    count, hq, hkv, length = 6, 24, 8, 20000
    pool = Pool(pace, 100, [length], hkv, dim, 64, spread=8)
    j = np.arange(length)
    curve = {"rise": j / length * 2 - 1, "fall": 1 - j / length * 2, "saw": (j % 170) / 170 * (0.2 + 0.8 * j / length)}[shape]
    u = _pattern(hkv, dim)
    of_scale, of_q = log2_size // 2 - 8, log2_size // 4
    _set_keys(pool, u, curve * 256, log2_size - 8 - of_scale - of_q)
    _upload(pool)
    steep = np.resize([1.0, -1.0, 0.125, 0.5, -0.25], count * hq).reshape(count, hq, 1)
    Q = torch.from_numpy(steep * 2.0 ** of_q * np.repeat(u, hq // hkv, axis=0)[None]).to(BF16).cuda()
    scale = float(np.float32(mantissa * math.log(2) * 2.0 ** of_scale / dim))
    parents = tree("random", count)
    lse = torch.empty(count, hq, device="cuda")
    out = pace.pace_kv_tree_attention(pool.cache, Q, [0, count], _ids(parents), pool.lens, pool.table, length, scale=scale, lse=lse)
    r = O.kv_attention_dense(_f64(Q), pool.read("k", 0), pool.read("v", 0), O.kv_tree_visible(length, parents), scale)
    # (as check_exact_scores of the range tests: one rounding to bf16, weights of 8 bits twice over, what is far below off by 2^-18; lse five roundings)
    err = np.abs(_f64(out) - r["out"])
    tol = 2.0 ** -8 * np.abs(r["out"]) + 2.0 ** -8 * r["abs_out"] + 2.0 ** -17 * r["peak"][..., None]
    assert np.all(err <= tol), (float((err - tol).max()), float(err.max()))
    off = np.abs(lse.cpu().numpy().astype(np.float64) - r["lse"])
    assert np.all(off <= 2.0 ** -21 * np.abs(r["lse"]) + 2.0 ** -18), float(off.max())


def test_check_tree_of_a_whole_batch(pace):  # noqa: F811
    nodes = [5 + i % 14 for i in range(40)]
    pool = Pool(pace, 101, [n + 1000 + 37 * i for i, n in enumerate(nodes)], 4, 64, 64)
    check_tree(pace, pool, _tokens(102, sum(nodes), 20, 64), [tree("forest", n, i) for i, n in enumerate(nodes)])
