"""Attention from trees of drafted tokens over the paged cache, and the walk along the accepted ones, against the fp64 oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import pace_oracle as O
from test_gpu_kv import BF16, Pool, _cu, _f64, _tokens, _upload, pace  # noqa: F401
from test_gpu_kv_range import _pattern, _set_keys

pytestmark = pytest.mark.gpu


def tree(shape, n, seed=0):
    """Parents of n nodes."""
    if n == 0:
        return []
    rng = np.random.default_rng(1000 + seed)
    if shape == "chain":
        return list(range(-1, n - 1))
    if shape == "flat":         # all of them follow the context
        return [-1] * n
    if shape == "star":         # all of them follow node 0
        return [-1] + [0] * (n - 1)
    if shape == "fours":
        return [(t - 1) // 4 if t else -1 for t in range(n)]
    p = [-1] + [int(rng.integers(0, t)) for t in range(1, n)]
    if shape == "forest":
        p = [-1 if rng.random() < 0.2 else x for x in p]
    return p


def _ids(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def check_tree(P, pool, Q, parents, window=0, sinks=0, **kw):
    """out and lse against the oracle; parents: a list per sequence.

    The kernels form scores and weights as they do for queries in a line, so the bounds are the same: out is rounded once to bf16 (2^-9 of
    it); a weight is held to 8 bits (2^-9) or, far below the largest weighted value, to 2^-18 of that, and carries the error of its
    score; the output can use up twice those.  A score is a sum of D products in fp32: off by at most 2^-23 (D + 8) times the sum
    of their sizes."""
    new = [len(p) for p in parents]
    cu = _cu(new)
    n, hq, D = Q.shape
    lse = torch.full((max(n, 1), hq), 7.0, device="cuda")
    out = P.pace_kv_tree_attention(pool.cache, Q, cu, _ids(sum(parents, [])), pool.lens, pool.table, max(pool.host_lens), window=window,
                                   sinks=sinks, lse=lse, **kw)
    q = _f64(Q)
    for b, up in enumerate(parents):
        if not up:
            continue
        k, v = pool.read("k", b), pool.read("v", b)
        see = O.kv_tree_visible(pool.host_lens[b], up, window, sinks)
        hidden = ~see.any(0)
        k[hidden] = v[hidden] = 0
        r = O.kv_attention_dense(q[cu[b]:cu[b + 1]], k, v, see, D ** -0.5)
        score = 2.0 ** -23 * (D + 8) * r["abs_score"] + 2.0 ** -20
        got = _f64(out[cu[b]:cu[b + 1]])
        tol = 2.0 ** -8 * np.abs(r["out"]) + (2.0 ** -8 + 2 * score[..., None]) * r["abs_out"] + 2.0 ** -17 * r["peak"][..., None]
        err = np.abs(got - r["out"])
        assert np.all(err <= tol), (b, float((err - tol).max()), float(err.max()))
        got = lse[cu[b]:cu[b + 1]].cpu().numpy().astype(np.float64)
        empty = np.isinf(r["lse"])
        assert np.array_equal(np.isneginf(got), empty)
        off = np.abs(got - np.where(empty, got, r["lse"]))[~empty]
        assert np.all(off <= (score + 2.0 ** -22 * np.abs(r["lse"]))[~empty]), float(off.max())
    return out, lse


# one node to more than two row tiles, few and many rows per KV head; a context of nothing, of one slot, ending inside a word, a block, a tile
@pytest.mark.parametrize("n,context", [(1, 0), (1, 1), (2, 0), (5, 27), (5, 126), (7, 404), (26, 31), (33, 1000), (64, 96), (100, 129), (257, 300)])
@pytest.mark.parametrize("shape", ["random", "forest", "fours"])
@pytest.mark.parametrize("hq,hkv,dim,page", [(28, 4, 128, 16), (14, 2, 64, 64), (8, 8, 128, 256), (32, 1, 64, 128)])
def test_one_tree(pace, n, context, shape, hq, hkv, dim, page):  # noqa: F811
    pool = Pool(pace, n, [n + context], hkv, dim, page)
    check_tree(pace, pool, _tokens(1, n, hq, dim), [tree(shape, n)])


@pytest.mark.parametrize("shape", ["chain", "flat", "star"])
@pytest.mark.parametrize("n,context", [(4, 60), (32, 10), (90, 700)])
@pytest.mark.parametrize("hq,hkv,dim", [(14, 2, 128), (4, 4, 64)])
def test_shapes(pace, shape, n, context, hq, hkv, dim):  # noqa: F811
    pool = Pool(pace, n, [n + context], hkv, dim, 32)
    check_tree(pace, pool, _tokens(2, n, hq, dim), [tree(shape, n)])


@pytest.mark.parametrize("shape", ["chain", "random", "flat"])
def test_the_largest_tree(pace, shape):  # noqa: F811
    n = pace.TREE_MAX
    pool = Pool(pace, 3, [n + 77], 1, 64, 64)
    check_tree(pace, pool, _tokens(3, n, 2, 64), [tree(shape, n)], window=0 if shape == "random" else 300, sinks=3)
    with pytest.raises(pace.PaceError):
        pace.pace_kv_tree_attention(pool.cache, _tokens(3, n + 1, 2, 64), [0, n + 1], _ids(tree("flat", n + 1)), pool.lens, pool.table, n + 77)


# ragged batches: single nodes among trees, sequences without nodes, empty ones, both forms in one call
@pytest.mark.parametrize("lens,nodes", [((300, 20, 4000, 17, 129, 640), (1, 7, 26, 17, 2, 64)), ((300, 0, 5, 129), (3, 0, 0, 40)), ((200,) * 40, (5,) * 40)])
@pytest.mark.parametrize("hq,hkv,dim,page", [(28, 4, 128, 64), (16, 2, 128, 32), (14, 2, 64, 16)])
def test_batches(pace, lens, nodes, hq, hkv, dim, page):  # noqa: F811
    pool = Pool(pace, 4, list(lens), hkv, dim, page)
    check_tree(pace, pool, _tokens(5, sum(nodes), hq, dim), [tree("forest" if b % 2 else "random", n, b) for b, n in enumerate(nodes)])


# windows: one slot, shorter than a path, inside the tree, across its edge, a tile's edge, wider than the sequence; sinks, some inside the tree
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 4), (5, 1), (40, 0), (128, 0), (100, 17), (129, 130), (1000, 4), (5000, 4), (30, 2000)])
@pytest.mark.parametrize("lens,nodes,shape", [((1500, 40, 7), (4, 3, 2), "chain"), ((1000, 300), (31, 64), "random"), ((600, 250), (233, 250), "chain"),
                                              ((500,), (100,), "forest")])
@pytest.mark.parametrize("hq,hkv,dim", [(14, 2, 128), (4, 2, 64)])
def test_windows(pace, window, sinks, lens, nodes, shape, hq, hkv, dim):  # noqa: F811
    pool = Pool(pace, 6, list(lens), hkv, dim, 32)
    check_tree(pace, pool, _tokens(7, sum(nodes), hq, dim), [tree(shape, n, b) for b, n in enumerate(nodes)], window=window, sinks=sinks)


# scales of blocks far apart (2^-12 .. 2^12 of each other), scores of many units
@pytest.mark.parametrize("lens,nodes", [((900, 300), (4, 3)), ((400,), (60,))])
@pytest.mark.parametrize("gain", [1.0, 30.0])
def test_uneven_scales(pace, lens, nodes, gain):  # noqa: F811
    pool = Pool(pace, 8, list(lens), 2, 128, 16, spread=6)
    check_tree(pace, pool, _tokens(9, sum(nodes), 14, 128) * gain, [tree("random", n) for n in nodes])


@pytest.mark.parametrize("n,hq", [(4, 8), (30, 8), (90, 4)])
def test_a_line_is_what_the_other_call_gives(pace, n, hq):  # noqa: F811
    """The same tiles and the same arithmetic, but for the order in that parts of an item are joined: sums of at most 64 parts, off by at most
    64 + 8 roundings of 2^-24 on either side, 2^-16.8 in all; then one rounding of the result."""
    pool = Pool(pace, 10, [n + 1300, n], 2, 64, 32)
    Q = _tokens(11, 2 * n, hq, 64)
    cu = [0, n, 2 * n]
    a, b = (torch.empty(2 * n, hq, device="cuda") for _ in range(2))
    want = pace.pace_kv_attention(pool.cache, Q, cu, pool.lens, pool.table, n + 1300, lse=a)
    got = pace.pace_kv_tree_attention(pool.cache, Q, cu, _ids(2 * tree("chain", n)), pool.lens, pool.table, n + 1300, lse=b)
    largest = max(np.abs(pool.read("v", i)).max() for i in range(2))
    np.testing.assert_allclose(_f64(got), _f64(want), rtol=2.0 ** -7, atol=2.0 ** -16 * largest)
    np.testing.assert_allclose(_f64(b), _f64(a), rtol=2.0 ** -22, atol=2.0 ** -16)


@pytest.mark.parametrize("n", [1, 5, 70])
def test_nodes_before_the_first_slot(pace, n):  # noqa: F811
    lens = [0, 3, n + 40]
    pool = Pool(pace, 12, lens, 2, 64, 16)
    Q = _tokens(13, 3 * n, 8, 64)
    parents = [tree("random", n, b) for b in range(3)]
    lse = torch.full((3 * n, 8), 7.0, device="cuda")
    out = pace.pace_kv_tree_attention(pool.cache, Q, _cu([n] * 3), _ids(sum(parents, [])), pool.lens, pool.table, max(lens), lse=lse)
    gone = n + max(0, n - 3)
    assert not out[:gone].any() and torch.isneginf(lse[:gone]).all()
    for b, length in ((1, 3), (2, n + 40)):
        base = length - n
        k, v = pool.read("k", b), pool.read("v", b)
        see = O.kv_tree_visible(length, parents[b])
        r = O.kv_attention_dense(_f64(Q[b * n:(b + 1) * n]), k, v, see, 64 ** -0.5)
        np.testing.assert_allclose(_f64(out[b * n:(b + 1) * n]), r["out"], rtol=0, atol=2.0 ** -6 * max(1.0, np.abs(r["out"]).max()))
        assert base >= 0 or not r["out"][:-base].any()


# NaN where a node does not look: its siblings' slots, slots before the window, behind its own row tile
@pytest.mark.parametrize("n,hq", [(4, 14), (8, 4), (70, 14), (200, 4)])
@pytest.mark.parametrize("dim", [64, 128])
def test_nan_in_hidden_slots_reaches_nobody(pace, n, hq, dim):  # noqa: F811
    length, window, sinks = 700, 90, 3
    pool = Pool(pace, 14, [length], 2, dim, 32)
    Q, base = _tokens(15, n, hq, dim), length - n
    parents = tree("random", n)
    parents[1:4] = [0, 0, 0]
    args = ([0, n], _ids(parents), pool.lens, pool.table, length)
    clean = pace.pace_kv_tree_attention(pool.cache, Q, *args, window=window, sinks=sinks).clone()
    for m in "kv":
        for j in range(sinks, base - window + 1):
            pool.raw[m][pool.pages[0][j // 32], :, j % 32] = 0x7F if j % 2 else 0xFF
    sick = base + 2      # a node that others have for a sibling
    pool.raw["k"][pool.pages[0][sick // 32], 0, sick % 32] = 0x7F
    pool.raw["v"][pool.pages[0][sick // 32], 1, sick % 32, 5] = 0x7F
    _upload(pool)
    got = pace.pace_kv_tree_attention(pool.cache, Q, *args, window=window, sinks=sinks)
    below = [2 in f for f in O.tree_family(parents)]
    for t in range(n):
        if below[t]:
            assert torch.isnan(got[t, 0]).all() and torch.isnan(got[t, hq // 2, 5])
        else:
            assert torch.equal(got[t], clean[t])


def test_bad_parents_are_reported(pace):  # noqa: F811
    pool = Pool(pace, 16, [100, 100], 2, 64, 16)
    Q = _tokens(17, 20, 4, 64)
    good = tree("random", 10)
    for at, what in ((3, 3), (3, 9), (0, 0), (5, -2), (9, 2 ** 31 - 1), (2, -2 ** 31)):
        bad = list(good)
        bad[at] = what
        got = pace.pace_kv_tree_attention(pool.cache, Q, [0, 10, 20], _ids(bad + good), pool.lens, pool.table, 100)
        assert pace.pace_device_status(clear=True) == (pace.PACE_ERR_INVALID_ARG, 16)
        bad[at] = -1
        want = pace.pace_kv_tree_attention(pool.cache, Q, [0, 10, 20], _ids(bad + good), pool.lens, pool.table, 100)
        assert torch.equal(got, want)


def test_lengths_and_pages_out_of_range_are_reported(pace):  # noqa: F811
    pool = Pool(pace, 18, [100, 100], 2, 64, 16)
    Q, ids = _tokens(19, 20, 4, 64), _ids(tree("random", 10) * 2)
    for lens in ([101, 100], [-1, 100], [2 ** 31 - 1, 100]):
        pace.pace_kv_tree_attention(pool.cache, Q, [0, 10, 20], ids, _ids(lens), pool.table, 100)
        assert pace.pace_device_status(clear=True) == (pace.PACE_ERR_INVALID_ARG, 15)
    table = pool.table.clone()
    table[0, 6] = pool.cache.n_pages
    pace.pace_kv_tree_attention(pool.cache, Q, [0, 10, 20], ids, pool.lens, table, 100)
    assert pace.pace_device_status(clear=True) == (pace.PACE_ERR_INVALID_ARG, 15)


def test_more_sequences_than_one_launch_takes(pace):  # noqa: F811
    nodes = [1 + i % 5 for i in range(300)]
    lens = [n + i % 37 for i, n in enumerate(nodes)]
    pool = Pool(pace, 20, lens, 1, 64, 16)
    check_tree(pace, pool, _tokens(21, sum(nodes), 4, 64), [tree("random", n, b) for b, n in enumerate(nodes)])


def test_captured_and_replayed_while_trees_and_lengths_change(pace):  # noqa: F811
    """Two graphs on one workspace, each replayed after the other: what they read is what the arrays hold then."""
    nodes, lens = [26, 3, 40], [900, 60, 2000]
    pool = Pool(pace, 22, lens, 2, 128, 32, poison=False)
    cu, hq, most = _cu(nodes), 8, 2000
    Q = [_tokens(23 + i, sum(nodes), hq, 128) for i in range(2)]
    parents = _ids(sum((tree("random", n, 1) for n in nodes), []))
    ws = torch.empty(pace.pace_kv_tree_attention_workspace_size(pool.cache, cu, hq, most), dtype=torch.uint8, device="cuda")
    out = [torch.empty_like(q) for q in Q]
    pace.pace_kv_tree_attention(pool.cache, Q[0], cu, parents, pool.lens, pool.table, most, out=out[0], ws=ws)
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            pace.pace_kv_tree_attention(pool.cache, Q[i], cu, parents, pool.lens, pool.table, most, window=50 * i, sinks=i, out=out[i], ws=ws)
        graphs.append(g)
    for step, now in enumerate(([700, 41, 1999], [33, 3, 900], [900, 60, 2000])):
        pool.lens.copy_(_ids(now))
        parents.copy_(_ids(sum((tree("forest", n, 5 + step) for n in nodes), [])))
        for g in graphs:
            g.replay()
        for i in range(2):
            want = pace.pace_kv_tree_attention(pool.cache, Q[i], cu, parents, pool.lens, pool.table, most, window=50 * i, sinks=i)
            assert torch.equal(out[i], want)


def test_another_stream(pace):  # noqa: F811
    pool = Pool(pace, 24, [300, 90], 2, 64, 16)
    Q, parents = _tokens(25, 40, 4, 64), _ids(tree("random", 20) * 2)
    want = pace.pace_kv_tree_attention(pool.cache, Q, [0, 20, 40], parents, pool.lens, pool.table, 300)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = pace.pace_kv_tree_attention(pool.cache, Q, [0, 20, 40], parents, pool.lens, pool.table, 300, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


# ---- the walk --------------------------------------------------------------------------------
def walk_inputs(nodes, shape, seed, few=3):
    """Trees whose tokens are few, so that children of one node often share one."""
    rng = np.random.default_rng(seed)
    parents = [tree(shape, n, seed + b) for b, n in enumerate(nodes)]
    tokens = [rng.integers(0, few, n) for n in nodes]
    picked = [rng.integers(0, few, n) for n in nodes]
    return parents, [t.tolist() for t in tokens], [t.tolist() for t in picked]


@pytest.mark.parametrize("nodes", [(1,), (2,), (31,), (32,), (33,), (128,), (129,), (700,), (5, 0, 26, 1, 64), (0,), tuple([7] * 1030)])
@pytest.mark.parametrize("shape", ["random", "forest", "star", "chain"])
def test_accept(pace, nodes, shape):  # noqa: F811
    for seed in range(4):
        parents, tokens, picked = walk_inputs(nodes, shape, seed, few=1 if shape == "chain" and seed == 0 else 3)
        cu = _cu(nodes)
        rows, counts, after = pace.pace_draft_accept(*(_ids(sum(x, [])) for x in (tokens, parents, picked)), cu)
        rows, counts, after = rows.cpu().numpy(), counts.cpu().numpy(), after.cpu().numpy()
        for b, n in enumerate(nodes):
            path = O.draft_accept(tokens[b], parents[b], picked[b])
            assert counts[b] == len(path)
            np.testing.assert_array_equal(rows[cu[b]:cu[b + 1]], [cu[b] + t for t in path] + [-1] * (n - len(path)))
            assert after[b] == (picked[b][path[-1]] if n else -1)


def test_accept_a_long_line(pace):  # noqa: F811
    n = 20011
    one = torch.ones(n, dtype=torch.int32, device="cuda")
    rows, counts, after = pace.pace_draft_accept(one, _ids(tree("chain", n)), one, [0, n])
    assert counts.item() == n and after.item() == 1 and torch.equal(rows, torch.arange(n, dtype=torch.int32, device="cuda"))


def test_accept_reports_bad_parents(pace):  # noqa: F811
    tokens = _ids([1, 1, 1, 1, 1, 1])
    for at, what, want in ((2, 2, [0, 1, -1]), (2, 5, [0, 1, -1]), (1, -2, [0, -1, -1]), (1, 2 ** 31 - 1, [0, -1, -1])):
        parents = [-1, 0, 1, -1, 0, 1]
        parents[at] = what
        rows, counts, _ = pace.pace_draft_accept(tokens, _ids(parents), tokens, [0, 3, 6])
        assert pace.pace_device_status(clear=True) == (pace.PACE_ERR_INVALID_ARG, 17)
        assert rows.tolist() == want + [3, 4, 5] and counts.tolist()[1] == 3


def test_accept_replayed(pace):  # noqa: F811
    nodes = (26, 40, 3)
    cu = _cu(nodes)
    first = [_ids(sum(x, [])) for x in walk_inputs(nodes, "random", 50)]
    outs = torch.empty(cu[-1], dtype=torch.int32, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")
    parents, tokens, picked = first
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pace.pace_draft_accept(tokens, parents, picked, cu, *outs)
    for seed in (51, 52):
        for t, x in zip(first, walk_inputs(nodes, "random", seed)):
            t.copy_(_ids(sum(x, [])))
        g.replay()
        for a, b in zip(outs, pace.pace_draft_accept(tokens, parents, picked, cu)):
            assert torch.equal(a, b)


# Scores in base 2 of up to +-mantissa 2^log2_size, exact (see the range tests): below, at and above where a row's are taken relative to one
@pytest.mark.parametrize("log2_size,mantissa", [(11, 1.9), (12, 1.0), (13, 1.0), (14, 1.3), (21, 1.9), (22, 1.0), (23, 1.0), (26, 1.7320508), (80, 1.3), (110, 1.1)])
@pytest.mark.parametrize("shape", ["rise", "fall", "saw"])
@pytest.mark.parametrize("count,hq,hkv,dim", [(90, 14, 2, 128), (50, 8, 8, 64), (3, 14, 2, 128), (2, 8, 8, 64)])
def test_scores_of_any_size(pace, shape, log2_size, mantissa, count, hq, hkv, dim):  # noqa: F811
    length = 1300
    pool = Pool(pace, 42, [length], hkv, dim, 64, spread=8)
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
    out = pace.pace_kv_tree_attention(pool.cache, Q, [0, count], _ids(parents), pool.lens, pool.table, length, scale=scale)
    r = O.kv_attention_dense(_f64(Q), pool.read("k", 0), pool.read("v", 0), O.kv_tree_visible(length, parents), scale)
    err = np.abs(_f64(out) - r["out"])
    tol = 2.0 ** -8 * np.abs(r["out"]) + 2.0 ** -8 * r["abs_out"] + 2.0 ** -17 * r["peak"][..., None]
    assert np.all(err <= tol), (float((err - tol).max()), float(err.max()))
