"""Kept tokens of the paged cache moved together, in place and to other pages, against the fp64 oracle: every code and scale of it."""
import math

import numpy as np
import pytest
import torch

from oracle import pace_oracle as O
from test_gpu_kv import DECODE, Pool, _cu, _f64, _tokens, _upload, pace  # noqa: F401

pytestmark = pytest.mark.gpu


def _ids(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda").contiguous()


def lists(nodes, kept, seed):
    """Per sequence, which of its newest tokens stay."""
    rng = np.random.default_rng(seed)
    return [np.sort(rng.permutation(n)[:k]) for n, k in zip(nodes, kept)]


class Case:
    """Layers of random caches, sequences' source pages and, if they move, pages of their own from the one on that their newest tokens
    begin in."""

    def __init__(self, P, seed, lens, nodes, kept, heads, dim, page, layers=1, away=False, spread=3):
        self.P, self.lens, self.nodes, self.page = P, list(lens), list(nodes), page
        extra = [-(-n // page) * page for n in lens] if away else []
        self.pools = [Pool(P, seed + l, list(lens) + extra, heads, dim, page, poison=False, spread=spread) for l in range(layers)]
        one = self.pools[0]
        for p in self.pools[1:]:      # one block table for all
            p.pages, p.table = one.pages, one.table
        B = len(lens)
        self.source = one.pages[:B]
        self.target = self.source
        if away:
            first = [(n - m) // page for n, m in zip(lens, nodes)]
            self.target = [np.concatenate([self.source[b][:f], one.pages[B + b][f:]]) for b, f in enumerate(first)]
        self.table, self.dst = (self._table(t) for t in (self.source, self.target))
        self.away = away
        self.cache = P.KvLayers([p.cache for p in self.pools]) if layers != 1 else one.cache
        self.kept = lists(nodes, kept, seed)
        self.dev_lens = _ids(lens)

    def _table(self, pages):
        t = np.full((len(pages), max([len(p) for p in pages] + [1]) + 1), -9, np.int32)
        for b, p in enumerate(pages):
            t[b, :len(p)] = p
        return torch.from_numpy(t).cuda()

    def rows(self):
        cu = _cu(self.nodes)
        return _cu([len(k) for k in self.kept]), _ids(np.concatenate([k + cu[b] for b, k in enumerate(self.kept)] + [[]]))

    def call(self, **kw):
        cu_rows, rows = self.rows()
        args = dict(cu_rows=cu_rows, rows=rows)
        if self.away:
            args["dst_table"] = self.dst
        args.update(kw)
        return self.P.pace_kv_compact(self.cache, _cu(self.nodes), self.dev_lens, self.table, **args)

    def check(self, new_lens, kept=None):
        """Everything in the layers: moved tokens, their scales, and all that was to stay as it was."""
        kept = self.kept if kept is None else kept
        assert new_lens.tolist() == [n - m + len(k) for n, m, k in zip(self.lens, self.nodes, kept)]
        for pool in self.pools:
            for n in "kv":
                values, scales = DECODE[pool.raw[n]], pool.s[n].copy()
                free = np.zeros(values.shape[:1] + values.shape[2:3], bool)      # slots behind the last kept token of a written block
                for b, k in enumerate(kept):
                    if len(k) == 0:
                        continue
                    base = self.lens[b] - self.nodes[b]
                    O.kv_compact(values, scales, self.source[b], self.target[b], base, k)
                    end = base + len(k)
                    for j in range(end, -(-end // 16) * 16):
                        free[self.target[b][j // self.page], j % self.page] = True
                codes, got_s = pool.now(n)
                np.testing.assert_array_equal(got_s, scales)
                got = DECODE[codes]
                same = (got == values) | (np.isnan(got) & np.isnan(values))
                assert np.all(same | free[:, None, :, None]), int((~(same | free[:, None, :, None])).sum())
                assert np.array_equal(codes[np.broadcast_to(free[:, None, :, None], codes.shape)],
                                      pool.raw[n][np.broadcast_to(free[:, None, :, None], codes.shape)])


# all, some and none kept; one token; starts and ends inside blocks and pages, several sequences, sequences without newest tokens
@pytest.mark.parametrize("lens,nodes,kept", [((1,), (1,), (1,)), ((40,), (26,), (1,)), ((40,), (26,), (0,)), ((407,), (23,), (23,)), ((64,), (64,), (17,)),
                                             ((300, 77, 9, 130, 50), (40, 77, 0, 2, 33), (7, 31, 0, 2, 33)), ((333,), (300,), (120,)),
                                             ((1500, 1031), (1500, 1000), (640, 401))])
@pytest.mark.parametrize("heads,dim,page", [(4, 128, 64), (2, 64, 16), (1, 128, 256), (5, 64, 32)])
@pytest.mark.parametrize("away", [False, True])
def test_move(pace, lens, nodes, kept, heads, dim, page, away):  # noqa: F811
    case = Case(pace, 30, lens, nodes, kept, heads, dim, page, away=away)
    case.check(case.call())


@pytest.mark.parametrize("layers", [2, 5, 70])
@pytest.mark.parametrize("away", [False, True])
def test_layers(pace, layers, away):  # noqa: F811
    case = Case(pace, 31, (60, 45), (30, 45), (9, 20), 2, 64, 16, layers=layers, away=away)
    case.check(case.call())


@pytest.mark.parametrize("away", [False, True])
def test_a_list_with_room_and_counts(pace, away):  # noqa: F811
    """As the walk leaves it: lists as long as the trees, and how much of them counts, none of one."""
    nodes = (26, 7, 40, 12)
    case = Case(pace, 32, (90, 40, 40, 100), nodes, (5, 7, 1, 3), 4, 128, 32, away=away)
    cu = _cu(nodes)
    rows = np.full(cu[-1], -1)
    for b, k in enumerate(case.kept):
        rows[cu[b]:cu[b] + len(k)] = k + cu[b]
    counts = [5, 7, 1, 0]
    got = case.call(cu_rows=None, rows=_ids(rows), counts=_ids(counts))
    case.check(got, [k[:c] for k, c in zip(case.kept, counts)])


@pytest.mark.parametrize("away", [False, True])
def test_all_of_them_without_a_list(pace, away):  # noqa: F811
    case = Case(pace, 33, (407, 100), (23, 100), (23, 100), 3, 128, 64, away=away)
    case.check(case.call(cu_rows=None, rows=None))


def test_counts_without_a_list(pace):  # noqa: F811
    """The first ones stay: the sequence is cut, and its last block gets the scale of what is left."""
    case = Case(pace, 34, (100, 60), (50, 60), (20, 33), 2, 64, 16)
    case.kept = [np.arange(20), np.arange(33)]
    case.check(case.call(cu_rows=None, rows=None, counts=_ids([20, 33])))


@pytest.mark.parametrize("away", [False, True])
def test_scales_far_apart(pace, away):  # noqa: F811
    """2^-120 to 2^120 of each other: what is lost under a large one is lost, what comes from under one comes back whole."""
    case = Case(pace, 35, (400,), (400,), (150,), 2, 64, 16, away=away, spread=60)
    case.check(case.call())


def test_zeros_get_the_smallest_scale(pace):  # noqa: F811
    case = Case(pace, 36, (64,), (64,), (40,), 2, 64, 16)
    for p in case.pools:
        p.raw["k"][:] = 0
        _upload(p)
    case.check(case.call())
    assert (case.pools[0].now("k")[1][case.source[0][0]] == 2.0 ** -64).all()


@pytest.mark.parametrize("what", ["code", "nan", "inf", "zero", "negative"])
@pytest.mark.parametrize("away", [False, True])
def test_nan_codes_and_bad_scales_count_as_zero_and_are_reported(pace, away, what):  # noqa: F811
    case = Case(pace, 37, (90,), (60,), (8,), 2, 64, 16, away=away)
    case.kept = [np.array([0, 3, 8, 9, 30, 31, 33, 59])]
    pool, pg = case.pools[0], case.source[0][3]      # slots 48 .. 63: of kept tokens 30, 31 and 33
    if what == "code":
        pool.raw["v"][pg, 1, 13, 17] = 0xFF
    else:
        pool.s["v"][pg, 1, 0] = dict(nan=math.nan, inf=math.inf, zero=0.0, negative=-1.0)[what]
    _upload(pool)
    got = case.call()
    assert pace.pace_device_status(clear=True) == (pace.PACE_ERR_INVALID_ARG, 18) and got.tolist() == [38]
    for n in "kv":
        values, scales = DECODE[pool.raw[n]], pool.s[n].copy()
        if n == "v":
            values[pg, 1, [13] if what == "code" else [12, 13, 15]] = 0
            scales[pg, 1, 0] = scales[pg, 1, 0] if what == "code" else 1.0
        O.kv_compact(values, scales, case.source[0], case.target[0], 30, case.kept[0])
        codes, got_s = pool.now(n)
        for slot in range(16, 38):
            p, at = case.target[0][slot // 16], slot % 16
            np.testing.assert_array_equal(DECODE[codes[p, :, at]], values[p, :, at])
            np.testing.assert_array_equal(got_s[p], scales[p])


# numbers out of range: reported; what they name counts as 0 or stays, the other sequence is as it should be
@pytest.mark.parametrize("what", ["row", "row_negative", "row_again", "row_falls", "page", "page_negative", "target", "count", "count_negative", "short"])
@pytest.mark.parametrize("away", [False, True])
def test_numbers_out_of_range(pace, what, away):  # noqa: F811
    case = Case(pace, 38, (80, 70), (50, 40), (20, 15), 2, 64, 16, away=away)
    cu_rows, rows = case.rows()
    counts, lens, table, dst = _ids([20, 15]), case.dev_lens.clone(), case.table.clone(), case.dst.clone()
    if what == "row":
        rows[4] = 50
    elif what == "row_negative":
        rows[4] = -1
    elif what == "row_again":
        rows[4] = rows[3]
    elif what == "row_falls":
        rows[4] = rows[3] - 1
    elif what.startswith("page"):
        table[0, 4] = case.pools[0].cache.n_pages if what == "page" else -1
    elif what == "target":
        dst[0, 2] = -1
        table = dst if not away else table
    elif what == "count":
        counts[0] = 21
    elif what == "count_negative":
        counts[0] = -1
    else:
        lens[0] = 49
    before = {n: case.pools[0].now(n) for n in "kv"}
    kw = dict(dst_table=dst) if away else {}
    got = pace.pace_kv_compact(case.cache, _cu(case.nodes), lens, table, cu_rows=cu_rows, rows=rows, counts=counts, **kw)
    assert pace.pace_device_status(clear=True) == (pace.PACE_ERR_INVALID_ARG, 18)
    nothing = what in ("count", "count_negative", "short")
    assert got.tolist() == [(lens[0].item() if nothing else 50), 45]
    for n in "kv":
        codes, scales = case.pools[0].now(n)
        values, want_s = DECODE[case.pools[0].raw[n]], case.pools[0].s[n].copy()
        O.kv_compact(values, want_s, case.source[1], case.target[1], 30, case.kept[1])
        pages = sorted(set(case.target[1][1:3].tolist()))
        for slot in range(16, 45):
            p, a = case.target[1][slot // 16], slot % 16
            np.testing.assert_array_equal(DECODE[codes[p, :, a]], values[p, :, a])
        np.testing.assert_array_equal(scales[pages], want_s[pages])
        mine = set(case.target[0].tolist()) | set(pages)
        spare = [p for p in range(len(codes)) if p not in mine]
        assert np.array_equal(codes[spare], before[n][0][spare])
        if nothing:
            own = case.target[0].tolist()
            assert np.array_equal(codes[own], before[n][0][own]) and np.array_equal(scales[own], before[n][1][own])
        if what == "row_negative":      # kept token 4, at slot 34
            p = case.target[0][2]
            assert not DECODE[codes[p, :, 2]].any()


def test_shared_prefix_and_source(pace):  # noqa: F811
    """A prompt's part-filled last page copied for several answers: they share its other pages, and the page that they copy from."""
    pool = Pool(pace, 39, [71, 16, 16, 16], 2, 128, 16, poison=False, spread=2)
    own = pool.pages[0]
    table = _ids([list(own)] * 3)
    dst = _ids([list(own[:4]) + [pool.pages[b + 1][0]] for b in range(3)])
    before = pool.now("k")
    lens = pace.pace_kv_compact(pool.cache, [0, 7, 14, 21], _ids([71] * 3), table, dst_table=dst)
    assert lens.tolist() == [71] * 3
    for n in "kv":
        values, scales = DECODE[pool.raw[n]], pool.s[n].copy()
        codes, got = pool.now(n)
        for b in range(3):
            O.kv_compact(values, scales, own, list(own[:4]) + [pool.pages[b + 1][0]], 64, np.arange(7))
            p = pool.pages[b + 1][0]
            np.testing.assert_array_equal(DECODE[codes[p, :, :7]], values[p, :, :7])
            np.testing.assert_array_equal(got[p], scales[p])
    after = pool.now("k")
    assert np.array_equal(before[0][own], after[0][own]) and np.array_equal(before[1][own], after[1][own])


def test_more_sequences_than_one_launch_takes(pace):  # noqa: F811
    nodes = [1 + i % 7 for i in range(300)]
    lens = [n + i % 23 for i, n in enumerate(nodes)]
    for away in (False, True):
        case = Case(pace, 40, lens, nodes, [1 + n // 2 for n in nodes], 1, 64, 16, away=away)
        case.check(case.call())


def test_pages_that_lie_apart(pace):  # noqa: F811
    """Layers side by side in one allocation: pages of a layer are as far apart as all layers' are long."""
    layers, n_pages, heads, page, dim = 3, 7, 2, 16, 64
    g = torch.Generator().manual_seed(41)
    codes = [torch.randint(0, 127, (n_pages, layers, heads, page, dim), dtype=torch.uint8, generator=g).cuda() for _ in "kv"]
    scales = [torch.ones(n_pages, layers, heads, 1, device="cuda") * 2.0 ** -i for i in range(2)]
    was = [c.clone() for c in codes]
    cache = pace.KvLayers([pace.KvCache(codes[0][:, l], codes[1][:, l], scales[0][:, l], scales[1][:, l]) for l in range(layers)])
    table, kept = [5, 0, 3], [1, 2, 17, 18, 30, 40]
    pace.pace_kv_compact(cache, [0, 41], _ids([45]), _ids([table]), cu_rows=[0, 6], rows=_ids(kept))
    for c, s, w, size in zip(codes, scales, was, (1.0, 0.5)):
        values, want = DECODE[w.cpu().numpy()], np.full((n_pages, layers, heads, 1), size)
        for l in range(layers):
            v, t = values[:, l].copy(), want[:, l].copy()
            O.kv_compact(v, t, table, table, 4, kept)
            np.testing.assert_array_equal(DECODE[c[:, l].cpu().numpy()][5, :, :10], v[5, :, :10])
            np.testing.assert_array_equal(s[:, l].cpu().numpy(), t)
        assert torch.equal(c[:, :, :, 10:], w[:, :, :, 10:]) and torch.equal(c[[0, 1, 2, 3, 4, 6]], w[[0, 1, 2, 3, 4, 6]])


def test_replayed(pace):  # noqa: F811
    """A captured call reads the lengths, lists and counts that the arrays hold at the replay."""
    nodes = (26, 12)
    case = Case(pace, 42, (100, 80), nodes, (5, 4), 2, 64, 16, away=True)
    cu = _cu(nodes)
    rows, counts, out = _ids(np.zeros(cu[-1])), _ids([0, 0]), _ids([0, 0])
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        pace.pace_kv_compact(case.cache, cu, case.dev_lens, case.table, rows=rows, counts=counts, dst_table=case.dst, new_lens=out)
    full = np.full(cu[-1], -1)
    for b, k in enumerate(case.kept):
        full[cu[b]:cu[b] + len(k)] = k + cu[b]
    rows.copy_(_ids(full)), counts.copy_(_ids([5, 4]))
    g.replay()
    case.check(out)


def test_a_step_of_drafts(pace):  # noqa: F811
    """Append a tree, attend from it, walk, close up, and append the next: as if the accepted tokens had been appended alone."""
    hq, hkv, dim, page, nodes = 8, 2, 64, 16, [26, 13]
    before = [75, 40]
    pool = Pool(pace, 43, [n + 60 for n in before], hkv, dim, page, poison=False)
    plain = Pool(pace, 43, [n + 60 for n in before], hkv, dim, page, poison=False)
    cu, n = _cu(nodes), sum(nodes)
    lens = _ids([a + m for a, m in zip(before, nodes)])
    rng = np.random.default_rng(44)
    parents = [[-1] + [int(rng.integers(0, t)) for t in range(1, m)] for m in nodes]
    tokens, picked = rng.integers(0, 3, n), rng.integers(0, 3, n)
    # every token of the size of the block's largest, so that no scale grows and no code is rounded twice
    K, V = (torch.sign(_tokens(45 + i, n, hkv, dim)) for i in range(2))
    Q = _tokens(47, n, hq, dim)
    for p in (pool, plain):
        for m in "kv":
            p.raw[m][:], p.s[m][:] = 0x38, 1.0
        _upload(p)
    pace.pace_kv_append(pool.cache, K, V, cu, lens, pool.table)
    out = pace.pace_kv_tree_attention(pool.cache, Q, cu, _ids(sum(parents, [])), lens, pool.table, 135)
    rows, counts, _ = pace.pace_draft_accept(_ids(tokens), _ids(sum(parents, [])), _ids(picked), cu)
    now = pace.pace_kv_compact(pool.cache, cu, lens, pool.table, rows=rows, counts=counts)
    paths = [O.draft_accept(tokens[cu[b]:cu[b + 1]], parents[b], picked[cu[b]:cu[b + 1]]) for b in range(2)]
    assert now.tolist() == [a + len(p) for a, p in zip(before, paths)] and max(map(len, paths)) > 1
    pick = np.concatenate([np.array(p) + cu[b] for b, p in enumerate(paths)])
    few = _cu([len(p) for p in paths])
    pace.pace_kv_append(plain.cache, K, V, few, now, plain.table, rows=_ids(pick))
    for m in "kv":
        (a, s), (b, t) = pool.now(m), plain.now(m)
        for i in range(2):
            x, y = (O.kv_read(DECODE[c], f, pool.pages[i], now.tolist()[i]) for c, f in ((a, s), (b, t)))
            np.testing.assert_array_equal(x, y)
    # and the accepted nodes' outputs are what they would have been in a line
    line = pace.pace_kv_attention(plain.cache, Q[torch.from_numpy(pick).cuda()], few, now, plain.table, 135)
    np.testing.assert_allclose(_f64(out)[pick], _f64(line), rtol=2.0 ** -7, atol=2.0 ** -7)


@pytest.mark.parametrize("away", [False, True])
def test_zeros_under_a_large_scale_join_a_small_one(pace, away):  # noqa: F811
    """A block of zeros (of either sign) may have any scale: its tokens are zeros still beside others 2^150 below."""
    case = Case(pace, 48, (96,), (96,), (40,), 2, 64, 16, away=away)
    pool, pages = case.pools[0], case.source[0]
    for n in "kv":
        pool.raw[n][pages[2]] = np.where(pool.raw[n][pages[2]] & 1, 0x80, 0)
        pool.s[n][pages] = 2.0 ** -40
        pool.s[n][pages[2]] = 2.0 ** 110
    _upload(pool)
    case.check(case.call())


def test_a_layer_is_listed_once(pace):  # noqa: F811
    caches = [Pool(pace, 49, [20], 1, 64, 16).cache for _ in range(2)]
    pace.KvLayers(caches)
    with pytest.raises(ValueError):
        pace.KvLayers([caches[0], caches[1], caches[0]])


@pytest.mark.parametrize("away", [False, True])
def test_scales_that_are_no_powers_of_two(pace, away):  # noqa: F811
    """Of another program's cache: 3/2 of a power, under which a code's product has six significant bits at most and is rounded once."""
    case = Case(pace, 50, (130, 77), (100, 77), (40, 30), 2, 64, 32, away=away)
    for n in "kv":
        case.pools[0].s[n][::2] *= 1.5
    _upload(case.pools[0])
    case.check(case.call())


def test_the_largest_values(pace):  # noqa: F811
    """The largest bf16 is stored as 256 under 2^120, past what 32 bits hold: it stays what it is."""
    pool = Pool(pace, 51, [40], 2, 64, 16, poison=False)
    x = torch.full((40, 2, 64), 3.3895e38, dtype=torch.bfloat16, device="cuda")
    x[::2] = -x[::2] * 0.5
    pace.pace_kv_append(pool.cache, x, x, [0, 40], pool.lens, pool.table)
    was = pool.now("k")
    kept = [1, 3, 4, 21, 39]
    lens = pace.pace_kv_compact(pool.cache, [0, 40], pool.lens, pool.table, cu_rows=[0, 5], rows=_ids(kept))
    codes, scales = pool.now("k")
    page = pool.pages[0]
    assert lens.tolist() == [5] and (scales[page[0]] == 2.0 ** 120).all()
    for i, j in enumerate(kept):
        assert np.array_equal(codes[page[0], :, i], was[0][page[j // 16], :, j % 16])
    assert pace.pace_device_status(clear=True) == (0, 0)
