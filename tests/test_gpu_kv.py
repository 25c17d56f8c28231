"""The paged 8-bit cache on the GPU against the fp64 oracle: append (rotation, gather, block scales) and attention."""
import math

import numpy as np
import pytest
import torch

from oracle import pace_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pace():
    from paper_2608_27206_gb300 import build
    build.build()
    from paper_2608_27206_gb300 import pace as P
    P.pace_init(0)
    P.pace_device_status(clear=True)
    yield P
    assert P.pace_device_status(clear=True)[0] == 0


DECODE = O.e4m3_values()
BF16 = torch.bfloat16


def _cu(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int32)


def _f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Pool:
    """A cache of random codes whose pages belong to sequences of `lens` tokens in shuffled order; what no token of a
    sequence covers is NaN, codes and scales."""

    def __init__(self, P, seed, lens, heads, dim, page, poison=True, spread=0):
        rng = np.random.default_rng(seed)
        need = [-(-n // page) for n in lens]
        n_pages = sum(need) + 2
        order = rng.permutation(n_pages)
        self.pages, at = [], 0
        for n in need:
            self.pages.append(order[at:at + n].astype(np.int64))
            at += n
        table = np.full((len(lens), max(need + [1])), -7, np.int32)
        for b, p in enumerate(self.pages):
            table[b, :len(p)] = p
        self.raw, self.s = {}, {}
        for n in "kv":
            x = rng.normal(size=(n_pages, heads, page, dim)) * np.exp(0.5 * rng.normal(size=(n_pages, 1, page, 1)))
            blk = x.reshape(n_pages, heads, page // 16, 16 * dim)
            s = O.kv_scale(np.abs(blk).max(3)) * 2.0 ** rng.integers(-spread, spread + 1, blk.shape[:3])
            codes = torch.from_numpy((blk / s[..., None]).reshape(x.shape)).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
            if poison:
                free = np.ones((n_pages, page), bool)
                for b, p in enumerate(self.pages):
                    for i, pg in enumerate(p):
                        free[pg, :max(0, min(page, lens[b] - i * page))] = False
                codes = np.where(free[:, None, :, None], 0x7F, codes).astype(np.uint8)
                s = np.where(free[:, None, ::16], np.nan, s)
            self.raw[n], self.s[n] = codes, s
        self.dev = {n: (torch.from_numpy(self.raw[n]).cuda().view(torch.float8_e4m3fn),
                        torch.from_numpy(self.s[n].astype(np.float32)).cuda()) for n in "kv"}
        self.cache = P.KvCache(self.dev["k"][0], self.dev["v"][0], self.dev["k"][1], self.dev["v"][1])
        self.table = torch.from_numpy(table).cuda()
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.host_lens = list(lens)

    def values(self, n):
        return DECODE[self.raw[n]]

    def read(self, n, b):
        return O.kv_read(self.values(n), self.s[n], self.pages[b], self.host_lens[b])

    def now(self, n):
        """(codes, scales) as they are on the device."""
        return self.dev[n][0].view(torch.uint8).cpu().numpy(), self.dev[n][1].cpu().numpy().astype(np.float64)


def _tokens(seed, rows, heads, dim):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, heads, dim, generator=g) * torch.exp(0.5 * torch.randn(rows, 1, 1, generator=g))
    return x.to(BF16).cuda()


# ---- append ----------------------------------------------------------------------------------
def check_append(pool, new, K, V, rows=None, cs=None):
    """The cache on the device against the oracle's; the pool's own copies take the oracle's values."""
    cu = _cu(new)
    pick = np.arange(cu[-1]) if rows is None else rows
    for n, x, turn in (("k", _f64(K)[pick], cs), ("v", _f64(V)[pick], None)):
        y = x if turn is None else O.rope_rotate(x, turn[..., 0], turn[..., 1])
        values, scales = pool.values(n).copy(), pool.s[n].copy()
        exact = np.full(values.shape, np.nan)       # new tokens' unrounded values over their scale
        slack = np.zeros(values.shape)
        for b, count in enumerate(new):
            if count == 0:
                continue
            first = pool.host_lens[b] - count
            O.kv_append(values, scales, y[cu[b]:cu[b + 1]], first, pool.pages[b])
        page = values.shape[2]
        size = np.abs(x[..., :x.shape[2] // 2]) + np.abs(x[..., x.shape[2] // 2:])
        for b, count in enumerate(new):
            for i in range(count):
                slot = pool.host_lens[b] - count + i
                pg, at = pool.pages[b][slot // page], slot % page
                s = scales[pg, :, at // 16][:, None]
                exact[pg, :, at] = y[cu[b] + i] / s
                # a rotated value is off by three roundings of at most |x1| + |x2|
                slack[pg, :, at] = 0 if turn is None else np.tile(size[cu[b] + i], 2) * 3 * 2.0 ** -24 / s
        codes, got_s = pool.now(n)
        np.testing.assert_array_equal(got_s, scales)
        got = DECODE[codes]
        same = (got == values) | (np.isnan(got) & np.isnan(values))
        near = np.abs(got - exact) <= np.abs(values - exact) + 2 * slack      # either neighbour of a tie
        assert np.all(same | near), int((~(same | near)).sum())
        if turn is None:
            assert same.all()
        untouched = np.isnan(exact) & (values == pool.values(n))
        assert np.array_equal(codes[untouched], pool.raw[n][untouched])
        pool.raw[n], pool.s[n] = codes, got_s


def rotation(P, dim, n, seed, rows_of_ids=3):
    table = P.pace_rope_table(2000, dim, 1e6)
    rng = np.random.default_rng(seed)
    if rows_of_ids == 3:
        sections = [dim // 8, dim // 16 * 3, dim // 16 * 3]
    else:
        sections = [dim // 2]
    pos = rng.integers(0, 2000, (rows_of_ids, n)).astype(np.int32)
    kw = dict(rope=table, positions=torch.from_numpy(pos if rows_of_ids == 3 else pos[0]).cuda(), sections=sections)
    return kw, lambda pick: O.rope_angles(table.cpu().numpy(), pos[:, pick], sections)


# block edges (15, 16, 17 tokens; starts inside a block, behind one), one token, sequences without new ones
@pytest.mark.parametrize("before,new", [((0,), (1,)), ((403,), (1,)), ((0, 15, 16, 17), (17, 1, 16, 15)), ((5, 0, 40), (0, 33, 0)),
                                        ((7, 100), (300, 5)), ((1, 31, 64, 129), (1, 1, 1, 1))])
@pytest.mark.parametrize("heads,dim,page", [(4, 128, 16), (2, 64, 64), (1, 128, 256)])
def test_append(pace, before, new, heads, dim, page):
    lens = [a + b for a, b in zip(before, new)]
    pool = Pool(pace, 1, lens, heads, dim, page)
    for n in "kv":      # the poison of unwritten slots goes: new tokens land there
        pool.raw[n][np.isnan(pool.values(n))] = 0
    _upload(pool)
    n = sum(new)
    K, V = _tokens(2, n, heads, dim), _tokens(3, n, heads, dim)
    kw, angles = rotation(pace, dim, n, 4)
    q = _tokens(5, n, 3 * heads, dim)
    q_out = pace.pace_kv_append(pool.cache, K, V, _cu(new), pool.lens, pool.table, q=q, **kw)
    cs = angles(np.arange(n))
    check_append(pool, new, K, V, cs=cs)
    ref = O.rope_rotate(_f64(q), cs[..., 0], cs[..., 1])
    np.testing.assert_allclose(_f64(q_out), ref, rtol=2.0 ** -8, atol=1e-6)


def _upload(pool):
    for n in "kv":
        pool.dev[n][0].view(torch.uint8).copy_(torch.from_numpy(pool.raw[n]))
        pool.dev[n][1].copy_(torch.from_numpy(pool.s[n].astype(np.float32)))


# gathered rows (any order, repeated), rows of a fused projection, one row of ids, no rotation, queries in place
@pytest.mark.parametrize("case", ["gather", "fused", "one_row_of_ids", "plain", "in_place"])
def test_append_sources(pace, case):
    before, new = (0, 20), (37, 14)
    pool = Pool(pace, 6, [37, 34], 2, 128, 32, poison=False)
    n = 90 if case == "gather" else 51
    x = _tokens(7, n, 10, 128)
    K, V, q = x[:, 6:8], x[:, 8:], x[:, :6]
    if case != "fused":
        K, V, q = K.contiguous(), V.contiguous(), q.contiguous()
    rows = np.random.default_rng(8).integers(0, n, 51).astype(np.int32) if case == "gather" else None
    kw, angles = rotation(pace, 128, n, 9, 1 if case == "one_row_of_ids" else 3)
    if case == "plain":
        kw, angles = {}, lambda pick: None
    pick = np.arange(51) if rows is None else rows
    q0 = _f64(q)[pick]
    q_out = pace.pace_kv_append(pool.cache, K, V, _cu(new), pool.lens, pool.table, q=q, q_out=q if case == "in_place" else None,
                                rows=None if rows is None else torch.from_numpy(rows).cuda(), **kw)
    cs = angles(pick)
    check_append(pool, new, K, V, rows=pick, cs=cs)
    ref = q0 if cs is None else O.rope_rotate(q0, cs[..., 0], cs[..., 1])
    np.testing.assert_allclose(_f64(q_out), ref, rtol=2.0 ** -8, atol=1e-6)


def test_append_again_changes_nothing(pace):
    pool = Pool(pace, 10, [50, 21], 4, 64, 16, poison=False)
    K, V = _tokens(11, 12, 4, 64) * 8, _tokens(12, 12, 4, 64)
    args = (pool.cache, K, V, _cu([5, 7]), pool.lens, pool.table)
    pace.pace_kv_append(*args)
    once = [pool.now(n) for n in "kv"]
    pace.pace_kv_append(*args)
    for a, b in zip(once, [pool.now(n) for n in "kv"]):
        assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


def test_append_token_by_token_with_growing_scales(pace):
    """Each token two and a half times the one before: every append raises its block's scale."""
    pool = Pool(pace, 13, [40], 2, 64, 16, poison=False)
    x = _tokens(14, 40, 2, 64) * (2.5 ** torch.arange(40, device="cuda") * 2.0 ** -30)[:, None, None].to(BF16)
    for i in range(40):
        pool.host_lens = [i + 1]
        pool.lens.fill_(i + 1)
        pace.pace_kv_append(pool.cache, x[i:i + 1], x[i:i + 1].flip(0), [0, 1], pool.lens, pool.table)
        check_append(pool, [1], x[i:i + 1], x[i:i + 1])


# the range of the scales: zeros, subnormal and the largest bf16 values, 448 2^e exactly
def test_append_extreme_values(pace):
    pool = Pool(pace, 15, [96], 1, 64, 16, poison=False)
    x = torch.zeros(96, 1, 64)
    for i, v in enumerate((0.0, 2.0 ** -133, 3.38e38, 448.0, 1.75 * 2.0 ** -60, 2.0 ** -64 * 448)):
        x[16 * i:16 * i + 16] = v * (1 - 2.0 ** -7 * torch.randint(0, 3, (16, 1, 64)).float())
    x = x.to(BF16).cuda()
    pace.pace_kv_append(pool.cache, x, -x, [0, 96], pool.lens, pool.table)
    check_append(pool, [96], x, -x)


def test_append_non_finite_values_are_stored_as_zero_and_reported(pace):
    pool = Pool(pace, 16, [16, 16], 2, 64, 16, poison=False)
    K, V = _tokens(17, 32, 2, 64), _tokens(18, 32, 2, 64)
    bad = K.clone()
    bad[3, 1, 5], bad[20, 0, 60], bad[21, 1, 0] = math.nan, math.inf, -math.inf
    pace.pace_kv_append(pool.cache, bad, V, [0, 16, 32], pool.lens, pool.table)
    assert pace.pace_device_status(clear=True) == (pace.PACE_ERR_INVALID_ARG, 14)
    K[3, 1, 5] = K[20, 0, 60] = K[21, 1, 0] = 0
    check_append(pool, [16, 16], K, V)


# numbers out of range: reported, nothing written for them, the others as they should be
@pytest.mark.parametrize("what", ["page", "page_negative", "row", "position", "short"])
def test_append_numbers_out_of_range(pace, what):
    lens = [20, 20]
    pool = Pool(pace, 19, lens, 2, 64, 16, poison=False)
    n = 40
    K, V = _tokens(20, n, 2, 64), _tokens(21, n, 2, 64)
    kw, angles = rotation(pace, 64, n, 22)
    rows = np.arange(n, dtype=np.int32)
    table, dev_lens = pool.table.clone(), pool.lens.clone()
    before = {k: pool.now(k) for k in "kv"}
    if what.startswith("page"):
        table[0, 1] = len(pool.raw["k"]) if what == "page" else -1
    elif what == "row":
        rows[5] = n
    elif what == "position":
        kw["positions"] = kw["positions"].clone()
        kw["positions"][1, 5] = 2000
    else:
        dev_lens[0] = 12
    pace.pace_kv_append(pool.cache, K, V, [0, 20, 40], dev_lens, table, rows=torch.from_numpy(rows).cuda(), **kw)
    assert pace.pace_device_status(clear=True) == (pace.PACE_ERR_INVALID_ARG, 14)
    # the second sequence alone, from the state before
    after = {k: pool.now(k) for k in "kv"}
    pages = pool.pages[1]
    pace.pace_kv_append(pool.cache, K[20:], V[20:], [0, 20], pool.lens[1:].clone(), pool.table[1:].contiguous(), rope=kw["rope"],
                        positions=pool_positions(kw["positions"], 20), sections=kw["sections"])
    for k in "kv":
        assert np.array_equal(after[k][0][pages], pool.now(k)[0][pages])
        spare = [p for p in range(len(pool.raw[k])) if p not in set(pool.pages[0]) | set(pages)]
        assert np.array_equal(after[k][0][spare], before[k][0][spare])
        if what.startswith("page"):
            assert np.array_equal(after[k][0][pool.pages[0][1]], before[k][0][pool.pages[0][1]])


def pool_positions(positions, start):
    return positions[:, start:].contiguous()


def test_append_more_sequences_than_one_launch_takes(pace):
    new = [1 + i % 3 for i in range(300)]
    lens = [n + i % 19 for i, n in enumerate(new)]
    pool = Pool(pace, 23, lens, 1, 64, 16, poison=False)
    K, V = _tokens(24, sum(new), 1, 64), _tokens(25, sum(new), 1, 64)
    pace.pace_kv_append(pool.cache, K, V, _cu(new), pool.lens, pool.table)
    check_append(pool, new, K, V)


def test_rope_table(pace):
    for dim in (64, 128):
        t = pace.pace_rope_table(70000, dim, 1e6).cpu().numpy()
        a = np.arange(70000)[:, None] * 1e6 ** (-np.arange(dim // 2) * 2.0 / dim)
        # rounded once to fp32; the angles themselves are off by 2^-52 of 70000
        np.testing.assert_allclose(t, np.stack([np.cos(a), np.sin(a)], 2), rtol=0, atol=2.0 ** -25 + 2.0 ** -34)


# ---- attention -------------------------------------------------------------------------------
def check_attention(P, pool, Q, new, window=0, sinks=0, scale=None, **kw):
    """out and lse against the oracle.

    out is rounded once to bf16 (2^-9 of it); each weight is held to 8 bits (2^-9) or, far below the largest weighted
    value, to 2^-18 of that, and carries the error of its score; the output can use up twice those.  A score is a sum of
    D products in fp32: off by at most 2^-23 (D + 8) times the sum of their sizes."""
    cu = _cu(new)
    n, hq, D = Q.shape
    scale = D ** -0.5 if scale is None else scale
    lse = torch.full((max(n, 1), hq), 7.0, device="cuda")
    out = P.pace_kv_attention(pool.cache, Q, cu, pool.lens, pool.table, max(pool.host_lens), scale=scale, window=window, sinks=sinks,
                              lse=lse, **kw)
    q = _f64(Q)
    for b, count in enumerate(new):
        if count == 0:
            continue
        k, v = pool.read("k", b), pool.read("v", b)
        length = pool.host_lens[b]
        see = O.kv_visible(length, count, window, sinks)
        hidden = ~see.any(0)
        k[hidden] = v[hidden] = 0
        r = O.kv_attention(q[cu[b]:cu[b + 1]], k, v, see, scale)
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


# one token to a few thousand slots, edges of tiles and pages
@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 127, 128, 129, 404, 1025, 4099])
@pytest.mark.parametrize("hq,hkv,dim,page", [(28, 4, 128, 16), (14, 2, 64, 64), (8, 8, 128, 256), (32, 1, 64, 128)])
def test_decode(pace, length, hq, hkv, dim, page):
    pool = Pool(pace, length, [length], hkv, dim, page)
    check_attention(pace, pool, _tokens(1, 1, hq, dim), [1])


# ragged batches: empty and one-token sequences among long ones, sequences without queries
@pytest.mark.parametrize("lens,new", [((300, 1, 4000, 17, 129, 640), (1, 1, 1, 1, 1, 1)), ((300, 0, 5, 129), (1, 0, 0, 1)),
                                      ((777, 60, 2500), (4, 3, 1)), ((200,) * 40, (1,) * 40)])
@pytest.mark.parametrize("hq,hkv,dim,page", [(28, 4, 128, 64), (16, 2, 128, 32), (14, 2, 64, 16)])
def test_decode_batches(pace, lens, new, hq, hkv, dim, page):
    pool = Pool(pace, 2, list(lens), hkv, dim, page)
    check_attention(pace, pool, _tokens(3, sum(new), hq, dim), list(new))


# group sizes and query counts on both sides of every row-tile edge
@pytest.mark.parametrize("group,count", [(1, 1), (1, 2), (1, 8), (1, 9), (3, 5), (5, 3), (4, 4), (7, 2), (8, 4), (7, 5), (33, 1), (64, 1),
                                         (64, 2), (1, 33), (2, 64), (7, 37)])
@pytest.mark.parametrize("dim", [64, 128])
def test_row_counts(pace, group, count, dim):
    pool = Pool(pace, 4, [count + 150, count + 3], 2, dim, 32)
    check_attention(pace, pool, _tokens(5, 2 * count, 2 * group, dim), [count, count])


# prefill: whole and behind earlier tokens, ragged, edges of tiles
@pytest.mark.parametrize("lens,new", [((64,), (64,)), ((130,), (130,)), ((513,), (513,)), ((700, 33, 300), (700, 20, 257)),
                                      ((1100, 40), (129, 1))])
@pytest.mark.parametrize("hq,hkv,dim,page", [(14, 2, 128, 64), (4, 2, 64, 16)])
def test_prefill(pace, lens, new, hq, hkv, dim, page):
    pool = Pool(pace, 6, list(lens), hkv, dim, page)
    check_attention(pace, pool, _tokens(7, sum(new), hq, dim), list(new))


# windows: one slot, inside a block, a tile's edge, wider than the sequence; sinks inside and across a block or tile
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 4), (5, 1), (128, 0), (100, 17), (129, 130), (1000, 4), (5000, 4), (300, 2000)])
@pytest.mark.parametrize("lens,new", [((1500, 40, 7), (1, 1, 1)), ((1000, 300), (4, 6)), ((600, 450), (333, 450))])
@pytest.mark.parametrize("hq,hkv,dim", [(14, 2, 128), (4, 2, 64)])
def test_windows(pace, window, sinks, lens, new, hq, hkv, dim):
    pool = Pool(pace, 8, list(lens), hkv, dim, 32)
    check_attention(pace, pool, _tokens(9, sum(new), hq, dim), list(new), window=window, sinks=sinks)


# scales of blocks far apart (2^-12 .. 2^12 of each other), scores of many units
@pytest.mark.parametrize("lens,new", [((900, 300), (1, 2)), ((400,), (120,))])
@pytest.mark.parametrize("gain", [1.0, 30.0])
def test_uneven_scales(pace, lens, new, gain):
    pool = Pool(pace, 10, list(lens), 2, 128, 16, spread=6)
    check_attention(pace, pool, _tokens(11, sum(new), 14, 128) * gain, list(new))


# rows that see nothing: sequences shorter than their queries, empty ones
@pytest.mark.parametrize("count", [1, 3, 90])
def test_rows_that_see_nothing(pace, count):
    lens = [0, 2, count + 40]
    pool = Pool(pace, 12, lens, 2, 64, 16)
    Q = _tokens(13, 3 * count, 8, 64)
    lse = torch.full((3 * count, 8), 7.0, device="cuda")
    out = pace.pace_kv_attention(pool.cache, Q, _cu([count] * 3), pool.lens, pool.table, max(lens), lse=lse)
    none = count + max(0, count - 2)
    assert not out[:none].any() and torch.isneginf(lse[:none]).all()
    pool2 = Pool(pace, 12, lens, 2, 64, 16)
    seen = min(2, count)
    for b, length, rows in ((1, 2, slice(2 * count - seen, 2 * count)), (2, count + 40, slice(2 * count, 3 * count))):
        n = rows.stop - rows.start
        alone = pace.pace_kv_attention(pool2.cache, Q[rows].contiguous(), [0, n], pool2.lens[b:b + 1].clone(),
                                       pool2.table[b:b + 1].contiguous(), length)
        np.testing.assert_allclose(_f64(out[rows]), _f64(alone), rtol=2.0 ** -7, atol=2.0 ** -7)


# NaN where a query does not look: before the window, behind a query inside its own call's tokens
@pytest.mark.parametrize("count,hq", [(1, 14), (4, 14), (8, 4), (70, 14), (200, 4)])
@pytest.mark.parametrize("dim", [64, 128])
def test_nan_in_hidden_slots_reaches_nobody(pace, count, hq, dim):
    length, window, sinks = 700, 90, 3
    pool = Pool(pace, 14, [length], 2, dim, 32)
    Q = _tokens(15, count, hq, dim)
    clean = pace.pace_kv_attention(pool.cache, Q, [0, count], pool.lens, pool.table, length, window=window, sinks=sinks).clone()
    first = length - count
    hidden = list(range(sinks, first - window + 1))
    for n in "kv":
        for j in hidden:
            pool.raw[n][pool.pages[0][j // 32], :, j % 32] = 0x7F if j % 2 else 0xFF
    if count > 1:     # the last token, which all queries but the last do not see
        j = length - 1
        pool.raw["k"][pool.pages[0][j // 32], 0, j % 32] = 0x7F
        pool.raw["v"][pool.pages[0][j // 32], 1, j % 32, 5] = 0x7F
    _upload(pool)
    got = pace.pace_kv_attention(pool.cache, Q, [0, count], pool.lens, pool.table, length, window=window, sinks=sinks)
    until = count - 1 if count > 1 else count
    assert torch.equal(got[:until], clean[:until])
    if count > 1:
        assert torch.isnan(got[-1, 0]).all() and torch.isnan(got[-1, hq // 2, 5])


def test_pages_far_apart(pace):
    """Offsets past 32 bits: pages 96 MB apart in one allocation that holds k and v of a layer side by side."""
    heads, dim, page, n = 2, 128, 64, 48
    stride = 96 << 20
    buf = torch.zeros(n * stride, dtype=torch.uint8, device="cuda")
    shape, inner = (n, heads, page, dim), (page * dim, dim, 1)
    k = torch.as_strided(buf, shape, (stride,) + inner)
    v = torch.as_strided(buf, shape, (stride,) + inner, storage_offset=heads * page * dim)
    scales = torch.zeros(n, 4, heads, page // 16, device="cuda")
    cache = pace.KvCache(k, v, scales[:, 0], scales[:, 1])
    length = n * page - 5
    table = torch.arange(n, dtype=torch.int32, device="cuda").flip(0)[None].contiguous()
    lens = torch.tensor([length], dtype=torch.int32, device="cuda")
    K, V = _tokens(16, length, heads, dim), _tokens(17, length, heads, dim)
    pace.pace_kv_append(cache, K, V, [0, length], lens, table)
    small = pace.KvCache(k.contiguous(), v.contiguous(), scales[:, 0].contiguous(), scales[:, 1].contiguous())
    assert int((small.k != 0).sum()) > 0.9 * length * heads * dim
    for count in (1, 100):
        Q = _tokens(18, count, 14, dim)
        a = pace.pace_kv_attention(cache, Q, [0, count], lens, table, length)
        b = pace.pace_kv_attention(small, Q, [0, count], lens, table, length)
        assert torch.equal(a, b)


def test_attention_more_sequences_than_one_launch_takes(pace):
    lens = [1 + 7 * i % 90 for i in range(300)]
    pool = Pool(pace, 19, lens, 1, 64, 16)
    check_attention(pace, pool, _tokens(20, 300, 4, 64), [1] * 300)


@pytest.mark.parametrize("count", [1, 60])
def test_attention_numbers_out_of_range(pace, count):
    """A page number or a length out of range is reported; the other sequence's rows stay right."""
    pool = Pool(pace, 21, [300, 250], 2, 64, 16)
    Q = _tokens(22, 2 * count, 4, 64)
    args = ([0, count, 2 * count], pool.lens, pool.table, 300)
    good = pace.pace_kv_attention(pool.cache, Q, *args).clone()
    for page in (len(pool.raw["k"]), -1, 1 << 30):
        table = pool.table.clone()
        table[0, 3] = page
        got = pace.pace_kv_attention(pool.cache, Q, args[0], pool.lens, table, 300)
        assert pace.pace_device_status(clear=True) == (pace.PACE_ERR_INVALID_ARG, 15)
        assert torch.equal(got[count:], good[count:])
    lens = pool.lens.clone()
    lens[0] = 301
    got = pace.pace_kv_attention(pool.cache, Q, args[0], lens, pool.table, 300)
    assert pace.pace_device_status(clear=True) == (pace.PACE_ERR_INVALID_ARG, 15)
    assert torch.equal(got[count:], good[count:])


@pytest.mark.parametrize("lens,new", [((5000, 77, 900), (1, 1, 1)), ((900, 300), (200, 300))])
def test_attention_repeats_bit_for_bit_on_any_stream(pace, lens, new):
    pool = Pool(pace, 23, list(lens), 4, 128, 64)
    Q = _tokens(24, sum(new), 28, 128)
    args = (pool.cache, Q, _cu(new), pool.lens, pool.table, max(lens))
    a = pace.pace_kv_attention(*args).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        b = pace.pace_kv_attention(*args, stream=side)
        side.synchronize()
        assert torch.equal(a, b)


def test_queries_of_a_fused_projection(pace):
    pool = Pool(pace, 25, [200, 90], 2, 128, 32)
    x = _tokens(26, 41, 18, 128)
    for new in ((1, 1), (40, 1)):
        Q = x[:sum(new), :14]
        a = pace.pace_kv_attention(pool.cache, Q, _cu(new), pool.lens, pool.table, 200)
        b = pace.pace_kv_attention(pool.cache, Q.contiguous(), _cu(new), pool.lens, pool.table, 200)
        assert torch.equal(a, b)


def test_captured_decode_steps_follow_growing_sequences(pace):
    """One captured step (append, attention), replayed while seq_lens grow, equals the calls made one by one."""
    start, steps, B = [30, 100], 40, 2
    pool = Pool(pace, 27, [s + steps for s in start], 2, 128, 16, poison=False)
    x = _tokens(28, B * steps, 18, 128).view(steps, B, 18, 128)
    cur, lens = x[0].clone(), torch.tensor(start, dtype=torch.int32, device="cuda")
    q_out, out = torch.empty(B, 14, 128, dtype=BF16, device="cuda"), torch.empty(B, 14, 128, dtype=BF16, device="cuda")
    rope = pace.pace_rope_table(256, 128)
    pos = torch.zeros(B, dtype=torch.int32, device="cuda")
    most = max(pool.host_lens)
    ws = torch.empty(max(16, pace.pace_kv_attention_workspace_size(pool.cache, [0, 1, 2], 14, most)), dtype=torch.uint8, device="cuda")

    def step(cache):
        lens.add_(1)
        pos.copy_(lens - 1)
        pace.pace_kv_append(cache, cur[:, 14:16], cur[:, 16:], [0, 1, 2], lens, pool.table, rope=rope, positions=pos, q=cur[:, :14],
                            q_out=q_out)
        pace.pace_kv_attention(cache, q_out, [0, 1, 2], lens, pool.table, most, out=out, ws=ws)

    other = pace.KvCache(*[t.clone() for t in (pool.cache.k, pool.cache.v, pool.cache.k_scale, pool.cache.v_scale)])
    eager = []
    for i in range(steps):
        cur.copy_(x[i])
        step(other)
        eager.append(out.clone())
    lens.copy_(torch.tensor(start, dtype=torch.int32))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(pool.cache)
    for i in range(steps):
        cur.copy_(x[i])
        graph.replay()
        assert torch.equal(out, eager[i]), i
    for a, b in ((pool.cache.k, other.k), (pool.cache.v, other.v)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
