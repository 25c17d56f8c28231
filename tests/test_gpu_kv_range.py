"""Attention over the paged cache at scores of every size that 32 bits hold.

Keys are code * (+-1, the same pattern in every slot) and queries a power of two on that pattern, so scores are whole multiples of one
number: equal codes give equal scores to the last bit, in the kernels and in 64 bits, and where scores are large others are too far
away to count.  So the weights have no error of their scores in them, and the bounds here leave none for it."""
import math

import numpy as np
import pytest
import torch

from oracle import pace_oracle as O
from test_gpu_kv import BF16, Pool, _cu, _f64, _tokens, _upload, check_attention, pace  # noqa: F401

pytestmark = pytest.mark.gpu


def _codes(x):
    return torch.from_numpy(x).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


def _set_keys(pool, pattern, curve, exponent):
    """Key j is curve[j], as a code, times the pattern [heads, D] times 2^exponent."""
    page_size = pool.raw["k"].shape[2]
    for p, page in enumerate(pool.pages[0]):
        at = np.arange(page_size * p, min(page_size * (p + 1), len(curve)))
        blocks = -(-len(at) // 16)
        pool.s["k"][page, :, :blocks] = 2.0 ** exponent
        pool.raw["k"][page, :, :len(at)] = _codes(pattern[:, None, :] * curve[at][None, :, None])


def check_exact_scores(P, pool, Q, count, scale, window=0, sinks=0):
    """out and lse of one sequence's last `count` queries.

    out: one rounding to bf16 (2^-9) and weights of 8 bits (2^-9 each, of numerator and denominator alike), twice over for the joins in
    fp32; what is far below the largest is off by 2^-18 of that.  lse: five roundings to fp32 (the scale, the score, the sum of two terms, a
    constant and the product with it)."""
    n, hq, _ = Q.shape
    scale = float(np.float32(scale))
    length = pool.host_lens[0]
    lse = torch.full((n, hq), 7.0, device="cuda")
    out = P.pace_kv_attention(pool.cache, Q, _cu([count]), pool.lens, pool.table, length, scale=scale, window=window, sinks=sinks, lse=lse)
    see = O.kv_visible(length, count, window, sinks)
    r = O.kv_attention(_f64(Q), pool.read("k", 0), pool.read("v", 0), see, scale)
    err = np.abs(_f64(out) - r["out"])
    tol = 2.0 ** -8 * np.abs(r["out"]) + 2.0 ** -8 * r["abs_out"] + 2.0 ** -17 * r["peak"][..., None]
    assert np.all(err <= tol), (float((err - tol).max()), float(err.max()))
    off = np.abs(lse.cpu().numpy().astype(np.float64) - r["lse"])
    assert np.all(off <= 2.0 ** -21 * np.abs(r["lse"]) + 2.0 ** -18), float(off.max())
    return out


def _pattern(heads, dim):
    return np.random.default_rng(40).choice([-1.0, 1.0], size=(heads, dim))


# Equal scores in two CTAs' parts, with 128 and 80 slots: the parts weigh as their slots do, however large the score
@pytest.mark.parametrize("log2_score", [4, 18, 21])
@pytest.mark.parametrize("count,group", [(1, 4), (30, 2)])
@pytest.mark.parametrize("dim", [64, 128])
def test_parts_of_equal_scores(pace, log2_score, count, group, dim):  # noqa: F811
    length = 128 + 80
    pool = Pool(pace, 41, [length], 1, dim, 16)
    u = _pattern(1, dim)
    _set_keys(pool, u, np.full(length, 1.375), 0)
    for p, page in enumerate(pool.pages[0]):      # values near 1 in the first tile, near -1 in the second
        pool.raw["v"][page] = _codes((1 if p < 8 else -1) * np.random.default_rng(p).choice([1.0, 1.125, 1.25], size=pool.raw["v"][page].shape))
        pool.s["v"][page] = 1.0
    _upload(pool)
    Q = torch.from_numpy(np.broadcast_to(u, (count, group, dim)) * 1.0).to(BF16).cuda()
    check_exact_scores(pace, pool, Q, count, math.log(2) * 2.0 ** log2_score / dim)


def _any_size(P, shape, log2_size, mantissa, count, hq, hkv, dim):
    length = 1300
    pool = Pool(P, 42, [length], hkv, dim, 64, spread=8)
    j = np.arange(length)
    curve = {"rise": j / length * 2 - 1, "fall": 1 - j / length * 2, "saw": (j % 170) / 170 * (0.2 + 0.8 * j / length),
             "steps": np.floor(j / 97) / np.floor(length / 97) * np.where(j % 97 == 50, 1, 0.9)}[shape]
    u = _pattern(hkv, dim)
    of_scale, of_q = log2_size // 2 - 8, log2_size // 4
    _set_keys(pool, u, curve * 256, log2_size - 8 - of_scale - of_q)
    _upload(pool)
    steep = np.resize([1.0, -1.0, 0.125, 0.5, -0.25], count * hq).reshape(count, hq, 1)
    Q = torch.from_numpy(steep * 2.0 ** of_q * np.repeat(u, hq // hkv, axis=0)[None]).to(BF16).cuda()
    check_exact_scores(P, pool, Q, count, mantissa * math.log(2) * 2.0 ** of_scale / dim)


# Scores in base 2 of up to +-mantissa 2^log2_size that climb, fall or jump along the sequence, other rows the other way round or less
# steep, V scales of 2^-8 to 2^8: a call returns, and what it returns is right, however far the maximum of a row moves
@pytest.mark.parametrize("log2_size,mantissa", [(16, 1.3), (21, 1.9), (23, 1.0), (26, 1.7320508), (28, 1.2345678), (32, 1.0), (40, 1.6), (80, 1.3),
                                                (110, 1.1)])
@pytest.mark.parametrize("shape", ["rise", "fall", "saw", "steps"])
@pytest.mark.parametrize("count,hq,hkv,dim", [(90, 14, 2, 128), (50, 8, 8, 64)])
def test_scores_of_any_size(pace, shape, log2_size, mantissa, count, hq, hkv, dim):  # noqa: F811
    _any_size(pace, shape, log2_size, mantissa, count, hq, hkv, dim)


# likewise where rows are few; from 2^26 to 2^27 a score's last bit is 8
@pytest.mark.parametrize("log2_size,mantissa", [(16, 1.3), (24, 1.2), (26, 1.05), (26, 1.2345678), (26, 1.4142135), (26, 1.7320508), (26, 1.9), (28, 1.3),
                                                (40, 1.6), (110, 1.1)])
@pytest.mark.parametrize("shape", ["rise", "fall", "saw", "steps"])
@pytest.mark.parametrize("count,hq,hkv,dim", [(1, 14, 2, 128), (3, 8, 8, 64), (2, 14, 1, 128)])
def test_scores_of_any_size_few_rows(pace, shape, log2_size, mantissa, count, hq, hkv, dim):  # noqa: F811
    _any_size(pace, shape, log2_size, mantissa, count, hq, hkv, dim)


# a row whose every score is far below 0 (-2^90 to -2^120 in base 2) is still a softmax of them
@pytest.mark.parametrize("log2_size", [90, 98, 101, 110, 120])
@pytest.mark.parametrize("count,hq,hkv,dim", [(1, 14, 2, 128), (2, 14, 1, 64), (50, 8, 2, 64), (90, 14, 2, 128)])
def test_scores_far_below_zero(pace, log2_size, count, hq, hkv, dim):  # noqa: F811
    length = 600
    pool = Pool(pace, 43, [length], hkv, dim, 64)
    u = _pattern(hkv, dim)
    _set_keys(pool, u, np.where(np.arange(length) % 7 == 3, -1.0, -1.5), 40)
    _upload(pool)
    Q = torch.from_numpy(2.0 ** 30 * np.broadcast_to(np.repeat(u, hq // hkv, axis=0)[None], (count, hq, dim))).to(BF16).cuda()
    check_exact_scores(pace, pool, Q, count, math.log(2) * 2.0 ** (log2_size - 70) / dim)


def _heavy_tokens(P, length, weight, size, hq, hkv, dim, tokens=slice(0, 1), count=1):
    """A sequence in which a few tokens draw about `weight` of every head's softmax, each as much, with values `size` times the others'
    (N(0, 1)) in blocks whose scale is theirs; queries."""
    pool = Pool(P, 44, [length], hkv, dim, 64, poison=False)
    rng, page = np.random.default_rng(45), tokens.start // 64
    heavy = (pool.pages[0][page], slice(None), slice(tokens.start - 64 * page, tokens.stop - 64 * page))
    for n in "kv":
        x = rng.normal(size=pool.raw[n].shape).astype(np.float32)
        if n == "k":
            x[..., 0] = 0      # channel 0 is theirs alone
            x[heavy] = 0
            x[heavy + (0,)] = 6
        else:
            x[heavy] *= size
        pool.raw[n], pool.s[n] = _codes(x * 64), np.full(pool.s[n].shape, 2.0 ** -6)
    _upload(pool)
    lead = math.log(weight / (1 - weight)) + math.log(length / (tokens.stop - tokens.start)) + 0.5      # a softmax of N(0, 1) scores sums up to about length e^(1/2)
    g = torch.Generator().manual_seed(46)
    Q = torch.randn(count, hq, dim, generator=g)
    Q[..., 0] = lead * math.sqrt(dim) / 6
    return pool, Q.to(BF16).cuda()


def check_in_norm(P, pool, Q, bits, floor, copies):
    """The output's error over all its elements (2-norm): every weight is rounded by itself to `bits` bits, 2^-(bits + 1) of it at most, or to
    `floor` of the largest (scales are all alike here), and the output once to bf16, so it is at most
    2^-9 |out| + 2^-(bits + 1) |sqrt(sum_j (p_j v_j)^2)| + floor |max p sqrt(sum_j v_j^2)|; twice that for joins and sums.

    The sequence is called for `copies` times at once, so many that a copy is walked in one piece or two."""
    length, n = pool.host_lens[0], len(Q)
    got = P.pace_kv_attention(pool.cache, Q.repeat(copies, 1, 1), [n * i for i in range(copies + 1)], pool.lens.repeat(copies),
                              pool.table.repeat(copies, 1), length)
    k, v = pool.read("k", 0), pool.read("v", 0)
    see = O.kv_visible(length, n)
    scale = Q.shape[2] ** -0.5
    r = O.kv_attention(_f64(Q), k, v, see, scale)
    group = Q.shape[1] // k.shape[1]
    each = np.zeros(r["out"].shape)
    for t in range(n):
        for h in range(Q.shape[1]):
            s = np.where(see[t], scale * (k[:, h // group] @ _f64(Q)[t, h]), -np.inf)
            p, v2 = np.exp(s - r["lse"][t, h]), v[:, h // group] ** 2
            each[t, h] = 2.0 ** -(bits + 1) * np.sqrt(p ** 2 @ v2) + floor * p.max() * np.sqrt(v2.sum(0))
    err = max(np.linalg.norm(_f64(x) - r["out"]) for x in got.split(n))
    size = np.linalg.norm(r["out"])
    bound = 2 * (2.0 ** -9 * size + np.linalg.norm(each))
    assert err <= bound, (err / size, bound / size)


# a first token that draws most of the weight and has next to no value: the others make up the output
@pytest.mark.parametrize("weight,size", [(0.3, 0.02), (0.6, 0.02), (0.6, 0.002), (0.9, 0.002), (0.99, 0.0002)])
@pytest.mark.parametrize("length,hq,hkv,dim", [(10825, 14, 2, 128), (28000, 8, 1, 128), (20011, 16, 1, 64), (20011, 32, 1, 64)])
def test_first_token_draws_the_weight(pace, weight, size, length, hq, hkv, dim):  # noqa: F811
    check_in_norm(pace, *_heavy_tokens(pace, length, weight, size, hq, hkv, dim), bits=8, floor=2.0 ** -31, copies=152 // hkv + 3)


# the same where rows are many, and with 64 such tokens behind 64 others: the weights of the 64 first slots are passed by 2^9, all at once
@pytest.mark.parametrize("weight,size,tokens", [(0.3, 0.02, slice(0, 1)), (0.9, 0.002, slice(0, 1)), (0.8, 0.002, slice(64, 128)),
                                                (0.95, 0.002, slice(64, 128)), (0.99, 0.0002, slice(64, 128))])
@pytest.mark.parametrize("length,count,hq,hkv,dim", [(20011, 17, 2, 1, 128), (12000, 10, 8, 2, 64)])
def test_few_tokens_draw_the_weight_of_many_rows(pace, weight, size, tokens, length, count, hq, hkv, dim):  # noqa: F811
    check_in_norm(pace, *_heavy_tokens(pace, length, weight, size, hq, hkv, dim, tokens, count), bits=11, floor=2.0 ** -24, copies=152 // hkv + 3)


# One channel of q stands out by far, and the keys have nothing there: the others' bits are all that scores are made of.  (With a window of
# one slot lse is the score.)  Elements under 2^-13 of the largest are off by 2^-21 of it at most; a score is a sum of D products in fp32.
@pytest.mark.parametrize("outlier", [100.0, 300.0, 1024.0, 3000.0, 8192.0])
@pytest.mark.parametrize("count,hq,hkv", [(4, 8, 2), (60, 8, 2), (33, 2, 2)])
@pytest.mark.parametrize("dim", [64, 128])
def test_queries_with_an_outlying_channel(pace, outlier, count, hq, hkv, dim):  # noqa: F811
    length = 300
    pool = Pool(pace, 47, [length], hkv, dim, 32, poison=False)
    x = np.random.default_rng(48).normal(size=pool.raw["k"].shape).astype(np.float32)
    x[..., 5] = 0
    pool.raw["k"], pool.s["k"] = _codes(x * 64), np.full(pool.s["k"].shape, 2.0 ** -6)
    _upload(pool)
    Q = torch.randn(count, hq, dim, generator=torch.Generator().manual_seed(49))
    Q[..., 5] = outlier
    Q = Q.to(BF16).cuda()
    k, q, scale = pool.read("k", 0), _f64(Q), dim ** -0.5
    for window in (1, 0):
        see = O.kv_visible(length, count, window, 0)
        lse = torch.empty(count, hq, device="cuda")
        out = pace.pace_kv_attention(pool.cache, Q, [0, count], pool.lens, pool.table, length, window=window, lse=lse)
        r = O.kv_attention(q, k, pool.read("v", 0), see, scale)
        most = np.abs(k[length - count if window else 0:]).sum(2).max(0).repeat(hq // hkv)      # of the slots seen, sum_d |k_d|
        score = scale * 2.0 ** -21 * outlier * most + 2.0 ** -23 * (dim + 8) * r["abs_score"] + 2.0 ** -20
        off = np.abs(lse.cpu().numpy() - r["lse"])
        assert np.all(off <= score + 2.0 ** -21 * np.abs(r["lse"])), float((off / score).max())
        tol = 2.0 ** -8 * np.abs(r["out"]) + (2.0 ** -8 + 2 * score[..., None]) * r["abs_out"] + 2.0 ** -17 * r["peak"][..., None]
        assert np.all(np.abs(_f64(out) - r["out"]) <= tol)


# V scales of blocks up to 2^80 apart: neither the sum of the weights nor the large blocks' part of the output suffers
@pytest.mark.parametrize("lens,new", [((900, 300), (1, 2)), ((400,), (120,)), ((2000, 70), (70, 3))])
@pytest.mark.parametrize("dim", [64, 128])
def test_v_scales_far_apart(pace, lens, new, dim):  # noqa: F811
    pool = Pool(pace, 50, list(lens), 2, dim, 16)
    pool.s["v"] = pool.s["v"] * 2.0 ** np.random.default_rng(51).integers(-40, 41, pool.s["v"].shape)
    _upload(pool)
    check_attention(pace, pool, _tokens(52, sum(new), 14, dim), list(new))
