"""Attention over the paged cache where its running maximum has to follow, and where hidden blocks hold nonsense scales."""
import math

import numpy as np
import pytest
import torch

from test_gpu_kv import BF16, DECODE, Pool, _tokens, _upload, check_attention, pace  # noqa: F401

pytestmark = pytest.mark.gpu


def _codes(x):
    return torch.from_numpy(x).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


# Scores of 2^-60 to 2^60 that climb, fall or jump along the sequence, other rows seeing them the other way round or a tenth
# as steep: the maximum that a row's weights are relative to is overtaken again and again, at every place of a tile.
@pytest.mark.parametrize("shape", ["rise", "fall", "saw", "steps"])
@pytest.mark.parametrize("hq,hkv,dim", [(14, 2, 128), (8, 8, 64), (28, 1, 128)])
@pytest.mark.parametrize("count", [1, 3, 90])
def test_scores_that_climb(pace, shape, hq, hkv, dim, count):  # noqa: F811
    length = 1300
    pool = Pool(pace, 30, [length], hkv, dim, 64, spread=3)
    j = np.arange(length)
    curve = {"rise": j / length * 2 - 1, "fall": 1 - j / length * 2, "saw": (j % 170) / 170 * (0.2 + 0.8 * j / length),
             "steps": np.floor(j / 97) / np.floor(length / 97) * np.where(j % 97 == 50, 1, 0.9)}[shape]
    rng = np.random.default_rng(31)
    u = rng.choice([-1.0, 1.0], size=(hkv, dim))
    size = 60 * math.log(2) / math.sqrt(dim)      # of an element, for a score of 60 in base 2
    for p, page in enumerate(pool.pages[0]):
        at = np.arange(64 * p, min(64 * p + 64, length))
        pool.s["k"][page] = np.where(np.arange(4)[None, :] * 16 + 64 * p < length, 2.0 ** -5, np.nan)
        pool.raw["k"][page, :, :len(at)] = _codes(u[:, None, :] * (size * curve[at])[None, :, None] * 2.0 ** 5)
    _upload(pool)
    steep = np.resize([1.0, -1.0, 0.125, 0.5, -0.25], count * hq).reshape(count, hq, 1)
    Q = torch.from_numpy(steep * np.repeat(u, hq // hkv, axis=0)[None]).to(BF16).cuda()
    check_attention(pace, pool, Q, [count])


# scales of blocks that no query of the call sees, whatever they are
@pytest.mark.parametrize("nonsense", [math.nan, math.inf, -math.inf, -1.0, 0.0, 3e38, 1e-45])
@pytest.mark.parametrize("count,hq", [(1, 14), (4, 14), (70, 14)])
@pytest.mark.parametrize("dim", [64, 128])
def test_nonsense_scales_of_hidden_blocks_reach_nobody(pace, nonsense, count, hq, dim):  # noqa: F811
    length, window, sinks = 700, 90, 3
    pool = Pool(pace, 32, [length], 2, dim, 32)
    Q = _tokens(33, count, hq, dim)
    args = (pool.cache, Q, [0, count], pool.lens, pool.table, length)
    clean = pace.pace_kv_attention(*args, window=window, sinks=sinks).clone()
    last = length - count - window      # slot that the first query sees no more
    for n in "kv":
        for block in range(1, (last + 1) // 16):      # (block 0 holds the sinks)
            pool.s[n][pool.pages[0][block // 2], :, block % 2] = nonsense
    _upload(pool)
    got = pace.pace_kv_attention(*args, window=window, sinks=sinks)
    assert torch.isfinite(got.float()).all()
    assert torch.equal(got, clean)


# a NaN scale that only the last tokens of a call see stays with them
@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("count,hq", [(20, 2), (40, 14)])
@pytest.mark.parametrize("dim", [64, 128])
def test_nan_scale_of_the_newest_block(pace, which, count, hq, dim):  # noqa: F811
    length = 336      # ends a block: its 16 slots are the last queries' own
    pool = Pool(pace, 34, [length], 2, dim, 32)
    Q = _tokens(35, count, hq, dim)
    args = (pool.cache, Q, [0, count], pool.lens, pool.table, length)
    clean = pace.pace_kv_attention(*args).clone()
    pool.s[which][pool.pages[0][(length - 16) // 32], :, (length - 16) % 32 // 16] = math.nan
    _upload(pool)
    got = pace.pace_kv_attention(*args)
    assert torch.equal(got[:count - 16], clean[:count - 16])
    assert torch.isnan(got[count - 16:]).any(dim=2).all()
