"""Attention from trees in a window with first tokens of any number that stay visible."""
import pytest
import torch

from test_gpu_kv import Pool, _tokens, pace  # noqa: F401
from test_gpu_kv_tree import _ids, check_tree, tree

pytestmark = pytest.mark.gpu

LENS, NODES = [400, 500, 30], [64, 100, 40]      # contexts of 336 and 400 slots, and a sequence shorter than its nodes


def _trees(shape):
    return [tree(shape, n, b) for b, n in enumerate(NODES)]


# more sinks than there are positions, up to the largest that the type holds: every ancestor stays visible, whatever the window; trees that
# branch have nodes whose number is above their depth
@pytest.mark.parametrize("sinks", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 11, 2 ** 31 - 64, 2 ** 31 - 1000, 2 ** 30, 500])
@pytest.mark.parametrize("window", [1, 3])
@pytest.mark.parametrize("shape", ["fours", "forest", "flat", "chain"])
@pytest.mark.parametrize("hq,hkv,dim", [(14, 2, 128), (4, 2, 64)])
def test_sinks_without_end(pace, sinks, window, shape, hq, hkv, dim):  # noqa: F811
    pool = Pool(pace, 120, LENS, hkv, dim, 32)
    Q, parents = _tokens(121, sum(NODES), hq, dim), _trees(shape)
    out, lse = check_tree(pace, pool, Q, parents, window=window, sinks=sinks)
    all_lse = torch.empty_like(lse)
    every = pace.pace_kv_tree_attention(pool.cache, Q, [0, 64, 164, 204], _ids(sum(parents, [])), pool.lens, pool.table, max(LENS), lse=all_lse)
    assert torch.equal(out, every) and torch.equal(lse, all_lse)      # the window leaves nothing out


# few rows to a KV head: trees of up to 16 of them, by themselves
@pytest.mark.parametrize("sinks", [2 ** 31 - 1, 2 ** 31 - 5, 2 ** 30])
@pytest.mark.parametrize("shape", ["fours", "flat"])
@pytest.mark.parametrize("n,hq", [(8, 2), (8, 4), (16, 2)])
def test_sinks_without_end_of_few_rows(pace, sinks, shape, n, hq):  # noqa: F811
    pool = Pool(pace, 122, [300, 70, 5], 2, 64, 16)
    Q, parents = _tokens(123, 3 * n, hq, 64), [tree(shape, n, b) for b in range(3)]
    out, lse = check_tree(pace, pool, Q, parents, window=1, sinks=sinks)
    every = pace.pace_kv_tree_attention(pool.cache, Q, [0, n, 2 * n, 3 * n], _ids(sum(parents, [])), pool.lens, pool.table, 300)
    assert torch.equal(out, every)
