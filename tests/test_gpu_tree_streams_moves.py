"""Moves of cached tokens on two streams at once, against the fp64 oracle: every code and scale that they write."""
import numpy as np
import pytest
import torch

from oracle import pace_oracle as O
from test_gpu_kv import DECODE, Pool, pace  # noqa: F401
from test_gpu_kv_compact import _ids

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page,heads,dim", [(16, 2, 64), (64, 4, 128)])
@pytest.mark.parametrize("count", [52, 640])
def test_two_moves_at_once(pace, page, heads, dim, count):  # noqa: F811
    """Both read the same sequence's newest tokens, of which each keeps others, and write pages of their own, over and over."""
    last = 1600 + count      # slots; the newest tokens begin at a page's first
    layers = [Pool(pace, 140 + l, [last, 640, 640], heads, dim, page, poison=False, spread=3) for l in range(2)]
    for p in layers[1:]:      # one block table for all
        p.pages, p.table = layers[0].pages, layers[0].table
    one, first = layers[0], 1600 // page
    rng = np.random.default_rng(3)
    kept = [np.sort(rng.permutation(count)[:k]) for k in (count // 2, count - 7)]
    table, lens = one.table[:1].contiguous(), _ids([last])
    target = [np.concatenate([one.pages[0][:first], one.pages[1 + i]]) for i in range(2)]
    dst = [_ids([t]) for t in target]
    rows, cu = [_ids(k) for k in kept], [[0, len(k)] for k in kept]
    cache = pace.KvLayers([p.cache for p in layers])
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i in range(2):
            got[i].append(pace.pace_kv_compact(cache, [0, count], lens, table, cu_rows=cu[i], rows=rows[i], dst_table=dst[i], stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert [x.tolist() for x in got[i]] == [[1600 + len(kept[i])]] * 20
    for p in layers:
        for n in "kv":
            values, scales = DECODE[p.raw[n]], p.s[n].copy()
            for i in range(2):
                O.kv_compact(values, scales, one.pages[0], target[i], 1600, kept[i])
            codes, now = p.now(n)
            np.testing.assert_array_equal(now, scales)
            free = np.zeros((len(codes), page), bool)      # slots behind the last kept token of a written block
            for i in range(2):
                end = 1600 + len(kept[i])
                for j in range(end, -(-end // 16) * 16):
                    free[target[i][j // page], j % page] = True
            assert ((DECODE[codes] == values) | free[:, None, :, None]).all()
    assert pace.pace_device_status(clear=True) == (0, 0)
