"""Attention over the paged cache in a window: pages that are gone, windows of any size."""
import pytest
import torch

from test_gpu_kv import Pool, _tokens, pace  # noqa: F401

pytestmark = pytest.mark.gpu


# pages that no query of the call looks at may be gone from the table: no error, and the others' results stay
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("window,sinks", [(90, 3), (40, 0), (1, 20), (300, 130)])
@pytest.mark.parametrize("count,hq,dim", [(1, 14, 128), (4, 14, 64), (70, 14, 64), (200, 4, 128)])
def test_pages_freed_behind_the_window(pace, page, window, sinks, count, hq, dim):  # noqa: F811
    lens = [700, 1203]
    pool = Pool(pace, 36, lens, 2, dim, page)
    Q = _tokens(37, 2 * count, hq, dim)
    args = (pool.cache, Q, [0, count, 2 * count], pool.lens)
    kw = dict(window=window, sinks=sinks)
    clean = pace.pace_kv_attention(*args, pool.table, max(lens), **kw).clone()
    assert pace.pace_device_status(clear=True)[0] == 0
    table, gone = pool.table.clone(), 0
    for b, n in enumerate(lens):
        for i in range(-(-sinks // page), (n - count - window + 1) // page):      # all its slots hidden from the first query on
            table[b, i] = -1
            gone += 1
    assert gone > 0
    got = pace.pace_kv_attention(*args, table, max(lens), **kw)
    assert pace.pace_device_status(clear=True) == (0, 0)
    assert torch.equal(got, clean)
