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


# a window of the whole range of its type leaves nothing out, for sequences that are shorter than their queries too
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 40, 2 ** 30, 400, -2 ** 31])
@pytest.mark.parametrize("sinks", [0, 4, 2 ** 31 - 1])
@pytest.mark.parametrize("count,hq,dim", [(4, 4, 64), (5, 14, 128), (90, 14, 64), (300, 4, 128)])
def test_windows_without_end(pace, window, sinks, count, hq, dim):  # noqa: F811
    lens = [max(count - short, 0) for short in (0, 1, 2, 3, 60)] + [400]
    pool = Pool(pace, 38, lens, 2, dim, 32)
    Q = _tokens(39, len(lens) * count, hq, dim)
    args = (pool.cache, Q, [count * i for i in range(len(lens) + 1)], pool.lens, pool.table, 400)
    lse, other = (torch.empty(len(Q), hq, device="cuda") for _ in range(2))
    want = pace.pace_kv_attention(*args, lse=lse)
    got = pace.pace_kv_attention(*args, window=window, sinks=sinks, lse=other)
    assert torch.equal(got, want) and torch.equal(other, lse)
    assert want.any(dim=2).all(dim=1).sum() == sum(min(n, count) for n in lens)      # (every query that has a slot sees something)
