"""Calls for drafted trees on other streams than the current one, and at the same time."""
import pytest
import torch

from test_gpu_kv import Pool, _tokens, pace  # noqa: F401
from test_gpu_kv_tree import _ids, tree
from test_gpu_streams import _taken_early

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("count", [1, 60])
def test_scratch_and_outputs_are_kept(pace, monkeypatch, count):  # noqa: F811
    pool = Pool(pace, 110, [3000, 900], 2, 64, 16, poison=False)
    Q, parents, tokens = _tokens(111, 2 * count, 14, 64), _ids(2 * tree("random", count)), _ids([1] * 2 * count)
    cu, seen = [0, count, 2 * count], []
    kept = pace._workspace
    monkeypatch.setattr(pace, "_workspace", lambda *a: seen.append(kept(*a)) or seen[-1])

    def make(side):
        out = pace.pace_kv_tree_attention(pool.cache, Q, cu, parents, pool.lens, pool.table, 3000, stream=side)
        rows, counts, after = pace.pace_draft_accept(tokens, parents, tokens, cu, stream=side)
        lens = pace.pace_kv_compact(pool.cache, cu, pool.lens, pool.table, stream=side)
        mine = [(t.numel() * t.element_size(), t.data_ptr()) for t in (out, rows, counts, after, lens, seen[0][0])]
        seen.clear()
        return mine

    assert _taken_early(make) == []
    assert pace.pace_device_status(clear=True) == (0, 0)


def test_two_streams_at_once(pace):  # noqa: F811
    """Each with a workspace of its own, over one cache that neither writes; and a move that both read from, to pages of their own."""
    pool = Pool(pace, 112, [2500, 700, 64, 64], 2, 64, 16, poison=False)
    cases = [(_tokens(113 + i, 90, 8, 64), _ids(tree("random", 30, i) + tree("forest", 60, i))) for i in range(2)]
    lens, table = pool.lens[:2].clone(), pool.table[:2].contiguous()
    want = [pace.pace_kv_tree_attention(pool.cache, q, [0, 30, 90], p, lens, table, 2500) for q, p in cases]
    n = pace.pace_kv_tree_attention_workspace_size(pool.cache, [0, 30, 90], 8, 2500)
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    one, here = lens[:1].clone(), table[:1].contiguous()
    there = []
    for i in range(2):      # the last 52 slots of the first sequence, from slot 2448, a page's first
        t = here.clone()
        t[0, 153:157] = pool.table[2 + i, :4]
        there.append(t)
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, (q, p) in enumerate(cases):
            got[i].append(pace.pace_kv_tree_attention(pool.cache, q, [0, 30, 90], p, lens, table, 2500, ws=ws[i], stream=streams[i]))
            pace.pace_kv_compact(pool.cache, [0, 52], one, here, dst_table=there[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])
    x = pool.cache.k.view(torch.uint8)
    for j in range(4):
        a, b = (x[pool.table[2 + i, j].item()] for i in range(2))
        assert torch.equal(a[:, :16 if j < 3 else 4], b[:, :16 if j < 3 else 4])
    assert pace.pace_device_status(clear=True) == (0, 0)
