"""Calls on another stream than the current one: what they allocate themselves is theirs from their first kernel to their last."""
import pytest
import torch

from test_gpu_kv import Pool, _tokens, pace  # noqa: F401

pytestmark = pytest.mark.gpu


def _taken_early(make):
    """Whether memory that make(stream) has allocated and let go of is handed out while the stream is still busy."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    make(side)      # (modules load and the allocator gets its memory: both wait for the device)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)      # some 50 ms
    sizes = make(side)
    assert torch.cuda.memory_allocated() == before      # all let go of
    busy = not side.query()
    again = [torch.empty(n, dtype=torch.uint8, device="cuda").data_ptr() for n, _ in sizes]      # (nothing is written there)
    side.synchronize()
    assert busy
    return [p for p, (_, q) in zip(again, sizes) if p == q]


@pytest.mark.parametrize("count", [1, 60])
def test_scratch_and_outputs_are_kept(pace, monkeypatch, count):  # noqa: F811
    pool = Pool(pace, 80, [3000, 900], 2, 64, 16, poison=False)
    x = _tokens(81, 2 * count, 18, 64)
    cu, seen = [0, count, 2 * count], []
    kept = pace._workspace
    monkeypatch.setattr(pace, "_workspace", lambda *a: seen.append(kept(*a)) or seen[-1])

    def make(side):
        q = pace.pace_kv_append(pool.cache, x[:, 14:16], x[:, 16:], cu, pool.lens, pool.table, q=x[:, :14], stream=side)
        out = pace.pace_kv_attention(pool.cache, q, cu, pool.lens, pool.table, 3000, stream=side)
        mine = [(t.numel() * t.element_size(), t.data_ptr()) for t in (q, out, seen[0][0])]
        seen.clear()
        return mine

    assert _taken_early(make) == []
    assert pace.pace_device_status(clear=True) == (0, 0)


def test_statistics_are_not_zeroed_after_the_call(pace):  # noqa: F811
    g = torch.Generator().manual_seed(82)
    img = torch.randint(0, 256, (224 * 224 * 3,), dtype=torch.uint8, generator=g).cuda()
    d, stats = pace.pace_apc_density(img, [0], [224], [224])
    want = stats.clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)      # the current stream is busy for some 50 ms
    _, got = pace.pace_apc_density(img, [0], [224], [224], stream=side)
    torch.cuda.synchronize()
    assert want.any() and torch.equal(got, want)
