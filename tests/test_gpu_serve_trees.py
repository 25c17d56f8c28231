"""The serving layer with drafted trees, a pruned cache and forked answers."""
import numpy as np
import pytest
import torch

from oracle import pace_oracle as O
from test_gpu_serve import D, HKV, HQ, _cu, _tokens, serve  # noqa: F401

pytestmark = pytest.mark.gpu

DECODE = O.e4m3_values()


def _layer(S, seqs=3, max_len=400, **kw):
    return S.ServeLayer(seqs, max_len, page_size=32, n_q_heads=HQ, n_kv_heads=HKV, head_dim=D, max_positions=900, **kw)


def _ids(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda").contiguous()


def _read(layer, name, b):
    x, s = getattr(layer.cache, name).view(torch.uint8).cpu().numpy(), getattr(layer.cache, name + "_scale").cpu().numpy().astype(np.float64)
    return O.kv_read(DECODE[x], s, layer.table[b].cpu().numpy(), int(layer.lens[b]))


def _tree(n, rng):
    return [-1] + [int(rng.integers(0, t)) for t in range(1, n)] if n else []


def _close(a, b, roundings):
    """Values of two caches that the same numbers have gone to: each rounding is off by 2^-4 of the value or half of the smallest step, 2^-10
    of a scale, which is at most 1/224 of its block's largest value."""
    assert a.shape == b.shape
    most = max(np.abs(a).max(), np.abs(b).max())
    assert np.all(np.abs(a - b) <= roundings * (1.1 * 2.0 ** -4 * np.abs(b) + 2.0 ** -10 * most / 224))


@pytest.mark.parametrize("window,sinks", [(0, 0), (24, 3)])
def test_drafted_and_accepted(serve, window, sinks):  # noqa: F811
    """Rounds of trees: the layer ends as one that was given the accepted tokens in a line, and attends as the oracle does."""
    layer, line = _layer(serve, window=window, sinks=sinks), _layer(serve, window=window, sinks=sinks)
    rng = np.random.default_rng(1)
    first = [40, 0, 7]
    m = sum(first)
    ids = _ids(np.tile(np.concatenate([np.arange(n) for n in first]), (3, 1)))
    for x in (layer, line):
        x.prompt(_tokens(1, m, HKV), _tokens(2, m, HKV), _tokens(3, m, HQ), _cu(first), ids)
    at, accepted = np.array(first), 0
    for r in range(6):
        nodes = [26, 5, 60] if r % 2 else [7, 0, 33]
        cu, n = _cu(nodes), sum(nodes)
        parents = [_tree(x, rng) for x in nodes]
        depth = [np.array([len(f) - 1 for f in O.tree_family(p)], dtype=int) for p in parents]
        pos = np.tile(np.concatenate([d + at[b] for b, d in enumerate(depth)]), (3, 1))
        K, V, Q = _tokens(10 + r, n, HKV), _tokens(30 + r, n, HKV), _tokens(50 + r, n, HQ)
        out = layer.draft(K, V, Q, _ids(sum(parents, [])), cu, _ids(pos))
        for b, p in enumerate(parents):
            if not p:
                continue
            q = layer_queries(layer, Q[cu[b]:cu[b + 1]], pos[:, cu[b]:cu[b + 1]])
            check(layer, b, q, O.kv_tree_visible(int(layer.lens[b]), p, window, sinks), out[cu[b]:cu[b + 1]])
        tokens, picked = rng.integers(0, 3, n), rng.integers(0, 3, n)
        rows, counts, after = layer.accept(_ids(tokens), _ids(picked))
        paths = [O.draft_accept(tokens[cu[b]:cu[b + 1]], parents[b], picked[cu[b]:cu[b + 1]]) for b in range(3)]
        assert counts.tolist() == [len(p) for p in paths]
        pick = np.concatenate([np.array(p, dtype=int) + cu[b] for b, p in enumerate(paths)])
        line.prompt(K, V, Q, _cu([len(p) for p in paths]), _ids(pos), rows=_ids(pick))
        at += [len(p) for p in paths]
        accepted += sum(len(p) for p in paths)
        assert layer.lens.tolist() == line.lens.tolist() == at.tolist()
    assert accepted > 20
    for b in range(3):
        for name in "kv":       # twice rounded in the trees' block and where it went, as often again where a later one raised its scale
            _close(_read(layer, name, b), _read(line, name, b), 5)
    layer.check()


def check(layer, b, q, see, out):
    """A sequence's outputs against the oracle, from what the cache holds: bf16 rounding and weights of 8 bits, twice over; a score's sum of D
    products in fp32."""
    ref = O.kv_attention(q, _read(layer, "k", b), _read(layer, "v", b), see, D ** -0.5)
    score = 2.0 ** -23 * (D + 8) * ref["abs_score"] + 2.0 ** -20
    tol = 2.0 ** -8 * np.abs(ref["out"]) + (2.0 ** -8 + 2 * score[..., None]) * ref["abs_out"] + 2.0 ** -17 * ref["peak"][..., None]
    assert np.all(np.abs(out.float().cpu().numpy().astype(np.float64) - ref["out"]) <= tol)


def layer_queries(layer, Q, pos):
    """Queries as the append rotates and rounds them."""
    cs = O.rope_angles(layer.rope.cpu().numpy(), pos, layer.sections)
    q = O.rope_rotate(Q.float().cpu().numpy().astype(np.float64), cs[..., 0], cs[..., 1])
    return torch.from_numpy(q).to(torch.bfloat16).double().numpy()


def test_pruned(serve):  # noqa: F811
    layer, line = _layer(serve), _layer(serve)
    first, kept = [300, 50, 9], [120, 50, 1]
    m, rng = sum(first), np.random.default_rng(2)
    cu = _cu(first)
    rows = np.concatenate([np.sort(rng.permutation(n)[:k]) + cu[b] for b, (n, k) in enumerate(zip(first, kept))])
    ids = _ids(rng.integers(0, 900, (3, m)))
    K, V, Q = _tokens(60, m, HKV), _tokens(61, m, HKV), _tokens(62, m, HQ)
    layer.prompt(K, V, Q, cu, ids)
    layer.prune(_ids(rows), _cu(kept))
    line.prompt(K, V, Q, _cu(kept), ids, rows=_ids(rows))
    assert layer.lens.tolist() == kept
    for b in range(3):
        for name in "kv":
            _close(_read(layer, name, b), _read(line, name, b), 3)
    one = (_tokens(63, 3, HKV), _tokens(64, 3, HKV), _tokens(65, 3, HQ), _ids(np.full((3, 3), 100)))
    layer.step(*one)
    assert layer.lens.tolist() == [k + 1 for k in kept]
    layer.check()


def test_forked(serve):  # noqa: F811
    layer = _layer(serve, seqs=4)
    first = [70, 0, 33, 5]
    m = sum(first)
    layer.prompt(_tokens(70, m, HKV), _tokens(71, m, HKV), _tokens(72, m, HQ), _cu(first), _ids(np.zeros((3, m))))
    layer.fork(0, [1, 3])
    assert layer.lens.tolist() == [70, 70, 33, 70]
    for name in "kv":
        x = _read(layer, name, 0)
        assert np.array_equal(x, _read(layer, name, 1)) and np.array_equal(x, _read(layer, name, 3))
    # they go on by themselves, each in its own pages
    pos = np.full((3, 4), 70)
    q = _tokens(75, 4, HQ)
    out = layer.step(_tokens(73, 4, HKV), _tokens(74, 4, HKV), q, _ids(pos))
    for b in range(4):
        n = int(layer.lens[b])
        check(layer, b, layer_queries(layer, q[b:b + 1], pos[:, :1]), O.kv_visible(n, 1), out[b:b + 1])
    last = [_read(layer, "k", b)[-1] for b in range(4)]
    assert layer.lens.tolist() == [71, 71, 34, 71] and not np.array_equal(last[0], last[1]) and not np.array_equal(last[1], last[3])
    layer.fork(1, [])
    layer.check()


def test_refusals_and_room(serve):  # noqa: F811
    layer = _layer(serve, seqs=1, max_len=32)
    x = lambda n: (_tokens(80, n, HKV), _tokens(81, n, HKV), _tokens(82, n, HQ))      # noqa: E731
    pos = lambda n: _ids(np.zeros((3, n)))      # noqa: E731
    layer.prompt(*x(10), [0, 10], pos(10))
    with pytest.raises(ValueError):
        layer.accept(_ids([0]), _ids([0]))
    flat = lambda n: _ids([-1] + [0] * (n - 1))      # noqa: E731
    layer.draft(*x(20), flat(20), [0, 20], pos(20))
    for call in (lambda: layer.draft(*x(1), flat(1), [0, 1], pos(1)), lambda: layer.step(*x(1), pos(1)), lambda: layer.prompt(*x(1), [0, 1], pos(1)),
                 lambda: layer.prune(_ids([0]), [0, 1]), lambda: layer.fork(0, [])):
        with pytest.raises(ValueError):
            call()
    assert layer.lens.tolist() == [30]
    layer.accept(_ids([7] * 20), _ids([8] * 20))      # node 0 alone
    assert layer.lens.tolist() == [11]
    layer.draft(*x(20), flat(20), [0, 20], pos(20))   # (the host had counted 30)
    layer.accept(_ids([7] * 20), _ids([7] * 20))      # node 0 and its first child
    assert layer.lens.tolist() == [13]
    with pytest.raises(ValueError):
        layer.draft(*x(20), flat(20), [0, 20], pos(20))
    layer.draft(*x(19), flat(19), [0, 19], pos(19))
    layer.reset()
    for call in (lambda: layer.draft(*x(1), flat(1), [0, 2000], pos(1)), lambda: layer.prune(_ids([0]), [0]), lambda: layer.fork(0, [0]),
                 lambda: layer.fork(0, [1])):
        with pytest.raises(ValueError):
            call()
    layer.prompt(*x(32), [0, 32], pos(32))
    assert layer.lens.tolist() == [32]
    layer.check()


def test_example(serve, capsys):  # noqa: F811
    serve.main(["--visual", "400", "--steps", "10", "--nodes", "26"])
    said = capsys.readouterr().out
    assert "200 of 440" in said and "20 trees of 26" in said
