"""A serving layer after a call that it refused: as it was before, and ready for the next."""
import pytest
import torch

from oracle import pace_oracle as O
from test_gpu_serve import HKV, HQ, _tokens, serve  # noqa: F401
from test_gpu_serve_trees import _ids, _layer, _read, check, layer_queries

pytestmark = pytest.mark.gpu

PARENTS, CU = [-1, 0, 0, 1, -1, 0], [0, 4, 6, 6]      # trees of four and two nodes, and a sequence without


def _kvq(n, seed=0):
    return _tokens(seed + 1, n, HKV), _tokens(seed + 2, n, HKV), _tokens(seed + 3, n, HQ)


def _begun(S):
    layer = _layer(S)
    layer.prompt(*_kvq(30), [0, 19, 26, 30], _ids([list(range(30))] * 3))
    return layer


def _state(layer):
    c = layer.cache
    return [layer.lens.clone()] + [x.view(torch.uint8).clone() for x in (c.k, c.v, c.k_scale, c.v_scale)]


def _as_before(layer, was):
    assert all(torch.equal(a, b) for a, b in zip(_state(layer), was))
    assert layer.lens.tolist() == layer._lengths()
    layer.check()


BAD = ["K's type", "K on the host", "rows of V", "heads of K", "rows of Q", "heads of Q", "type of ids", "number of ids"]


def _bad_tokens(n, what):
    """Arguments K, V, Q, positions that no call takes, `what` of them wrong."""
    k, v, q = _kvq(n)
    pos = torch.zeros(3, n, dtype=torch.int32, device="cuda")
    return {"K's type": (k.float(), v, q, pos), "K on the host": (k.cpu(), v, q, pos), "rows of V": (k, v[:-1], q, pos), "heads of K": (k[:, :1], v, q, pos),
            "rows of Q": (k, v, q[:-1], pos), "heads of Q": (k, v, torch.cat([q, q[:, :1]], 1), pos), "type of ids": (k, v, q, pos.long()),
            "number of ids": (k, v, q, pos[:, :-1].contiguous())}[what]


@pytest.mark.parametrize("what", BAD + ["parents of 64 bits", "parents on the host", "parents too few", "parents apart"])
def test_a_refused_draft_changes_nothing(serve, what):  # noqa: F811
    layer, n = _begun(serve), CU[-1]
    k, v, q = _kvq(n, 10)
    parents, pos = _ids(PARENTS), _ids([[19, 20, 20, 21, 7, 8]] * 3)
    bad = {"parents of 64 bits": parents.long(), "parents on the host": parents.cpu(), "parents too few": parents[:-1].contiguous(),
           "parents apart": torch.stack([parents, parents], 1)[:, 0]}
    if what in bad:
        args = (k, v, q, bad[what], CU, pos)
    else:
        *kvq, ids = _bad_tokens(n, what)
        args = (*kvq, parents, CU, ids)
    was = _state(layer)
    with pytest.raises(ValueError):
        layer.draft(*args)
    _as_before(layer, was)
    with pytest.raises(ValueError):      # nothing is pending
        layer.accept(_ids([0] * n), _ids([0] * n))
    # the next one works
    out = layer.draft(k, v, q, parents, CU, pos)
    assert layer.lens.tolist() == [23, 9, 4]
    for b in range(2):
        mine = slice(CU[b], CU[b + 1])
        turned = layer_queries(layer, q[mine], pos.cpu().numpy()[:, mine])
        check(layer, b, turned, O.kv_tree_visible(int(layer.lens[b]), PARENTS[mine], 0, 0), out[mine])
    _rows, counts, _after = layer.accept(_ids([5, 6, 7, 8, 5, 9]), _ids([7, 0, 1, 0, 9, 0]))      # node 2 after node 0; node 1 after node 0
    assert counts.tolist() == [2, 2, 0] and layer.lens.tolist() == layer._lengths() == [21, 9, 4]
    layer.check()


@pytest.mark.parametrize("what", BAD + ["rows on the host"])
def test_a_refused_prompt_changes_nothing(serve, what):  # noqa: F811
    layer, cu = _begun(serve), [0, 2, 2, 5]
    good = (*_kvq(5, 20), _ids([[30] * 5] * 3))
    args, kw = (good, dict(rows=torch.arange(5, dtype=torch.int32))) if what == "rows on the host" else (_bad_tokens(5, what), {})
    was = _state(layer)
    with pytest.raises(ValueError):
        layer.prompt(*args[:3], cu, args[3], **kw)
    _as_before(layer, was)
    other = _begun(serve)
    a, b = (x.prompt(*good[:3], cu, good[3]) for x in (layer, other))
    assert torch.equal(a, b) and layer.lens.tolist() == layer._lengths() == [21, 7, 7]
    assert all((_read(layer, name, i) == _read(other, name, i)).all() for name in "kv" for i in range(3))


@pytest.mark.parametrize("what", BAD + ["fewer heads of Q"])
def test_a_refused_step_changes_nothing(serve, what):  # noqa: F811
    layer = _begun(serve)
    good = (*_kvq(3, 30), _ids([[30] * 3] * 3))
    args = (good[0], good[1], good[2][:, :HKV], good[3]) if what == "fewer heads of Q" else _bad_tokens(3, what)
    was = _state(layer)
    with pytest.raises(ValueError):
        layer.step(*args)
    _as_before(layer, was)
    other = _begun(serve)
    assert torch.equal(layer.step(*good).clone(), other.step(*good))
    assert layer.lens.tolist() == layer._lengths() == [20, 8, 5]


def test_a_replay_that_fails_is_not_counted(serve):  # noqa: F811
    layer = _begun(serve)
    graph = serve.CapturedStep()      # (nothing captured)
    graph.layer = layer
    was = _state(layer)
    with pytest.raises(RuntimeError):
        graph.replay()
    _as_before(layer, was)


@pytest.mark.parametrize("call", ["draft", "prompt"])
def test_a_call_that_fails_behind_the_append_takes_its_tokens_back(serve, monkeypatch, call):  # noqa: F811
    """As when the attention's scratch has no room: the tokens lie behind the sequences' ends."""
    layer = _begun(serve)
    k, v, q = _kvq(CU[-1], 40)
    pos = _ids([[19, 20, 20, 21, 7, 8]] * 3)
    run = (lambda: layer.draft(k, v, q, _ids(PARENTS), CU, pos)) if call == "draft" else (lambda: layer.prompt(k, v, q, CU, pos))
    before = [_read(layer, "v", b) for b in range(3)]

    def full(*_a, **_k):
        raise torch.cuda.OutOfMemoryError("no room")
    with monkeypatch.context() as m:
        m.setattr(serve.P, "pace_kv_tree_attention", full)
        m.setattr(serve.P, "pace_kv_attention", full)
        with pytest.raises(torch.cuda.OutOfMemoryError):
            run()
    assert layer.lens.tolist() == layer._lengths() == [19, 7, 4]
    for b in range(3):      # (a block's scale may have grown for the tokens beside it: a value is then off by half a step of the new one, 2^-4 of it at most,
        was, now = before[b], _read(layer, "v", b)      # or by half of the smallest code, 2^-10 of a scale that is at most 1/224 of the largest value there)
        most = max(float(v.abs().max()), abs(was).max(initial=0.0))
        assert (abs(was - now) <= 2.0 ** -4 * abs(was) + 2.0 ** -10 * most / 224).all()
    run()
    assert layer.lens.tolist() == [23, 9, 4]
    layer.check()
