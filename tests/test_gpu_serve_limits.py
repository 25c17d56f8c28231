"""What a serving layer refuses: tokens past its last slot, by whichever way they come; and what its calls report."""
import pytest
import torch

from test_gpu_serve import D, HKV, HQ, _tokens, serve  # noqa: F401

pytestmark = pytest.mark.gpu


def _layer(S, max_len):
    layer = S.ServeLayer(2, max_len, page_size=16, n_q_heads=HQ, n_kv_heads=HKV, head_dim=D, max_positions=100)
    ids = torch.zeros(3, 40, dtype=torch.int32, device="cuda")
    return layer, ids


def _kvq(n):
    return _tokens(1, n, HKV), _tokens(2, n, HKV), _tokens(3, n, HQ)


def _refused(layer, call):
    lens, codes = layer.lens.clone(), layer.cache.k.view(torch.uint8).clone()
    with pytest.raises(ValueError):
        call()
    assert torch.equal(layer.lens, lens) and torch.equal(layer.cache.k.view(torch.uint8), codes)
    layer.check()


def test_prompts_end_at_the_last_slot(serve):  # noqa: F811
    layer, ids = _layer(serve, 20)
    layer.prompt(*_kvq(22), [0, 17, 22], ids[:, :22].contiguous())
    _refused(layer, lambda: layer.prompt(*_kvq(5), [0, 4, 5], ids[:, :5].contiguous()))
    layer.prompt(*_kvq(18), [0, 3, 18], ids[:, :18].contiguous())
    assert layer.lens.tolist() == [20, 20]
    _refused(layer, lambda: layer.prompt(*_kvq(1), [0, 0, 1], ids[:, :1].contiguous()))
    _refused(layer, lambda: layer.prompt(*_kvq(1), [0, 1], ids[:, :1].contiguous()))
    layer.reset()
    layer.prompt(*_kvq(22), [0, 17, 22], ids[:, :22].contiguous())
    assert layer.lens.tolist() == [17, 5]
    layer.check()


@pytest.mark.parametrize("graph", [False, True])
def test_steps_end_at_the_last_slot(serve, graph):  # noqa: F811
    layer, ids = _layer(serve, 20)
    layer.prompt(*_kvq(20), [0, 17, 20], ids[:, :20].contiguous())
    one = (*_kvq(2), ids[:, :2].contiguous())
    step = layer.capture_step(*one).replay if graph else lambda: layer.step(*one)
    for _ in range(3):
        step()
    assert layer.lens.tolist() == [20, 6]
    _refused(layer, step)


def test_what_kernels_report(serve):  # noqa: F811
    layer, ids = _layer(serve, 20)
    layer.prompt(*_kvq(4), [0, 2, 4], ids[:, :4].contiguous() + 100)      # ids past the rotation table
    with pytest.raises(RuntimeError):
        layer.check()
    layer.check()
