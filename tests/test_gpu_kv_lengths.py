"""Lengths on the device that no sequence can have: reported, and nothing but their own tokens is lost."""
import numpy as np
import pytest
import torch

from test_gpu_kv import Pool, _tokens, check_append, pace  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("length", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 15, 2 ** 31 - 17, 2 ** 31 - 100, 2 ** 30, 33, -1, -2 ** 31, -2 ** 31 + 5])
@pytest.mark.parametrize("count", [1, 20])
def test_append_behind_the_table(pace, length, count):  # noqa: F811
    pool = Pool(pace, 70, [32, 32], 2, 64, 16, poison=False)
    K, V = _tokens(71, 2 * count, 2, 64), _tokens(72, 2 * count, 2, 64)
    lens = torch.tensor([length, 32], dtype=torch.int32, device="cuda")
    pace.pace_kv_append(pool.cache, K, V, [0, count, 2 * count], lens, pool.table)
    assert pace.pace_device_status(clear=True) == (pace.PACE_ERR_INVALID_ARG, 14)
    if length != 33:      # (with 33 slots the tokens before the last one have their place)
        check_append(pool, [0, count], K[count:], V[count:])


@pytest.mark.parametrize("length", [-1, -2 ** 31, 301, 2 ** 31 - 1])
@pytest.mark.parametrize("count,hq", [(1, 4), (60, 4)])
def test_attention_of_no_such_length(pace, length, count, hq):  # noqa: F811
    pool = Pool(pace, 73, [300, 250], 2, 64, 16)
    Q = _tokens(74, 2 * count, hq, 64)
    args = (pool.cache, Q, [0, count, 2 * count])
    good = pace.pace_kv_attention(*args, pool.lens, pool.table, 300).clone()
    assert pace.pace_device_status(clear=True) == (0, 0)
    lens = torch.tensor([length, 250], dtype=torch.int32, device="cuda")
    got = pace.pace_kv_attention(*args, lens, pool.table, 300)
    assert pace.pace_device_status(clear=True) == (pace.PACE_ERR_INVALID_ARG, 15)
    assert torch.equal(got[count:], good[count:])
