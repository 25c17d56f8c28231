"""Append to the paged cache, bit for bit: every product and sum of the rotation rounded to fp32 by itself."""
import numpy as np
import pytest
import torch

from oracle import pace_oracle as O
from test_gpu_kv import BF16, Pool, _cu, _f64, _tokens, pace, rotation  # noqa: F401

pytestmark = pytest.mark.gpu


def _turn32(x, cs):
    """x [tokens, heads, D] turned in fp32, one rounding per operation."""
    a, b = np.split(x.astype(np.float32), 2, axis=2)
    c, s = cs[:, None, :, 0].astype(np.float32), cs[:, None, :, 1].astype(np.float32)
    y = np.concatenate([a * c - b * s, b * c + a * s], axis=2)
    assert y.dtype == np.float32
    return y


@pytest.mark.parametrize("heads,dim", [(4, 128), (2, 64)])
@pytest.mark.parametrize("first,count", [(0, 3000), (7, 1)])
def test_rotated_keys_and_queries(pace, heads, dim, first, count):  # noqa: F811
    pool = Pool(pace, 60, [first + count], heads, dim, 64, poison=False)
    K, V, q = _tokens(61, count, heads, dim), _tokens(62, count, heads, dim), _tokens(63, count, 3 * heads, dim)
    kw, angles = rotation(pace, dim, count, 64)
    q_out = pace.pace_kv_append(pool.cache, K, V, _cu([count]), pool.lens, pool.table, q=q, **kw)
    cs = angles(np.arange(count))
    for n, x in (("k", _turn32(_f64(K), cs)), ("v", _f64(V))):
        values, scales = pool.values(n).copy(), pool.s[n].copy()
        O.kv_append(values, scales, x, first, pool.pages[0])
        codes, got = pool.now(n)
        np.testing.assert_array_equal(got, scales)
        np.testing.assert_array_equal(O.e4m3_values()[codes], values)
    want = torch.from_numpy(_turn32(_f64(q), cs)).to(BF16)
    assert torch.equal(q_out.cpu(), want)


# as many query heads as attention takes
@pytest.mark.parametrize("hq", [256, 257, 320, 1000, 16384])
def test_queries_of_many_heads(pace, hq):  # noqa: F811
    pool = Pool(pace, 65, [19, 3], 1, 64, 16, poison=False)
    K, q = _tokens(66, 22, 1, 64), _tokens(67, 22, hq, 64)
    kw, angles = rotation(pace, 64, 22, 68)
    q_out = pace.pace_kv_append(pool.cache, K, K, [0, 19, 22], pool.lens, pool.table, q=q, **kw)
    assert torch.equal(q_out.cpu(), torch.from_numpy(_turn32(_f64(q), angles(np.arange(22)))).to(BF16))
