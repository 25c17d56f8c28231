"""What the calls on the paged cache refuse for its size, before anything is launched."""
import ctypes

import pytest

from paper_2608_27206_gb300 import pace as P
from test_kv_cpu import call  # noqa: F401

WIDE = dict(page_size=256, n_kv_heads=256, page_stride=256 * 256 * 128, scale_stride=256 * 16)
EDGE = ((2 ** 31 - 1) // 256 - 3) * 128      # longest max_len of one row tile with 256 KV heads


def _prefix(n):
    cu = (ctypes.c_int32 * (len(n) + 1))()
    for i, x in enumerate(n):
        cu[i + 1] = cu[i] + x
    return cu


# one row tile too long; two of them half as long; the second launch of a form (256 sequences on), the second form
@pytest.mark.parametrize("new,max_len,ok", [([1], EDGE, True), ([1], EDGE + 1, False), ([1, 1], EDGE // 2 - 512, True), ([1, 1], EDGE // 2 + 512, False),
                                            ([1] * 256 + [1] * 100, 1 << 21, True), ([1] * 256 + [512] * 256, 1 << 21, False),
                                            ([1, 40 * 256], EDGE // 40 - 1024, True), ([1, 40 * 256], EDGE // 40 + 1024, False)])
def test_attention_refuses_more_than_a_launch_takes(call, new, max_len, ok):  # noqa: F811
    c, cu = call.cache(**WIDE), _prefix(new)
    size = call.L.pace_kv_attention_workspace_size(ctypes.addressof(c), ctypes.addressof(cu), len(new), 256, max_len)
    assert (size > 0) == ok
    if not ok:
        got = call.attend(c=c, cu=ctypes.addressof(cu), B=len(new), hq=256, qs=256 * 128, ts=1 << 22, max_len=max_len)
        assert got == P.PACE_ERR_INVALID_ARG
