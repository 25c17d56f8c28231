"""Tokens kept in place where a warp's blocks end and a CTA's begin: lists with room for 49 tokens touch four blocks of 16 slots at most, with room for 50 five."""
import numpy as np
import pytest

from test_gpu_kv import _cu, pace  # noqa: F401
from test_gpu_kv_compact import Case, _ids

pytestmark = pytest.mark.gpu


# every place in a block that the first token may land at, with the whole list kept or a few
@pytest.mark.parametrize("room", [1, 16, 17, 33, 48, 49, 50])
@pytest.mark.parametrize("few", [False, True])
@pytest.mark.parametrize("heads,dim,page,layers", [(4, 128, 32, 2), (3, 64, 16, 3)])
def test_every_first_slot(pace, room, few, heads, dim, page, layers):  # noqa: F811
    nodes = [room] * 16
    lens = [16 + b + room for b in range(16)]
    keep = [min(room, 3) if few else room] * 16
    case = Case(pace, 40, lens, nodes, keep, heads, dim, page, layers=layers)
    cu = _cu(nodes)
    rows = np.full(cu[-1], -1)
    for b, k in enumerate(case.kept):
        rows[cu[b]:cu[b] + len(k)] = k + cu[b]
    case.check(case.call(cu_rows=None, rows=_ids(rows), counts=_ids(keep)))      # the list's room is the sequence's nodes


# lists with less room than there are nodes: the tokens come from far behind where they go
@pytest.mark.parametrize("room", [49, 50])
def test_from_far_behind(pace, room):  # noqa: F811
    case = Case(pace, 41, [400 + b for b in range(16)], [370 + b % 3 for b in range(16)], [room] * 16, 2, 128, 64)
    case.check(case.call())
    assert pace.pace_device_status(clear=True) == (0, 0)
