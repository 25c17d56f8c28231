"""The size of a launch of the attention from trees: what the header states is what the calls take."""
import ctypes
import os
import re

import pytest

from paper_2608_27206_gb300 import pace as P
from test_abi_cpu import HEADER
from test_kv_cpu import call  # noqa: F401
from test_kv_limits_cpu import WIDE, _prefix
from test_kv_tree_cpu import attend


def _stated():
    """Places of a row tile and head beside its slot tiles, as include/pace.h gives them for trees."""
    assert os.path.exists(HEADER)
    text = open(HEADER).read().split("pace_kv_tree_attention_workspace_size")[1].split("pace_kv_tree_attention(")[0]
    return int(re.search(r"max_len \+ (\d+)\) < 2\^31", re.sub(r"\s*\n \*\s*", " ", text)).group(1))


# one row tile; three of one tree; many trees, a launch of 256 after another; few rows and many
@pytest.mark.parametrize("nodes,tiles", [([1], 1), ([20], 1), ([600], 3), ([20] * 256 + [20] * 100, 256), ([1, 20] * 100, 100)])
def test_tree_attention_takes_what_the_header_states(call, nodes, tiles):  # noqa: F811
    c, cu = call.cache(**WIDE), _prefix(nodes)
    most = ((2 ** 31 - 1) // (256 * tiles) - _stated()) * 128      # the longest max_len with row tiles * 256 heads * (tiles + stated) < 2^31

    def size(max_len):
        return call.L.pace_kv_tree_attention_workspace_size(ctypes.addressof(c), ctypes.addressof(cu), len(nodes), 256, max_len)
    assert size(most) > 0 and size(most + 1) == 0
    assert attend(call, c=c, cu=ctypes.addressof(cu), B=len(nodes), hq=256, qs=256 * 128, ts=1 << 23, max_len=most + 1) == P.PACE_ERR_INVALID_ARG
