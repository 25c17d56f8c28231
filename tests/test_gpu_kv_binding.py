"""What the binding of the calls on the paged cache refuses before anything reaches the library."""
import pytest
import torch

from test_gpu_kv import pace  # noqa: F401

pytestmark = pytest.mark.gpu


def test_caches_whose_pages_overlap(pace):  # noqa: F811
    codes, scales = torch.zeros(6, 2, 32, 64, dtype=torch.uint8, device="cuda"), torch.zeros(6, 2, 2, device="cuda")
    pace.KvCache(codes, codes.clone(), scales, scales.clone())
    one = torch.as_strided(codes, (1, 2, 32, 64), (0, 2048, 64, 1))
    assert pace.KvCache(one, one, scales[:1], scales[:1]).view.page_stride == 4096      # (of a single page the distance says nothing)
    same, near = codes[:1].expand(6, -1, -1, -1), torch.as_strided(codes, (3, 2, 32, 64), (2048, 2048, 64, 1))
    for k, s in ((same, scales), (near, scales[:3]), (codes, scales[:1].expand(6, -1, -1)), (codes[:0], scales[:0])):
        with pytest.raises(ValueError):
            pace.KvCache(k, k, s, s)


def test_rotation_tables_that_do_not_fit(pace):  # noqa: F811
    good = torch.empty(10, 32, 2, device="cuda")
    assert pace.pace_rope_table(10, 64, out=good) is good
    for bad in (good[:9], good.to(torch.bfloat16), good.double()):
        with pytest.raises(ValueError):
            pace.pace_rope_table(10, 64, out=bad)
