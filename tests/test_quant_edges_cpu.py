"""What the binding refuses of a cache's tensors before any call is made with them."""
import pytest
import torch

import paper_2606_26631_gb300 as prcr


def _t(shape, dtype=torch.bfloat16, device="cpu"):
    return torch.zeros(shape, dtype=dtype, device=device)


def test_caches_are_on_one_device():
    """A tensor of another device is an address that means nothing on this one: descriptors are not made of both."""
    i32, u8, e4 = torch.int32, torch.uint8, torch.float8_e4m3fn
    wide, table = _t((3, 2, 9, 2, 64)), _t((3, 4), i32)
    codes, scales = _t((3, 2, 9, 2, 64), e4), _t((3, 2, 9, 2, 1), u8)
    prcr.cache_paged(wide, wide, table)
    prcr.qcache_paged(codes, codes, scales, scales, table)
    with pytest.raises(ValueError, match="device"):
        prcr.cache_paged(wide, wide, table.to("meta"))
    with pytest.raises(ValueError, match="device"):
        prcr.cache_paged(wide, wide.to("meta"), table)
    with pytest.raises(ValueError, match="device"):
        prcr.cache_contiguous(wide, wide.to("meta"))
    with pytest.raises(ValueError, match="device"):
        prcr.qcache_paged(codes, codes, scales, scales, table.to("meta"))
    for i in range(1, 4):
        parts = [codes, codes, scales, scales]
        parts[i] = parts[i].to("meta")
        with pytest.raises(ValueError, match="device"):
            prcr.qcache_paged(*parts, table)
        with pytest.raises(ValueError, match="device"):
            prcr.qcache_contiguous(*parts)


def test_a_quantised_cache_has_a_row_of_blocks_for_each_sequence():
    codes, scales = _t((3, 2, 9, 2, 32), torch.uint8), _t((3, 2, 9, 2, 2), torch.uint8)
    for shape in ((4,), (1, 3, 4)):
        with pytest.raises(ValueError, match="max_blocks"):
            prcr.qcache_paged(codes, codes, scales, scales, _t(shape, torch.int32))
