"""Sizes of the 8-bit cache's calls that are refused by name, before anything is enqueued."""
import pytest

from .test_abi_cpu import lib  # noqa: F401
from .test_kv8_cpu import INVALID, UNSUPPORTED, append, attention, cache, status


@pytest.mark.parametrize("rows,nkv,hd,dtype", [(1 << 22, 512, 64, 1), (1 << 22, 128, 128, 0), (1 << 21, 256, 64, 1)])
def test_an_append_larger_than_a_grid_is_refused(lib, rows, nkv, hd, dtype):  # noqa: F811
    c = cache(n_kv_heads=nkv, head_dim=hd, page_stride=32 * nkv * hd, scale_stride=2 * nkv)
    a = append(rows=rows, dtype=dtype, q=None, n_q_heads=0, k_stride=nkv * hd, v_stride=nkv * hd)
    assert status(lib, "osprey_kv8_append", c, a) == UNSUPPORTED
    assert b"grid" in lib.osprey_last_error()


def test_a_softmax_scale_that_is_no_float_to_base_2_is_refused(lib):  # noqa: F811
    for scale in (3.0e38, 2.4e38):
        assert status(lib, "osprey_kv8_attention", cache(), attention(scale=scale)) == INVALID
    assert status(lib, "osprey_kv8_attention", cache(), attention(scale=2.3e38, q=None)) == INVALID and b"q is NULL" in lib.osprey_last_error()
