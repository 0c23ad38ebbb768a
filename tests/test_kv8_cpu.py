"""The 8-bit cache without a GPU: what its calls refuse before anything is enqueued, and the
pins of the float64 description that the GPU tests compare with."""
import ctypes as C
import math

import pytest
import torch

from . import kv8_ref as R
from .test_abi_cpu import lib  # noqa: F401

P = 1 << 20   # an aligned address that no call may follow


def cache(**kw):
    from paper_2609_09338_amd import _lib as L
    c = L.osprey_kv8_cache(P, 2, 4, 9, 8, 128, P, 2 * 8 * 16 * 128, P, 16)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def append(**kw):
    from paper_2609_09338_amd import _lib as L
    a = L.osprey_kv8_append_args(rows=5, cu_rows=P, cached=P, dtype=1, n_q_heads=16, q=P, k=P, v=P, q_stride=4096, k_stride=4096,
                                 v_stride=4096, eps=1e-6, q_out=2 * P, q_out_stride=2048)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def attention(**kw):
    from paper_2609_09338_amd import _lib as L
    a = L.osprey_kv8_attention_args(rows=5, max_rows=3, max_context=64, cu_rows=P, cached=P, dtype=1, n_q_heads=16, q=P, q_stride=2048,
                                    scale=0.1, out=P, out_stride=2048, workspace=P, workspace_bytes=1 << 30)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def status(lib, fn, c, a):
    return getattr(lib, fn)(C.byref(c), C.byref(a), None)


INVALID, SHAPE, UNSUPPORTED = -1, -2, -6


def test_the_entry_points_are_declared_exported_and_bound(lib):  # noqa: F811
    import os
    from paper_2609_09338_amd import _lib as L
    src = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "osprey.h")).read()
    for n in ("osprey_kv8_append", "osprey_kv8_workspace_bytes", "osprey_kv8_attention", "osprey_kv8_keep"):
        assert n + "(" in src and hasattr(lib, n) and n in L.SIGNATURES


@pytest.mark.parametrize("kw,want", [
    (dict(page_table=None), INVALID), (dict(codes=None), INVALID), (dict(scales=None), INVALID), (dict(batch=0), INVALID),
    (dict(batch=4097), INVALID), (dict(max_pages=0), INVALID), (dict(max_pages=(1 << 25) + 1), INVALID), (dict(num_pages=0), INVALID),
    (dict(n_kv_heads=0), SHAPE), (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED), (dict(codes=P + 8), INVALID),
    (dict(page_stride=2 * 8 * 16 * 128 + 8), INVALID), (dict(page_stride=2 * 8 * 16 * 128 - 16), SHAPE), (dict(scales=P + 2), INVALID),
    (dict(scale_stride=15), SHAPE),
])
def test_caches_that_every_call_refuses(lib, kw, want):  # noqa: F811
    from paper_2609_09338_amd import _lib as L
    c = cache(**kw)
    assert status(lib, "osprey_kv8_append", c, append()) == want
    assert lib.osprey_last_error()
    assert status(lib, "osprey_kv8_attention", c, attention()) == want
    assert status(lib, "osprey_kv8_keep", c, L.osprey_kv8_keep_args(P, P, 4, P, None)) == want
    assert lib.osprey_kv8_workspace_bytes(C.byref(c), 5, 16, 3, 64) == 0


@pytest.mark.parametrize("kw,want", [
    (dict(cached=None), INVALID), (dict(rows=-1), INVALID), (dict(cu_rows=None), SHAPE), (dict(dtype=2), INVALID), (dict(k=None), INVALID),
    (dict(v=None), INVALID), (dict(k=P + 2), INVALID), (dict(v_stride=4097), INVALID), (dict(k_stride=1016), SHAPE),
    (dict(n_q_heads=0), SHAPE), (dict(q_out=None), INVALID), (dict(q_stride=2040), SHAPE), (dict(q_out_stride=2046), INVALID),
    (dict(q_out=P), INVALID), (dict(q_norm=P, eps=0.0), INVALID), (dict(k_norm=P, eps=math.nan), INVALID), (dict(rope_cos=P), INVALID),
    (dict(rope_cos=P, rope_sin=P, rope_len=0), INVALID), (dict(rows=(1 << 22) + 1), INVALID),
    (dict(rows=1 << 22, n_q_heads=128, q_stride=1 << 20, q_out_stride=1 << 20), UNSUPPORTED),
])
def test_appends_that_are_refused(lib, kw, want):  # noqa: F811
    assert status(lib, "osprey_kv8_append", cache(), append(**kw)) == want
    assert status(lib, "osprey_kv8_append", cache(), append(rows=0)) == 0   # nothing to do


@pytest.mark.parametrize("kw,want", [
    (dict(cached=None), INVALID), (dict(rows=-1), INVALID), (dict(cu_rows=None), SHAPE), (dict(n_q_heads=12), SHAPE),
    (dict(n_q_heads=0), SHAPE), (dict(dtype=-1), INVALID), (dict(max_rows=0), INVALID), (dict(max_context=0), INVALID),
    (dict(tree_mask=P, max_rows=129), SHAPE), (dict(tree_mask=P + 4), INVALID), (dict(scale=0.0), INVALID), (dict(scale=math.inf), INVALID),
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(q=P + 8), INVALID), (dict(out_stride=2047), INVALID), (dict(q_stride=1024), SHAPE),
])
def test_attention_calls_that_are_refused(lib, kw, want):  # noqa: F811
    assert status(lib, "osprey_kv8_attention", cache(), attention(**kw)) == want


def test_kept_paths_that_are_refused(lib):  # noqa: F811
    from paper_2609_09338_amd import _lib as L
    for a in ((None, P, 4, P), (P, None, 4, P), (P, P, 4, None)):
        assert status(lib, "osprey_kv8_keep", cache(), L.osprey_kv8_keep_args(*a, None)) == INVALID
    assert status(lib, "osprey_kv8_keep", cache(), L.osprey_kv8_keep_args(P, P, 0, P, None)) == SHAPE


def test_the_binding_refuses_tensors_of_the_wrong_kind():
    from paper_2609_09338_amd import binding as B
    codes = torch.zeros((3, 2, 4, 16 * 64), dtype=torch.uint8)
    scales, table = torch.ones((3, 4, 2)), torch.zeros((1, 2), dtype=torch.int32)
    for bad in ((codes.float(), scales, table), (codes, scales.double(), table), (codes, scales[:, :3], table), (codes, scales, table.long()),
                (codes[:, :, :, :512], scales, table), (codes, scales, table), (codes.transpose(1, 2).contiguous().transpose(1, 2), scales, table)):
        with pytest.raises(ValueError):   # (host tensors, where nothing else is wrong)
            B.Kv8Cache(*bad, 64)


def test_rounding_to_eight_bits_equals_torch_conversion():
    tab = R.e4m3_values()
    codes = torch.arange(127, dtype=torch.uint8)
    assert torch.equal(tab, codes.view(torch.float8_e4m3fn).double())
    g = torch.Generator().manual_seed(3)
    x = torch.cat([(torch.rand(20000, generator=g, dtype=torch.float64) * 2 - 1) * 448, (tab[1:] + tab[:-1]) / 2, -tab,
                   torch.randn(20000, generator=g, dtype=torch.float64) * 0.02]).float().double()
    assert torch.equal(R.round8(x), x.float().to(torch.float8_e4m3fn).double())


def test_scales_are_the_smallest_powers_of_two():
    assert R.scale_for(448.0) == 1.0 and R.scale_for(448.0000001) == 2.0 and R.scale_for(224.0) == 0.5
    assert R.scale_for(0.0) == 2.0 ** -100 == R.scale_for(1e-40)
    assert R.scale_for(3.4e38) == 2.0 ** 120


def test_value_places_are_a_permutation_with_four_tokens_to_a_dword():
    for hd in (64, 128):
        p = R.value_places(hd)
        assert torch.equal(p.flatten().sort().values, torch.arange(16 * hd))
        assert torch.equal(p[4:8] - p[4:5], torch.arange(4)[:, None].expand(4, hd))


def test_what_is_written_is_read_within_a_rounding():
    codes = torch.zeros((3, 2, 2, 16 * 64), dtype=torch.uint8)
    ref = R.Cache(codes, torch.ones((3, 2, 2)), torch.tensor([[2, 0, 1]]), 64)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn((40, 2, 64), generator=g, dtype=torch.float64) for _ in range(2))
    ref.write(0, 0, k, v)
    kc, vc = ref.context(0, 40)
    for got, x in ((kc, k), (vc, v)):
        x = x.transpose(0, 1)
        # half a step of 4 bits, or of the smallest code at the block's scale
        assert bool(((got - x).abs() <= 2.0 ** -4 * x.abs() + 2.0 ** -10 * ref.s.max()).all())
    for t in (0, 17, 39):
        assert torch.equal(ref.read(0, t)[0], kc[:, t])


def test_attention_of_one_position_returns_its_value_and_of_none_zeros():
    ref = R.Cache(torch.zeros((1, 2, 1, 16 * 64), dtype=torch.uint8), torch.ones((1, 1, 2)), torch.tensor([[0]]), 64)
    x = torch.randn((2, 1, 64), generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    ref.write(0, 0, x, x)
    sees = torch.tensor([[True, False], [False, False]])
    o, _ = R.attention(ref, 0, torch.ones((2, 1, 64)), sees, 0.1, 0.0, 0.0)
    assert torch.equal(o[0, 0], ref.read(0, 0)[1][0]) and bool((o[1] == 0).all())


def test_an_8_bit_configuration_is_valid_and_its_pool_about_half(lib):  # noqa: F811
    from paper_2609_09338_amd import binding as bd
    from .test_abi_cpu import _cfg
    assert bd.config_validate(_cfg(dtype=2)) == 0
    codes = bd.kv_bytes(_cfg()) // 2
    assert bd.kv_bytes(_cfg(dtype=2)) == codes + 256 * 2 * 8 * 2 * 4   # a scale per page, layer, head, keys and values
    assert bd.workspace_bytes(_cfg(dtype=2)) == bd.workspace_bytes(_cfg())
    assert bd.config_validate(_cfg(dtype=3)) == INVALID
