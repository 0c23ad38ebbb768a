"""Appends of a part of a packed batch, in both forms of the queries (one row and four a wavefront)."""
import pytest
import torch

from .test_gpu_kv8 import BF, DEV, F32, bd, gen_of, ints, make_cache, tables

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("first", [1, 6, 4099])
@pytest.mark.parametrize("rows", [[3, 2], [18000, 3]])
def test_queries_of_a_part_of_a_batch_are_those_of_the_part_alone(rows, first, dtype):
    hd, nq, nkv, behind = 64, 8, 1, 5
    n, total = sum(rows), first + sum(rows) + behind
    gen = gen_of(n)
    k, v = (torch.randn((total, nkv, hd), generator=gen, device=DEV).to(dtype) for _ in range(2))
    q = torch.randn((total, nq, hd), generator=gen, device=DEV).to(dtype)
    q[:first] = float("nan")
    gain = (1 + 0.2 * torch.randn(hd, generator=gen, device=DEV)).to(dtype)
    cos, sin = (t.to(DEV) for t in tables(max(rows), hd))
    got = []
    for lo, hi in ((0, total), (first, first + n)):
        cache = make_cache(2, max(rows) // 16 + 1, nkv, hd, 5)
        out = torch.full((hi - lo, nq, hd), 7.0, dtype=dtype, device=DEV)
        cu = ints([first - lo, first - lo + rows[0], first - lo + n])
        bd().kv8_append(cache, k[lo:hi], v[lo:hi], ints([0, 0]), q=q[lo:hi], q_out=out, cu_rows=cu, q_norm=gain, rope_cos=cos, rope_sin=sin)
        got.append((out, cache))
    (whole, a), (part, b) = got
    assert torch.equal(whole[first:first + n], part)
    assert bool((whole[:first] == 7.0).all()) and bool((whole[first + n:] == 7.0).all())
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales.nan_to_num(), b.scales.nan_to_num())


@pytest.mark.parametrize("hd", [64, 128])
def test_a_rejected_rows_mark_on_its_page_and_the_copy_that_undoes_it(hd):
    """A dropped row with a large key leaves the page's older codes rounded to its scale; pages put back are as
    they were, and rows that are appended again then are what they would have been without the draft."""
    nkv, n = 2, 21
    gen = gen_of(9)
    k, v = (torch.randn((n + 1, nkv, hd), generator=gen, device=DEV) for _ in range(2))
    cache, other = make_cache(1, 3, nkv, hd, 5), make_cache(1, 3, nkv, hd, 5)
    for c in (cache, other):
        bd().kv8_append(c, k[:n], v[:n], ints([0]), cu_rows=ints([0, n]))
    page = int(cache.page_table[0, 1])
    before = cache.codes[page].clone(), cache.scales[page].clone()
    bd().kv8_append(cache, k[n:] * 4096.0, v[n:], ints([n]))                    # a draft
    assert bool((cache.scales[page, :, 0] > before[1][:, 0]).all())
    assert not torch.equal(cache.codes[page, 0].view(nkv, 16, hd)[:, :5], before[0][0].view(nkv, 16, hd)[:, :5])
    cache.codes[page], cache.scales[page] = before
    for c in (cache, other):
        bd().kv8_append(c, k[n:], v[n:], ints([n]))
    assert torch.equal(cache.codes, other.codes) and torch.equal(cache.scales.nan_to_num(), other.scales.nan_to_num())
